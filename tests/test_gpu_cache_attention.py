"""Attention over a paged cache on the GPU against its definition in 64 bits."""
import numpy as np
import pytest
import torch

from cache_ref import Case, tolerances

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def check(case, causal=True, scale=None, accumulate=True):
    import paper_2604_02945_amd as msao
    cache, start = case.device(DEV)
    scale = case.dim ** -0.5 if scale is None else scale
    out = torch.full((case.rows, case.heads, case.dim), 7.0, dtype=case.dtype, device=DEV)
    lse = torch.full((case.rows, case.heads), 7.0, device=DEV)
    msao.msao_cache_attention(cache, start, case.max_new, case.q.to(DEV), scale=scale, causal=causal, out=out, lse=lse,
                              accumulate=accumulate)
    torch.cuda.synchronize()
    want, z, weight, mag, span = case.attention(scale, causal)
    tol_z, tol = tolerances(case, mag, span, want)
    got, got_z, got_w = out.double().cpu().numpy(), lse.double().cpu().numpy(), cache.weight.double().cpu().numpy()
    mine = np.arange(case.rows) < case.start[-1]
    assert (got[~mine] == 7).all() and (got_z[~mine] == 7).all()
    empty = np.isinf(z[mine])
    assert (got_z[mine][empty] == -np.inf).all() and (got[mine][empty] == 0).all()
    assert np.abs(got_z[mine][~empty] - z[mine][~empty]).max(initial=0) <= tol_z
    assert np.isfinite(got[mine]).all()
    assert (np.abs(got - want)[mine] <= tol[mine]).all()
    if accumulate:
        # p is off by 2 d relative, and the sum over up to n rows and the addition round
        rows = case.max_new * case.heads // case.kv_heads
        tol_w = (2 * tol_z + (rows + 4) * 2.0 ** -24) * (weight + 1)
        assert (np.abs(got_w - weight) <= tol_w).all()
    else:
        assert torch.equal(cache.weight.cpu(), case.weight)


EDGES = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 64])
def test_single_tokens_at_every_edge_of_a_tile(dtype, page):
    check(Case(1, EDGES, [1] * len(EDGES), 8, 2, 64, page, dtype))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
@pytest.mark.parametrize("heads,kv_heads,dim,page", [(4, 4, 128, 16), (7, 1, 128, 32), (28, 4, 128, 64), (5, 5, 8, 16),
                                                     (8, 2, 72, 32), (12, 3, 96, 16), (6, 2, 136, 64),
                                                     (4, 2, 200, 16), (8, 1, 256, 128), (16, 1, 64, 16)])
def test_heads_dims_and_pages(dtype, causal, heads, kv_heads, dim, page):
    check(Case(2, [130, 7, 0, 33, 1, 500], [3, 7, 0, 1, 1, 6], heads, kv_heads, dim, page, dtype, extra_rows=3), causal)


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
@pytest.mark.parametrize("heads,kv_heads,dim,page", [(6, 1, 64, 16), (4, 2, 88, 32), (3, 1, 128, 64), (2, 1, 256, 16), (4, 2, 176, 32)])
def test_many_rows_with_holes_and_tails(heads, kv_heads, dim, page, causal):
    """128 rows and more, in one workgroup and over several; a page that is none; odd lengths."""
    check(Case(14, [333, 150, 64, 130, 40], [101, 150, 64, 3, 40], heads, kv_heads, dim, page, BF16, bad_page=(0, 1, -1),
               extra_rows=2), causal)
    check(Case(15, [700, 30], [70, 9], heads, kv_heads, dim, page, BF16, bad_page=(0, 2, 10 ** 6)), causal, scale=-0.2)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("new,length", [(1, 1), (2, 2), (17, 17), (40, 300), (70, 70), (130, 150), (257, 700)])
def test_chunks_of_prompts(dtype, new, length):
    check(Case(3, [length, max(1, length // 3)], [new, min(new, max(1, length // 3))], 4, 2, 128, 32, dtype))


def test_a_chunk_longer_than_the_cache_leaves_rows_empty():
    case = Case(4, [5, 0, 40], [9, 3, 40], 4, 2, 64, 16, BF16)
    check(case)
    check(Case(4, [5, 0, 40], [9, 3, 40], 4, 2, 64, 16, F32), causal=False)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_long_rows_are_split_and_joined(dtype):
    check(Case(5, [9000, 3, 4097, 2048], [2, 1, 5, 1], 4, 1, 128, 64, dtype))


@pytest.mark.parametrize("dim", [16, 24, 40, 56, 80, 88, 104, 120, 168, 248])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_dims_between_the_padded_ones(dtype, dim):
    """The last channels of the last token end inside a lane's piece of a row."""
    check(Case(13, [48, 17, 150], [2, 1, 40], 6, 2, dim, 16, dtype, spare_pages=0))


@pytest.mark.parametrize("order", ["token", "mixed"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_pool_layouts(order, dtype):
    check(Case(6, [100, 37, 260], [2, 5, 20], 8, 4, 80, 32, dtype, order=order))


@pytest.mark.parametrize("bad", [-1, -2 ** 31, 10 ** 6, 2 ** 31 - 1])
def test_tokens_of_no_page_are_no_tokens(bad):
    check(Case(7, [100, 40], [3, 3], 4, 2, 64, 16, BF16, bad_page=(0, 2, bad)))
    check(Case(7, [16, 40], [3, 3], 4, 2, 64, 16, F32, bad_page=(0, 0, bad)))


def test_a_scale_that_makes_scores_far_apart():
    check(Case(8, [300], [4], 4, 2, 64, 16, F32, scale_q=8.0), scale=1.0)
    check(Case(8, [300], [4], 4, 2, 64, 16, BF16, scale_q=8.0), scale=-0.5)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_each_token_gives_its_own_value(dtype, dim):
    """Rows that look at one token alone return its value exactly: a wrong place of K, V or a row shows."""
    import paper_2604_02945_amd as msao
    L = 96
    case = Case(9, [L], [L], 2, 2, dim, 16, dtype)
    eye = torch.zeros(L, dim)
    for j in range(L):  # tokens are told apart by two channels
        eye[j, j % dim] += 64.0
        eye[j, (j // dim * 7 + j + 11) % dim] -= 64.0
    p = torch.from_numpy(case.pages[0, np.arange(L) // 16].astype(np.int64))
    slot = torch.arange(L) % 16
    case.k[p, :, slot] = eye[:, None].to(dtype).expand(L, 2, dim)
    case.q = eye[:, None].to(dtype).expand(L, 2, dim).contiguous()
    cache, start = case.device(DEV)
    out = msao.msao_cache_attention(cache, start, L, case.q.to(DEV), scale=1.0, causal=False, accumulate=True)
    _, v, _ = case.tokens(0)
    assert np.array_equal(out.double().cpu().numpy(), v.transpose(1, 0, 2))
    assert np.array_equal(cache.weight[0, :, :L].cpu().numpy(), (case.weight[0, :, :L] + 1).numpy())


def test_rows_past_max_new_are_left():
    import paper_2604_02945_amd as msao
    case = Case(10, [50], [8], 4, 2, 64, 16, BF16)
    cache, start = case.device(DEV)
    out = torch.full((8, 4, 64), 7.0, dtype=BF16, device=DEV)
    msao.msao_cache_attention(cache, start, 3, case.q.to(DEV), out=out)
    full = msao.msao_cache_attention(cache, start, 8, case.q.to(DEV))
    torch.cuda.synchronize()
    assert torch.equal(out[:3], full[:3]) and (out[3:] == 7).all()


def test_queries_beside_keys_and_values_in_one_projection():
    import paper_2604_02945_amd as msao
    case = Case(11, [70, 90], [4, 9], 8, 2, 64, 16, BF16)
    cache, start = case.device(DEV)
    row = torch.randn(13, 12 * 64).to(BF16).to(DEV)
    q = row[:, :8 * 64].view(13, 8, 64)
    q.copy_(case.q)
    wide = torch.zeros(13, 10, 64, dtype=BF16, device=DEV)
    a = msao.msao_cache_attention(cache, start, 9, q, out=wide[:, :8])
    b = msao.msao_cache_attention(cache, start, 9, case.q.to(DEV))
    torch.cuda.synchronize()
    assert torch.equal(a, b) and (wide[:, 8:] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")], ids=str)
@pytest.mark.parametrize("dim,heads", [(128, 4), (64, 14), (256, 2), (96, 34), (128, 36), (256, 32)])
@pytest.mark.parametrize("at", ["k", "v", "both"])
def test_what_a_row_does_not_see_has_no_effect(dtype, value, dim, heads, at):
    """Token L - n + bad holds no finite value: rows before it are as without it, rows from it on
    are what the definition gives: NaN in what it reaches."""
    import paper_2604_02945_amd as msao
    L, n, bad = 70, 9, 4
    case = Case(12, [L, 33], [n, 2], heads, 2, dim, 16, dtype)
    j = L - n + bad
    page, slot = int(case.pages[0, j // 16]), j % 16
    clean, start = case.device(DEV)
    q = case.q.to(DEV)
    lse0, lse = (torch.zeros(n + 2, heads, device=DEV) for _ in range(2))
    want = msao.msao_cache_attention(clean, start, n, q, lse=lse0)
    if at in ("k", "both"):
        case.k[page, :, slot, dim // 2] = value
    if at in ("v", "both"):
        case.v[page, 1, slot, 3] = value
        case.v[page, 1, slot, dim - 1] = value
    cache, _ = case.device(DEV)
    got = msao.msao_cache_attention(cache, start, n, q, lse=lse, accumulate=True)
    torch.cuda.synchronize()
    others = [i for i in range(n + 2) if i < bad or i >= n]
    assert torch.equal(got[others], want[others]) and torch.equal(lse[others], lse0[others])
    if at == "v":
        G = heads // 2
        hit = got[bad:n, G:]
        assert not torch.isfinite(hit[..., [3, dim - 1]]).any()
        if value != value:
            assert torch.isnan(hit[..., [3, dim - 1]]).all()
        else:
            assert (hit[..., [3, dim - 1]] == value).all()
        rest = [d for d in range(dim) if d not in (3, dim - 1)]
        # the same products; the slow path only leaves out and adds those two channels
        assert torch.equal(got[bad:n][..., rest], want[bad:n][..., rest])
        assert torch.equal(got[bad:n, :G], want[bad:n, :G])
    elif value != value:
        assert torch.isnan(got[bad:n]).all() and torch.isnan(lse[bad:n]).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 3, 9, 40])
@pytest.mark.parametrize("dim,heads", [(128, 14), (256, 2)])
def test_a_key_at_minus_infinity_gives_nothing(dtype, n, dim, heads):
    """Every row that sees token 20 has the score -inf there: all is as with a score of -1e30."""
    import paper_2604_02945_amd as msao
    case = Case(16, [70, 50], [n, 1], heads, 2, dim, 16, dtype)
    case.q[..., 0] = case.q[..., 0].abs() + 1
    out = []
    for value in (-1e30, float("-inf")):
        case.k[int(case.pages[0, 1]), :, 4, 0] = value
        cache, start = case.device(DEV)
        lse = torch.zeros(n + 1, heads, device=DEV)
        o = msao.msao_cache_attention(cache, start, n, case.q.to(DEV), lse=lse, accumulate=True)
        out.append((o, lse, cache.weight))
    torch.cuda.synchronize()
    for a, b in zip(*out):
        assert torch.isfinite(a).all() and torch.equal(a, b)


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
@pytest.mark.parametrize("heads,kv_heads,dim,page", [(33, 1, 64, 16), (10, 2, 88, 32), (7, 1, 96, 16), (14, 2, 120, 64), (7, 1, 128, 16),
                                                     (8, 1, 256, 32), (14, 2, 176, 16)])
def test_rows_of_one_tile(heads, kv_heads, dim, page, causal):
    """33 to 64 rows: a single token of many heads, drafts; holes, tails, sequences of none; split and not."""
    n = 64 * kv_heads // heads
    new = [n, max(1, n - 1), 0, 1, n]
    check(Case(17, [333, 150, 0, 31, 64], new, heads, kv_heads, dim, page, BF16, bad_page=(0, 1, -1), extra_rows=2), causal)
    check(Case(18, [3000, n], [n, n], heads, kv_heads, dim, page, BF16, bad_page=(0, 2, 10 ** 6)), causal, scale=-0.2)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")], ids=str)
@pytest.mark.parametrize("dim,heads", [(128, 14), (96, 14), (64, 10), (256, 14)])
def test_values_not_seen_by_rows_of_one_tile(value, dim, heads):
    """Only the rows that see the token get its value."""
    import paper_2604_02945_amd as msao
    L, n, bad = 150, 9, 4
    case = Case(19, [L, 33], [n, 2], heads, 2, dim, 16, BF16)
    j = L - n + bad
    clean, start = case.device(DEV)
    want = msao.msao_cache_attention(clean, start, n, case.q.to(DEV))
    case.v[int(case.pages[0, j // 16]), 1, j % 16, 5] = value
    cache, _ = case.device(DEV)
    got = msao.msao_cache_attention(cache, start, n, case.q.to(DEV))
    torch.cuda.synchronize()
    hit = torch.zeros(n + 2, heads, dim, dtype=torch.bool)
    hit[bad:n, heads // 2:, 5] = True
    assert torch.equal(got.cpu()[~hit], want.cpu()[~hit])
    assert (torch.isnan(got.cpu()[hit]) if value != value else got.cpu()[hit] == value).all()
