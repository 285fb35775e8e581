"""Attention of large batches over a paged cache against its definition in 64 bits (on
the GPU: products of many sequences)."""
import numpy as np
import pytest
import torch

from cache_ref import Case, tolerances

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def attention64(case, scale, causal):
    """Case.attention, a kv head's rows at a time."""
    out, mag = (torch.zeros(case.rows, case.heads, case.dim, dtype=torch.float64, device=DEV) for _ in range(2))
    lse = torch.zeros(case.rows, case.heads, dtype=torch.float64, device=DEV)
    weight = case.weight.double().to(DEV)
    span = torch.zeros((), dtype=torch.float64, device=DEV)
    G, K = case.heads // case.kv_heads, case.kv_heads
    for b in range(case.B):
        n, m, at = case.lengths[b], case.new[b], int(case.start[b])
        if n == 0 or m == 0:
            continue
        k, v, _ = case.tokens(b)
        k, v = torch.from_numpy(k).to(DEV), torch.from_numpy(v).to(DEV)
        q = case.q[at:at + m].double().to(DEV).view(m, K, G, case.dim).permute(1, 0, 2, 3).reshape(K, m * G, case.dim)
        kt = k.transpose(1, 2).contiguous()
        s = scale * torch.bmm(q.contiguous(), kt)
        span = torch.maximum(span, scale * torch.bmm(q.abs(), kt.abs()).max())
        if causal:
            tok = torch.arange(m, device=DEV).repeat_interleave(G)[:, None]
            s.masked_fill_(torch.arange(n, device=DEV)[None] > n - m + tok, -np.inf)
        z = torch.logsumexp(s, -1, keepdim=True)
        p = torch.exp(s - z)
        weight[b, :, :n] += p.sum(1)
        back = lambda x: x.view(K, m, G, -1).permute(1, 0, 2, 3).reshape(m, case.heads, -1)  # noqa: E731
        out[at:at + m], mag[at:at + m] = back(torch.bmm(p, v)), back(torch.bmm(p, v.abs()))
        lse[at:at + m] = back(z)[..., 0]
    return out.cpu().numpy(), lse.cpu().numpy(), weight.cpu().numpy(), mag.cpu().numpy(), float(span)


def check(case, accumulate=True, per=None, causal=True):
    """`per`: columns of a page table wider than the sequences need. Returns the workspace's bytes."""
    import paper_2604_02945_amd as msao
    if per is not None:
        wide = np.full((case.B, per), -3, np.int32)
        wide[:, :case.per] = case.pages
        case.pages = wide
        if accumulate:
            old = case.weight
            case.weight = torch.zeros(case.B, case.kv_heads, per * case.page)
            case.weight[..., :old.shape[2]] = old
    cache, start = case.device(DEV, with_weight=accumulate)
    scale = case.dim ** -0.5
    out = torch.full((case.rows, case.heads, case.dim), 7.0, dtype=case.dtype, device=DEV)
    lse = torch.full((case.rows, case.heads), 7.0, device=DEV)
    msao.msao_cache_attention(cache, start, case.max_new, case.q.to(DEV), causal=causal, out=out, lse=lse, accumulate=accumulate)
    torch.cuda.synchronize()
    want, z, weight, mag, span = attention64(case, scale, causal)
    tol_z, tol = tolerances(case, mag, span, want)
    assert np.abs(lse.double().cpu().numpy() - z).max() <= tol_z
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
    if accumulate:
        rows = case.max_new * case.heads // case.kv_heads
        tol_w = (2 * tol_z + (rows + 4) * 2.0 ** -24) * (weight + 1)
        assert (np.abs(cache.weight.double().cpu().numpy() - weight) <= tol_w).all()
    return msao.cache_attention_workspace(cache, start, case.rows, case.max_new, case.heads, causal, accumulate)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("accumulate", [False, True], ids=["out", "weight"])
def test_one_prompts_chunk_beside_generating_requests(dtype, accumulate):
    """256 requests of 32 heads, one with 2,048 new tokens."""
    rng = np.random.RandomState(0)
    lengths = rng.randint(1, 120, 256).tolist()
    lengths[77] = 2100
    new = [1] * 256
    new[77] = 2048
    check(Case(91, lengths, new, 32, 8, 64, 64, dtype), accumulate)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,new", [(8, 3), (32, 3), (32, 16)], ids=["few", "rows", "tile"])
def test_wide_tables(dtype, heads, new):
    """Short requests and a few longer ones in a table of 131,072 tokens: parts longer than most of them."""
    rng = np.random.RandomState(1)
    lengths = rng.randint(new, 200, 64).tolist()
    lengths[5], lengths[40], lengths[63] = 9000, 4096, 4097
    case = Case(92, lengths, [new if i % 3 else 1 for i in range(64)], heads, 8, 64, 64, dtype)
    tight = check(case, accumulate=False)
    wide = check(case, accumulate=False, per=2048)
    # parts of 64 * 8 * 131,072 / 16,384 = 4,096 tokens: 32, each with 64 channels and two sums a row
    assert 0 < tight and wide <= 32 * case.rows * heads * 66 * 4 + 512


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
@pytest.mark.parametrize("dtype,dim", [(BF16, 64), (BF16, 128), (BF16, 256), (F32, 64), (F32, 96)])
def test_many_prompts_with_weight_that_no_parts_are_made_for(dtype, dim, causal):
    """128 prompts of 8 kv heads and up to 80 rows: rows and tokens whole, the weight added without a join."""
    rng = np.random.RandomState(2)
    new = rng.randint(1, 41, 128).tolist()
    new[17] = 40
    lengths = [n + int(rng.randint(0, 300)) for n in new]
    lengths[3], lengths[17], lengths[90] = 0, 700, new[90]
    new[3] = 0
    case = Case(93, lengths, new, 16, 8, dim, 16, dtype)
    # no parts of rows or tokens: the workspace is the sums of the rows
    assert check(case, causal=causal) == (case.rows * 16 * 4 + 255) // 256 * 256


def test_one_sequence_of_a_strided_table():
    """Lengths, pages, starts and positions of one entry, at the strides that a slice leaves them."""
    import paper_2604_02945_amd as msao
    case = Case(94, [90], [1], 4, 2, 64, 16, BF16)
    cache, start = case.device(DEV)
    q, kv = case.q.to(DEV), torch.randn(1, 2, 64, device=DEV).to(BF16)
    inv = torch.rand(32, device=DEV)
    table = torch.zeros(1, 9, dtype=torch.int32, device=DEV)
    table[0, 3:3 + case.per] = torch.from_numpy(case.pages[0]).to(DEV)
    table[0, 1] = 90
    odd = msao.KvCache(cache.k.clone(), cache.v.clone(), table[:, 3:3 + case.per], table[:, 1], cache.weight.clone())
    at = torch.tensor([[5, 6, 7], [1, 2, 3]], dtype=torch.int32, device=DEV)
    got = []
    for c, pos in ((cache, at[:, :1].contiguous()), (odd, at.t().contiguous().t()[:, :1])):
        x = msao.msao_cache_append(c, start, 1, kv, kv, q=q, inv_freq=inv, positions=pos, sections=(20, 12))
        got.append((msao.msao_cache_attention(c, start, 1, x, accumulate=True), c.weight, x))
    for a, b in zip(*got):
        assert torch.equal(a, b)
