"""Attention of sequences that share prefixes on the GPU against its definition in 64 bits. Tolerances are
those of attention (see cache_ref.tolerances): the join of a prefix' and a sequence's own parts adds three
roundings a part, within the L + 8 counted for the sums over L tokens."""
import numpy as np
import pytest
import torch

from cache_ref import Case, tolerances

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def share(case, group, tokens):
    """Sequences group[g] .. group[g+1]-1 of the case have the first one's tokens 0 .. tokens[g]-1: whole pages by
    their tables, the rest as a copy."""
    for g, t in enumerate(tokens):
        lead = group[g]
        for s in range(lead + 1, min(group[g + 1], case.B)):
            n = min(t, case.lengths[s], case.lengths[lead])
            whole = n // case.page
            case.pages[s, :whole] = case.pages[lead, :whole]
            rest = n - whole * case.page
            if rest > 0:
                a, b = case.pages[lead, whole], case.pages[s, whole]
                case.k[b, :, :rest], case.v[b, :, :rest] = case.k[a, :, :rest], case.v[a, :, :rest]
    return case


def run(case, group, tokens, causal=True, scale=None, accumulate=False, max_seqs=None, max_tokens=None, max_own=None, max_new=None,
        q=None, **kw):
    import paper_2604_02945_amd as msao
    cache, start = case.device(DEV)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    prefix = msao.SharedPrefix(ints(group), ints(tokens),
                               max(np.diff(group).max(initial=0), 0) if max_seqs is None else max_seqs,
                               max(max(tokens, default=0), 0) if max_tokens is None else max_tokens, max_own)
    out = torch.full((case.rows, case.heads, case.dim), 7.0, dtype=case.dtype, device=DEV)
    lse = torch.full((case.rows, case.heads), 7.0, device=DEV)
    msao.msao_cache_attention_shared(cache, prefix, start, case.max_new if max_new is None else max_new,
                                     (case.q if q is None else q).to(DEV),
                                     scale=case.dim ** -0.5 if scale is None else scale, causal=causal, out=out, lse=lse,
                                     accumulate=accumulate, **kw)
    torch.cuda.synchronize()
    return cache, out, lse


def check(case, group, tokens, causal=True, scale=None, accumulate=True, **kw):
    cache, out, lse = run(case, group, tokens, causal, scale, accumulate, **kw)
    scale = case.dim ** -0.5 if scale is None else scale
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
        rows = case.max_new * case.heads // case.kv_heads
        tol_w = (2 * tol_z + (rows + 4) * 2.0 ** -24) * (weight + 1)
        assert (np.abs(got_w - weight) <= tol_w).all()
    else:
        assert torch.equal(cache.weight.cpu(), case.weight)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 160, 255, 256, 300])
def test_prefixes_that_end_anywhere(dtype, tokens):
    """In a page, a tile, a stage; the sequences' own tokens as well."""
    lengths = [tokens + n for n in (1, 2, 3, 17, 64, 100, 7, 40)]
    check(share(Case(1, lengths, [1, 2, 3, 2, 1, 6, 7, 1], 8, 2, 64, 16, dtype), [0, 8], [tokens]), [0, 8], [tokens])


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
@pytest.mark.parametrize("heads,kv_heads,dim,page", [(4, 4, 128, 16), (7, 1, 128, 32), (28, 4, 128, 64), (5, 5, 8, 16), (12, 3, 96, 16),
                                                     (6, 2, 136, 64), (4, 2, 200, 16), (8, 1, 256, 128), (16, 1, 64, 16)])
def test_groups_heads_and_dims(dtype, causal, heads, kv_heads, dim, page):
    """Groups of several sizes, sequences in none, sequences without rows and without tokens."""
    lengths = [200, 130, 210, 133, 90, 0, 150, 161, 155, 30, 300]
    new = [3, 1, 6, 2, 4, 0, 0, 1, 5, 2, 6]
    group, tokens = [0, 4, 4, 6, 9], [128, 50, 80, 144]
    check(share(Case(2, lengths, new, heads, kv_heads, dim, page, dtype, extra_rows=3), group, tokens), group, tokens, causal)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_sequences_that_cannot_share(dtype):
    """Shorter than the prefix, or new tokens inside it: they see what they would see alone."""
    lengths, new = [100, 99, 97, 96, 95, 50, 0, 200, 96], [4, 4, 1, 1, 1, 2, 0, 110, 0]
    group, tokens = [0, 9], [96]
    for causal in (True, False):
        check(share(Case(3, lengths, new, 6, 2, 64, 32, dtype), group, tokens), group, tokens, causal)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("lead", [0, 1, 95, 96, 97])
def test_a_first_sequence_that_holds_less_than_the_prefix(dtype, lead):
    """Nothing is read from it then: a server's first request ended, the others go on."""
    lengths, new = [lead, 200, 150, 99, 0, 120, 130], [min(lead, 1), 4, 1, 2, 0, 1, 3]
    for causal in (True, False):
        check(share(Case(6, lengths, new, 6, 2, 64, 32, dtype), [0, 5, 7], [96, 96]), [0, 5, 7], [96, 96], causal)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_bounds_that_are_too_small(dtype):
    """More sequences, tokens, own tokens than the host said: the same results."""
    lengths, new = [400, 390, 500, 333, 700, 340], [2, 1, 6, 3, 5, 1]
    group, tokens = [0, 4, 6], [320, 336]
    case = share(Case(4, lengths, new, 4, 2, 64, 16, dtype), group, tokens)
    for kw in (dict(max_seqs=1), dict(max_seqs=0), dict(max_seqs=2), dict(max_tokens=0), dict(max_tokens=330), dict(max_own=1), dict(max_own=10 ** 6),
               dict(max_seqs=10 ** 6, max_tokens=10 ** 6)):
        check(case, group, tokens, **kw)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_long_prefixes_and_many_sequences(dtype):
    lengths = [5000 + (37 * i) % 300 for i in range(24)]
    new = [1 + i % 4 for i in range(24)]
    check(share(Case(5, lengths, new, 4, 1, 128, 64, dtype), [0, 24], [4992]), [0, 24], [4992], accumulate=False)
    check(share(Case(6, [300] * 70, [1] * 70, 4, 2, 64, 16, dtype), [0, 1, 3, 70], [272, 16, 288]), [0, 1, 3, 70], [272, 16, 288])


def test_many_groups():
    """More than one load of them a wavefront."""
    group = [2 * i for i in range(101)]
    tokens = [16 * (i % 5) for i in range(100)]
    check(share(Case(7, [70 + i % 30 for i in range(203)], [1 + i % 2 for i in range(203)], 4, 2, 64, 16, BF16), group, tokens), group, tokens)


def test_the_first_sequences_pages_are_read():
    case = share(Case(8, [150, 160, 170], [1, 2, 3], 4, 2, 64, 16, BF16), [0, 3], [128])
    want = run(case, [0, 3], [128])
    case.pages[1:, :8] = -1
    got = run(case, [0, 3], [128])
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])


def test_holes_in_a_prefix():
    """A page that is none in the middle of the shared tokens."""
    case = Case(9, [150, 160, 170, 40], [1, 2, 3, 1], 4, 2, 64, 16, BF16)
    case.pages[0, 3] = -1
    check(share(case, [0, 3], [128]), [0, 3], [128])


@pytest.mark.parametrize("order", ["token", "mixed"])
def test_layouts_of_the_pool_and_strided_rows(order):
    case = share(Case(10, [333, 340, 350], [3, 2, 6], 6, 2, 96, 32, BF16, order=order), [0, 3], [320])
    check(case, [0, 3], [320], causal=True)
    wide = torch.zeros(case.rows, 2, case.heads, case.dim, dtype=BF16)
    wide[:, 1] = case.q
    a, b = run(case, [0, 3], [320], q=wide.to(DEV)[:, 1]), run(case, [0, 3], [320])
    assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])


def test_groups_out_of_order_and_out_of_range_do_not_fault():
    case = share(Case(11, [100, 110, 120, 130], [1, 2, 1, 2], 4, 2, 64, 16, BF16), [0, 2], [80])
    for group, tokens in (([-5, 2, 900], [80, 16]), ([0, 2, 2], [80, -7]), ([0, 2, 4], [80, 10 ** 9])):
        share(case, [0, 2], [80])
        check(case, group, [tokens[0], 0 if tokens[1] in (16,) else tokens[1]], max_seqs=4, max_tokens=100)


def test_rows_past_max_new_and_streams():
    case = share(Case(12, [100, 110, 120], [1, 5, 3], 4, 2, 64, 16, BF16), [0, 3], [64])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    _, out, lse = run(case, [0, 3], [64], max_new=2, stream=side)
    want, z, _, mag, span = case.attention(case.dim ** -0.5, True)
    _, tol = tolerances(case, mag, span, want)
    left = [3, 4, 5, 8]  # rows 2.. of the second sequence and row 2 of the third
    done = [r for r in range(9) if r not in left]
    assert (out[left] == 7).all() and (lse[left] == 7).all()
    assert (np.abs(out.double().cpu().numpy() - want)[done] <= tol[done]).all()


def test_the_same_bits_and_replays():
    import paper_2604_02945_amd as msao
    case = share(Case(13, [2000 + 5 * i for i in range(20)], [1 + i % 3 for i in range(20)], 8, 2, 128, 32, BF16), [0, 12, 20], [1984, 1600])
    cache, start = case.device(DEV)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    prefix = msao.SharedPrefix(ints([0, 12, 20]), ints([1984, 1600]), 12, 1984)
    q = case.q.to(DEV)
    out, lse = torch.zeros_like(q), torch.zeros(case.rows, 8, device=DEV)
    ws = torch.empty(msao.cache_attention_shared_workspace(cache, prefix, start, case.rows, 3, 8) + 256, dtype=torch.uint8, device=DEV)
    ws = ws[-ws.data_ptr() % 256:][:ws.numel() - 256]

    def call(out, lse, ws=None):
        msao.msao_cache_attention_shared(cache, prefix, start, 3, q, out=out, lse=lse, workspace=ws)
    call(out, lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, lse, ws)
    for i in range(4):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(i)).to(BF16))
        prefix.tokens.copy_(ints([[1984, 1600], [16, 0], [1000, 1600], [1984, 32]][i]))
        ws.fill_(255)  # NaN
        graph.replay()
        torch.cuda.synchronize()
        a, b = torch.zeros_like(out), torch.zeros_like(lse)
        call(a, b)
        c, d = torch.zeros_like(out), torch.zeros_like(lse)
        call(c, d)
        torch.cuda.synchronize()
        assert torch.equal(out, a) and torch.equal(lse, b) and torch.equal(a, c) and torch.equal(b, d)
