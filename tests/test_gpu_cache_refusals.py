"""Calls of the paged cache's operators that are refused once a device is at hand. Nothing is enqueued."""
import pytest
import torch

from cache_ref import Case

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("accumulate", [False, True], ids=["out", "weight"])
def test_out_in_the_queries_memory(dtype, accumulate):
    import paper_2604_02945_amd as msao
    case = Case(95, [40, 70], [2, 7], 8, 2, 64, 16, dtype)
    cache, start = case.device(DEV)
    both = torch.zeros(9, 2, 8, 64, dtype=dtype, device=DEV)
    both[:, 0] = case.q.to(DEV)
    q = both[:, 0]
    flat = torch.zeros(20, 8, 64, dtype=dtype, device=DEV)
    flat[:9] = case.q.to(DEV)
    before = cache.weight.clone()
    for x, out in ((q, q), (flat[:9], flat[:9]), (flat[:9], flat[8:17]), (flat[8:17], flat[:9]),
                   (flat[:9], torch.as_strided(flat, (9, 8, 64), (1024, 64, 1)))):
        kept = out.clone()
        with pytest.raises(msao.MsaoError, match="out overlaps q"):
            msao.msao_cache_attention(cache, start, 7, x, out=out, accumulate=accumulate)
        assert torch.equal(out, kept) and torch.equal(cache.weight, before)
    # between one another's rows, and behind them
    want = msao.msao_cache_attention(cache, start, 7, case.q.to(DEV))
    assert torch.equal(msao.msao_cache_attention(cache, start, 7, q, out=both[:, 1]), want)
    assert torch.equal(msao.msao_cache_attention(cache, start, 7, flat[:9], out=flat[9:18]), want)


def test_numbers_past_an_integer():
    """Counts that only bound others: more than there are counts as all; below 0 they are refused."""
    import paper_2604_02945_amd as msao
    case = Case(96, [40, 70], [2, 7], 8, 2, 64, 16, BF16)
    cache, start = case.device(DEV)
    q = case.q.to(DEV)
    want = msao.msao_cache_attention(cache, start, 7, q)
    for many in (2 ** 31, 2 ** 32, 2 ** 32 + 1, 2 ** 64):
        assert torch.equal(msao.msao_cache_attention(cache, start, many, q), want)
    budget = torch.tensor([20, 30], dtype=torch.int32, device=DEV)
    for many in (70, 2 ** 31, 2 ** 32, 2 ** 64 + 3):
        for first, recent, ids in ((0, many, [range(20, 40), range(40, 70)]), (many, 0, [range(20), range(30)])):
            c, _ = case.device(DEV)
            r = msao.msao_cache_evict(c, budget, first, recent)
            for b in range(2):
                for h in range(2):
                    assert r["kept_idx"][b, h, :len(ids[b])].tolist() == list(ids[b])
    for first, recent, error in ((-1, 0, msao.MsaoError), (0, -1, msao.MsaoError), (-2 ** 32, 0, ValueError), (0, -2 ** 33, ValueError)):
        with pytest.raises(error, match="negative|out of range"):
            msao.msao_cache_evict(cache, budget, first, recent)
    with pytest.raises(ValueError, match="out of range"):
        msao.msao_cache_attention(cache, start, -2 ** 32, q)


def test_a_workspace_of_one_byte_expanded():
    import paper_2604_02945_amd as msao
    case = Case(97, [2000, 70], [2, 7], 8, 2, 64, 16, BF16)
    cache, start = case.device(DEV)
    q = case.q.to(DEV)
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    for bad in (ws[:1].expand(1 << 28), torch.as_strided(ws, (1 << 20, 16), (0, 1))):
        with pytest.raises(ValueError, match="workspace must be contiguous"):
            msao.msao_cache_attention(cache, start, 7, q, workspace=bad)
        with pytest.raises(ValueError, match="workspace must be contiguous"):
            msao.msao_cache_evict(cache, torch.tensor([20, 30], dtype=torch.int32, device=DEV), workspace=bad)
    with pytest.raises(msao.MsaoError, match="workspace too small"):
        msao.msao_cache_attention(cache, start, 7, q, workspace=ws)
