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
