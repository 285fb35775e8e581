"""Forms of the paged cache that its header allows and the other tests do not take: no pages,
the largest pages, weight rows longer than the capacity, many heads on one, thousands of sequences."""
import numpy as np
import pytest
import torch

from cache_ref import Case, evicted
from test_gpu_cache_batches import check

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 20, 70])
def test_a_pool_of_no_pages(dtype, n):
    """Every token lies in no page: rows see nothing, and eviction keeps indices and weight alone."""
    import paper_2604_02945_amd as msao
    k = torch.zeros(0, 2, 16, 64, dtype=dtype, device=DEV)
    w = torch.rand(2, 2, 96, device=DEV)
    cache = msao.KvCache(k, k.clone(), torch.zeros(2, 6, dtype=torch.int32, device=DEV), i32(90, 40), w.clone())
    start, T = i32(0, n, n + 1), n + 1
    q, kv = torch.randn(T, 4, 64, device=DEV).to(dtype), torch.randn(T, 2, 64, device=DEV).to(dtype)
    lse = torch.zeros(T, 4, device=DEV)
    q2 = msao.msao_cache_append(cache, start, n, kv, kv, q=q)
    want = w.clone()
    want[0, :, 90 - n:90] = 0
    want[1, :, 39] = 0
    assert torch.equal(q2, q) and torch.equal(cache.weight, want)
    out = msao.msao_cache_attention(cache, start, n, q, lse=lse, accumulate=True)
    assert (out == 0).all() and (lse == -np.inf).all() and torch.equal(cache.weight, want)
    r = msao.msao_cache_evict(cache, i32(30, 30), 1, 2)
    want = want.cpu().numpy()
    for b, length in enumerate((90, 40)):
        for h in range(2):
            kept = evicted(want[b, h], length, 30, 96, 1, 2)
            assert r["kept_idx"][b, h, :30].tolist() == kept.tolist()
            assert np.array_equal(cache.weight[b, h, :30].cpu().numpy(), want[b, h][kept])
    assert cache.length.tolist() == [30, 30]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("new", [3, 100])
def test_pages_of_65536_tokens(dtype, new):
    check(Case(101, [66000, 65536, 200], [new, 1, new], 4, 1, 64, 65536, dtype, spare_pages=0))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,new", [(71, 1), (71, 3), (130, 2), (200, 9)])
def test_many_query_heads_on_one(dtype, heads, new):
    check(Case(102, [150, new, 33], [new, new, 1], heads, 1, 64, 16, dtype))


@pytest.mark.parametrize("n", [2, 60], ids=["few rows", "many rows"])
def test_weight_rows_longer_than_the_capacity(n):
    import paper_2604_02945_amd as msao
    case = Case(103, [300, 80], [n, 1], 4, 2, 64, 16, BF16)
    cache, start = case.device(DEV)
    wide = torch.full((2, 2, case.cap + 37), 9.0, device=DEV)
    wide[..., :case.cap] = cache.weight
    long = msao.KvCache(cache.k.clone(), cache.v.clone(), cache.pages, cache.length.clone(), wide)
    q = case.q.to(DEV)
    for c in (cache, long):
        msao.msao_cache_attention(c, start, n, q, accumulate=True)
    assert torch.equal(long.weight[..., :case.cap], cache.weight) and (long.weight[..., case.cap:] == 9).all()
    idx = torch.full((2, 2, case.cap + 5), 11, dtype=torch.int32, device=DEV)
    a = msao.msao_cache_evict(cache, i32(100, 50), 1, 2)["kept_idx"]
    msao.msao_cache_evict(long, i32(100, 50), 1, 2, kept_idx=idx)
    assert torch.equal(idx[..., :case.cap], a) and (idx[..., case.cap:] == 11).all()
    assert torch.equal(long.weight[..., :case.cap], cache.weight) and (long.weight[..., case.cap:] == 9).all()
    bits = lambda x: x.view(torch.int16)  # noqa: E731
    assert torch.equal(bits(long.k), bits(cache.k)) and torch.equal(bits(long.v), bits(cache.v))


def test_thousands_of_sequences():
    """3,001 short requests, most with one token, some with none: append finds each row's, attention each request's."""
    import paper_2604_02945_amd as msao
    rng = np.random.RandomState(3)
    B = 3001
    new = rng.randint(0, 4, B).tolist()
    lengths = [n + int(rng.randint(0, 30)) for n in new]
    case = Case(104, lengths, new, 4, 2, 64, 16, BF16)
    cache, start = case.device(DEV)
    kv = torch.randn(case.rows, 2, 64, generator=case.g).to(BF16)
    k, v = kv, kv.flip(0)
    msao.msao_cache_append(cache, start, 3, k.to(DEV), v.to(DEV))
    for b in range(B):
        for i in range(new[b]):
            j, row = lengths[b] - new[b] + i, int(case.start[b]) + i
            p = int(case.pages[b, j // 16])
            case.k[p, :, j % 16], case.v[p, :, j % 16] = k[row], v[row]
            case.weight[b, :, j] = 0
    bits = lambda x: x.cpu().contiguous().view(torch.int16)  # noqa: E731
    assert torch.equal(bits(cache.k), bits(case.k)) and torch.equal(bits(cache.v), bits(case.v))
    assert torch.equal(cache.weight.cpu(), case.weight)
    check(case)
