"""A chunk whose starts are not ascending: append takes the rows that the definition gives
each sequence, and attention's, wherever they lie in the step's arrays."""
import numpy as np
import pytest
import torch

from cache_ref import Case

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16


def runs(rows, blocks, per, seed):
    """Starts of blocks * per - 1 sequences: blocks of rows in descending order, ascending starts inside each."""
    rng = np.random.RandomState(seed)
    cuts = sorted(rng.choice(np.arange(1, rows), blocks - 1, replace=False).tolist())
    start = []
    for a, b in list(zip([0] + cuts, cuts + [rows]))[::-1]:
        start += [a] + sorted(rng.randint(a, b + 1, per - 1).tolist())
    return start


@pytest.mark.parametrize("start,rows", [([5, 2, 9], 9), ([0, 100, 4], 9), ([7, 8, 1000], 9), ([-4, 3, 3], 9), ([3, 3, -1], 9),
                                        ([9, 4, 2, 6, 1], 9), ([6, 9, 3, 6, 0, 2, 2], 9), (runs(200, 12, 12, 0), 200),
                                        (runs(90, 3, 25, 1), 90), (runs(500, 40, 5, 2), 500)],
                         ids=["drop", "past", "far", "below", "none", "drops", "blocks", "143", "74", "199"])
def test_append_takes_the_rows_of_each_sequence(start, rows):
    import paper_2604_02945_amd as msao
    B, page, K, H, D = len(start) - 1, 16, 2, 4, 64
    b = np.clip(start, 0, rows)
    new = [max(0, int(e - s)) for s, e in zip(b[:-1], b[1:])]
    owner = np.full(rows, -1)
    for s in range(B):
        assert (owner[b[s]:b[s] + new[s]] == -1).all()
        owner[b[s]:b[s] + new[s]] = s
    lengths = [n + s % 5 for s, n in enumerate(new)]
    case = Case(61, lengths, [0] * B, H, K, D, page, BF16)
    cache, _ = case.device(DEV)
    before_k, before_v, before_w = cache.k.cpu(), cache.v.cpu(), cache.weight.cpu()
    g = torch.Generator().manual_seed(62)
    q, k, v = (torch.randn(rows, n, D, generator=g).to(BF16) for n in (H, K, K))
    st = torch.tensor(start, dtype=torch.int32, device=DEV)
    q_out = torch.full((rows, H, D), 7.0, dtype=BF16, device=DEV)
    msao.msao_cache_append(cache, st, rows, k.to(DEV), v.to(DEV), q=q.to(DEV), q_out=q_out)
    torch.cuda.synchronize()
    mine = torch.from_numpy(owner >= 0)
    got = q_out.cpu()
    assert torch.equal(got[mine], q[mine]) and (got[~mine] == 7).all()
    for s in range(B):
        for i in range(new[s]):
            j = lengths[s] - new[s] + i
            p = int(case.pages[s, j // page])
            before_k[p, :, j % page], before_v[p, :, j % page] = k[b[s] + i], v[b[s] + i]
            before_w[s, :, j] = 0
    bits = lambda x: x.cpu().contiguous().view(torch.int16)  # noqa: E731
    assert torch.equal(bits(cache.k), bits(before_k)) and torch.equal(bits(cache.v), bits(before_v))
    assert torch.equal(cache.weight.cpu(), before_w)
    # attention over the same rows reads what append stored
    out = torch.full((rows, H, D), 7.0, dtype=BF16, device=DEV)
    msao.msao_cache_attention(cache, st, rows, q.to(DEV), out=out)
    assert ((out.cpu() != 7).any(-1).any(-1) == mine).all()
