"""Attention over a paged cache where queries, keys or values are not finite: what the
definition makes NaN is NaN in out, lse and weight, whichever kernel, tile or part it
falls to, and nothing else changes."""
import numpy as np
import pytest
import torch

from cache_ref import Case

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def attend(case, causal=True, scale=None):
    """out, lse, weight on the host."""
    import paper_2604_02945_amd as msao
    cache, start = case.device(DEV)
    lse = torch.full((case.rows, case.heads), 7.0, device=DEV)
    out = msao.msao_cache_attention(cache, start, case.max_new, case.q.to(DEV), lse=lse, causal=causal, scale=scale,
                                    accumulate=True)
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu(), cache.weight.cpu()


def same_but(got, want, hit):
    """NaN where `hit`, the same bits elsewhere."""
    assert torch.isnan(got[hit]).all()
    bits = torch.int16 if got.dtype == BF16 else torch.int32
    assert torch.equal(got[~hit].view(bits), want[~hit].view(bits))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 3, 8, 20, 40])
@pytest.mark.parametrize("heads,dim", [(4, 64), (2, 96), (4, 128), (2, 256)])
@pytest.mark.parametrize("long", [70, 1300], ids=["whole", "split"])
def test_a_nan_query(dtype, n, heads, dim, long):
    """Its row is NaN, and so is the weight of every token that it sees; a row that sees none stays empty."""
    case = Case(71, [long, 0, 33], [n, 1, 2], heads, 2, dim, 16, dtype)
    out0, lse0, w0 = attend(case)
    row, head, none = n - 1, heads - 1, n  # the last row of the first sequence, and the row of the empty one
    case.q[row, head, 5] = float("nan")
    case.q[none, :, 1] = float("nan")
    out, lse, w = attend(case)
    hit = torch.zeros(out.shape, dtype=torch.bool)
    hit[row, head] = True
    same_but(out, out0, hit)
    same_but(lse, lse0, hit[..., 0])
    assert (out[none] == 0).all() and (lse[none] == -np.inf).all()
    seen = torch.zeros(w.shape, dtype=torch.bool)
    seen[0, 1, :long] = True
    same_but(w, w0, seen)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 8, 20, 40])
@pytest.mark.parametrize("heads,dim", [(4, 64), (2, 96), (4, 128), (2, 256)])
@pytest.mark.parametrize("length", [1, 17, 33, 65, 97, 1025, 1281])
def test_a_nan_key_alone_in_its_tile(dtype, n, heads, dim, length):
    """The last token, the first of a tile (or of a part) and seen by the last row alone."""
    n = min(n, length)
    case = Case(72, [length, 40], [n, 2], heads, 2, dim, 16, dtype)
    out0, lse0, w0 = attend(case)
    j = length - 1
    case.k[int(case.pages[0, j // 16]), 1, j % 16, 3] = float("nan")
    out, lse, w = attend(case)
    hit = torch.zeros(out.shape, dtype=torch.bool)
    hit[n - 1, heads // 2:] = True
    same_but(out, out0, hit)
    same_but(lse, lse0, hit[..., 0])
    seen = torch.zeros(w.shape, dtype=torch.bool)
    seen[0, 1, :length] = True
    same_but(w, w0, seen)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 8, 20, 40])
@pytest.mark.parametrize("heads,dim", [(4, 64), (2, 96), (4, 128), (2, 256)])
@pytest.mark.parametrize("length", [70, 1300], ids=["whole", "split"])
@pytest.mark.parametrize("value", [float("inf"), float("nan")], ids=str)
def test_only_scores_of_minus_infinity(dtype, n, heads, dim, length, value):
    """Rows without a score above -inf are empty, whatever the values hold: out 0, lse -inf, no weight."""
    case = Case(73, [length, 40], [n, 2], heads, 2, dim, 16, dtype)
    out0, lse0, w0 = attend(case)
    case.q[:n, :, 0] = case.q[:n, :, 0].abs() + 1
    for j in range(length):
        case.k[int(case.pages[0, j // 16]), 1, j % 16, 0] = float("-inf")
    for j in (0, length // 2, length - n, length - 1):  # tiles that every row sees, and those of the chunk
        case.v[int(case.pages[0, j // 16]), 1, j % 16, 2] = value
    out, lse, w = attend(case)
    G = heads // 2
    assert (out[:n, G:] == 0).all() and (lse[:n, G:] == -np.inf).all()
    assert torch.equal(w[0, 1], case.weight[0, 1])
    assert torch.equal(out[n:], out0[n:]) and torch.equal(lse[n:], lse0[n:]) and torch.equal(w[1], w0[1])
    assert torch.isfinite(out[:n, :G]).all() and torch.isfinite(lse[:n, :G]).all() and torch.isfinite(w[0, 0]).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n", [3, 20, 40])
@pytest.mark.parametrize("heads,dim", [(4, 64), (2, 96), (4, 128), (2, 256)])
@pytest.mark.parametrize("score", ["-inf", "far below"])
@pytest.mark.parametrize("value", [float("inf"), float("nan")], ids=str)
def test_values_of_no_weight_that_are_not_finite(dtype, n, heads, dim, score, value):
    """A token whose p is 0: its value still reaches the rows that see it, in a tile that all see and in the chunk's."""
    L = 170
    for j, first in ((5, 0), (L - 2, n - 2)):  # the token, and the first row that sees it
        case = Case(74, [L, 40], [n, 2], heads, 2, dim, 16, dtype)
        case.q[:n, :, 0] = case.q[:n, :, 0].abs() + 1
        p, slot = int(case.pages[0, j // 16]), j % 16
        case.k[p, 1, slot, 0] = float("-inf") if score == "-inf" else -1e6
        out0, lse0, w0 = attend(case)
        case.v[p, 1, slot, 7] = value
        out, lse, w = attend(case)
        hit = torch.zeros(out.shape, dtype=torch.bool)
        hit[first:n, heads // 2:, 7] = True
        assert not torch.isfinite(out[hit]).any()
        assert torch.isfinite(out0).all() and torch.equal(out[~hit], out0[~hit])
        assert torch.equal(lse, lse0) and torch.equal(w, w0)
