"""Attention where scores are far from 0, as tokens are that a key's channel masks: rows of nothing else too. Every
key has one channel alone, so that a row's scores are equal: p is 1 / n of n tokens seen, exactly, and out is their
values' mean. In 32 bits lse is the score plus ln n, rounded: off by 2^-22 of it (as in cache_ref.tolerances)."""
import numpy as np
import pytest
import torch

from cache_ref import Case
from test_gpu_cache_shared import DEV, run, share

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
LENGTHS, NEW, GROUP, TOKENS = [1100, 1060, 1043, 70], [9, 3, 1, 2], [0, 3], [1040]


def far_case(dtype, heads, kv_heads, dim, value, new=NEW):
    case = share(Case(51, LENGTHS, new, heads, kv_heads, dim, 16, dtype), GROUP, TOKENS)
    case.q[..., 0] = case.q[..., 0].abs() + 1
    case.k[~torch.isnan(case.k)] = 0
    case.k[..., 0] = torch.where(torch.isnan(case.k[..., 0]), case.k[..., 0], torch.tensor(value).to(dtype))
    return case


def alone(case, accumulate=False):
    import paper_2604_02945_amd as msao
    cache, start = case.device(DEV)
    lse = torch.zeros(case.rows, case.heads, device=DEV)
    out = msao.msao_cache_attention(cache, start, case.max_new, case.q.to(DEV), lse=lse, accumulate=accumulate)
    return cache, out, lse


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shared", [False, True], ids=["alone", "shared"])
@pytest.mark.parametrize("value", [-1e30, 1e30, -3e34, 1e10, -3e9, 2e8, -1e7, 100.0])
@pytest.mark.parametrize("heads,kv_heads,dim,new", [(14, 2, 128, NEW), (4, 2, 64, NEW), (34, 2, 96, NEW), (4, 2, 256, NEW), (4, 2, 64, [60, 20, 1, 70])])
def test_rows_whose_scores_are_all_far(dtype, shared, value, heads, kv_heads, dim, new):
    case = far_case(dtype, heads, kv_heads, dim, value, new)
    _, out, lse = run(case, GROUP, TOKENS) if shared else alone(case)
    k0 = float(torch.tensor(value).to(dtype))
    got, z = out.double().cpu().numpy(), lse.double().cpu().numpy()
    q0 = case.q[..., 0].double().numpy()
    half = 2.0 ** -8 if dtype is BF16 else 2.0 ** -24
    assert np.isfinite(got).all() and np.isfinite(z).all()
    for b in range(case.B):
        _, v, _ = case.tokens(b)
        for i in range(case.new[b]):
            row, n = case.start[b] + i, case.lengths[b] - case.new[b] + i + 1
            for h in range(heads):
                vv = v[h // (heads // kv_heads)][:n]
                # sums over n tokens in 32 bits; p and the result rounded to the type (p in bf16 only)
                err = (n + 8) * 2.0 ** -23 * np.abs(vv).mean(0) + half * (np.abs(vv).mean(0) + np.abs(vv.mean(0))) * 1.01
                assert (np.abs(got[row, h] - vv.mean(0)) <= err).all()
                s = q0[row, h] * k0 * dim ** -0.5
                assert abs(z[row, h] - (s + np.log(n))) <= 2.0 ** -21 * (abs(s) + 10)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,dim", [(14, 2, 128), (4, 2, 64), (34, 2, 96), (4, 2, 256)])
@pytest.mark.parametrize("scale", [0.088, 1.0, 1.9, -0.7])
@pytest.mark.parametrize("order", ["up", "down", "mixed"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_the_largest_of_far_scores_has_all_weight(dtype, heads, kv_heads, dim, scale, order, sign):
    """Scores from some 2^26 to 2^34, in base 2, each 1/256 and more of it from the next: p is 1 for one token and 0 for the
    others, and out is its value. In float32 bit for bit; in bf16 the power of what a reference of less than 2^30 has
    lost, which is not 1, is rounded where it multiplies v and not in the sum, and the quotient again: 2^-8 each."""
    n, new = 1040, 40
    case = Case(52, [n], [new], heads, kv_heads, dim, 16, dtype)
    value = sign * np.array([(1 + (i % 128) / 128) * 2.0 ** (26 + i // 128) for i in range(n)])
    by_score = np.argsort(value * scale)
    at = {"up": by_score, "down": by_score[::-1], "mixed": np.random.default_rng(5).permutation(n)}[order]
    case.q[:] = 0
    case.q[..., 0] = 1
    case.k[~torch.isnan(case.k)] = 0
    for j in range(n):
        case.k[int(case.pages[0, j // 16]), :, j % 16, 0] = value[at[j]]
    import paper_2604_02945_amd as msao
    cache, start = case.device(DEV)
    lse = torch.zeros(new, heads, device=DEV)
    out = msao.msao_cache_attention(cache, start, new, case.q.to(DEV), scale=scale, lse=lse)
    _, v, _ = case.tokens(0)
    tol = 2.02 * 2.0 ** -8 if dtype is BF16 else 0.0
    for i in range(new):
        best = int(np.argmax(value[at[:n - new + i + 1]] * scale))
        for h in range(heads):
            want = v[h // (heads // kv_heads), best]
            assert (np.abs(out[i, h].double().cpu().numpy() - want) <= tol * np.abs(want)).all()
        s = value[at[best]] * scale
        assert (np.abs(lse[i].double().cpu().numpy() - s) <= 2.0 ** -21 * abs(s)).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shared", [False, True], ids=["alone", "shared"])
@pytest.mark.parametrize("value", [-1e30, 1e30, 1e10, -3e9, 5e8, -1e6, 100.0])
@pytest.mark.parametrize("heads,kv_heads,dim,new", [(14, 2, 128, NEW), (4, 2, 64, NEW), (4, 2, 64, [60, 20, 1, 70]), (34, 2, 96, [40, 3, 1, 2]), (4, 2, 256, NEW)])
def test_weights_of_far_scores(dtype, shared, value, heads, kv_heads, dim, new):
    """A row past 2^24 in base 2 adds nothing; of another the tokens' weights are the 1 / n that they are, times 2 to the
    power of what lse has lost, 2^-24 of it at most, and of the other roundings of exponents of that size."""
    case = far_case(dtype, heads, kv_heads, dim, value, new)
    cache, _, _ = run(case, GROUP, TOKENS, accumulate=True) if shared else alone(case, True)
    got = cache.weight.double().cpu().numpy() - case.weight.double().numpy()
    z = case.q[..., 0].double().numpy() * float(torch.tensor(value).to(dtype)) * dim ** -0.5 / np.log(2)
    far = np.abs(z) >= 2.0 ** 24 * 1.001
    assert (far | (np.abs(z) < 2.0 ** 24 * 0.999)).all()
    G = heads // kv_heads
    for b in range(case.B):
        for g in range(kv_heads):
            least, most = np.zeros(case.cap), np.zeros(case.cap)
            for i in range(case.new[b]):
                row, n = case.start[b] + i, case.lengths[b] - case.new[b] + i + 1
                for h in range(g * G, (g + 1) * G):
                    if far[row, h]:
                        continue
                    off = 2.0 ** (4 * 2.0 ** -24 * abs(z[row, h]) + 2.0 ** -10)
                    least[:n] += 1 / n / off
                    most[:n] += 1 / n * off
            # (added in 32 bits to a weight of up to 1)
            assert (got[b, g] >= least - 2.0 ** -22).all() and (got[b, g] <= most + 2.0 ** -22 * (1 + most)).all()
