"""Attention of sequences that share prefixes: chunks of prompts of several tiles of rows behind one, and keys and
values that are not finite in it and behind it. Tolerances as in the other tests of shared prefixes; what holds no
finite value is compared by what the definition gives there, everything else by bits with the call without it."""
import pytest
import torch

from cache_ref import Case
from test_gpu_cache_shared import check, run, share

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
SHAPES = [(14, 2, 128), (4, 2, 64), (34, 2, 96), (4, 2, 256)]
LENGTHS, NEW, GROUP, TOKENS = [1100, 1060, 1043, 70], [9, 3, 1, 2], [0, 3], [1040]  # the last sequence is in no group


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
@pytest.mark.parametrize("heads,kv_heads,dim,page", [(4, 2, 64, 16), (28, 4, 128, 64), (7, 1, 96, 16), (8, 1, 256, 32), (5, 5, 128, 128)])
def test_chunks_of_prompts_behind_a_prefix(dtype, causal, heads, kv_heads, dim, page):
    """Sequences that share and have rows for one, two and many tiles, and one tile's last or first row."""
    prefix, own, new = 400, [300, 129, 128, 64, 33, 1], [290, 129, 127, 64, 17, 1]
    case = Case(41, [prefix + n for n in own] + [77], new + [70], heads, kv_heads, dim, page, dtype)
    check(share(case, [0, 4, 6], [prefix, prefix - 16]), [0, 4, 6], [prefix, prefix - 16], causal)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_a_long_chunk_behind_a_long_prefix(dtype):
    """Parts of both; the host's bounds right, and too small."""
    case = share(Case(42, [3300, 2600, 2560], [700, 41, 5], 4, 1, 128, 64, dtype), [0, 3], [2512])
    check(case, [0, 3], [2512])
    check(case, [0, 3], [2512], max_seqs=1, max_own=64, accumulate=False)


def both(case, change):
    """The call on the case, and on the case after change(case)."""
    share(case, GROUP, TOKENS)
    a = run(case, GROUP, TOKENS, accumulate=True)
    change(case)
    b = run(case, GROUP, TOKENS, accumulate=True)
    return [x.cpu() for x in (a[1], a[2], a[0].weight)], [x.cpu() for x in (b[1], b[2], b[0].weight)]


def place(case, s, j):
    return int(case.pages[s, j // case.page]), j % case.page


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")], ids=str)
@pytest.mark.parametrize("heads,kv_heads,dim", SHAPES)
@pytest.mark.parametrize("at", [0, 700, 1039])
def test_values_of_a_prefix_that_are_not_finite(dtype, value, heads, kv_heads, dim, at):
    """Their channels in every row that shares them, and nothing else."""
    def change(c):
        page, slot = place(c, 0, at)
        c.v[page, 1, slot, 3] = c.v[page, 1, slot, dim - 1] = value
    a, b = both(Case(43, LENGTHS, NEW, heads, kv_heads, dim, 16, dtype), change)
    hit = torch.zeros(sum(NEW), heads, dim, dtype=torch.bool)
    hit[:sum(NEW[:3]), heads // 2:, [3, dim - 1]] = True
    assert torch.equal(a[0][~hit], b[0][~hit]) and torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
    assert (torch.isnan(b[0][hit]) if value != value else b[0][hit] == value).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")], ids=str)
@pytest.mark.parametrize("heads,kv_heads,dim", SHAPES)
def test_values_behind_a_prefix_that_some_rows_do_not_see(dtype, value, heads, kv_heads, dim):
    """The first sequence's row 4 on, and nothing else."""
    def change(c):
        page, slot = place(c, 0, LENGTHS[0] - NEW[0] + 4)
        c.v[page, 1, slot, 5] = value
    a, b = both(Case(44, LENGTHS, NEW, heads, kv_heads, dim, 16, dtype), change)
    hit = torch.zeros(sum(NEW), heads, dim, dtype=torch.bool)
    hit[4:9, heads // 2:, 5] = True
    assert torch.equal(a[0][~hit], b[0][~hit]) and torch.equal(a[1], b[1])
    assert (torch.isnan(b[0][hit]) if value != value else b[0][hit] == value).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")], ids=str)
@pytest.mark.parametrize("heads,kv_heads,dim", SHAPES)
@pytest.mark.parametrize("at", [0, 700, 1039, 1091])
def test_keys_that_are_not_finite(dtype, value, heads, kv_heads, dim, at):
    """A score that is NaN or inf makes the rows that see it NaN; the others are as without it."""
    case = Case(45, LENGTHS, NEW, heads, kv_heads, dim, 16, dtype)
    case.q[..., 2] = case.q[..., 2].abs() + 1

    def change(c):
        page, slot = place(c, 0, at)
        c.k[page, 1, slot, 2] = value
    a, b = both(case, change)
    hit = torch.zeros(sum(NEW), heads, dtype=torch.bool)
    hit[slice(0, sum(NEW[:3])) if at < 1040 else slice(at - (LENGTHS[0] - NEW[0]), NEW[0]), heads // 2:] = True
    assert hit.any() and torch.isnan(b[0][hit]).all() and not torch.isfinite(b[1][hit]).any()
    assert torch.equal(a[0][~hit], b[0][~hit]) and torch.equal(a[1][~hit], b[1][~hit])


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,dim", SHAPES)
def test_parts_without_any_weight(dtype, heads, kv_heads, dim):
    """Every token of the prefix, of the prefix' first or last part, of the own ones, or all of a sequence at -inf: as at
    a score of -1e30, but for a row that sees nothing else, which gets 0 and -inf, whatever the values hold."""
    part = 256 if dtype is BF16 else 128
    for lo, hi in ((0, 1040), (0, part), (1040 - part, 1040), (16, 1024), (1040, LENGTHS[0])):
        got = []
        for value in (-1e30, float("-inf")):
            case = share(Case(46, LENGTHS, NEW, heads, kv_heads, dim, 16, dtype), GROUP, TOKENS)
            case.q[..., 0] = case.q[..., 0].abs() + 1
            for j in range(lo, hi):
                page, slot = place(case, 0, j)
                case.k[page, :, slot, 0] = value
            cache, out, lse = run(case, GROUP, TOKENS, accumulate=True)
            got.append((out, lse, cache.weight))
        for x, y in zip(*got):
            assert torch.isfinite(x).all() and torch.equal(x, y)
    case = share(Case(47, LENGTHS, NEW, heads, kv_heads, dim, 16, dtype), GROUP, TOKENS)
    case.q[..., 0] = case.q[..., 0].abs() + 1
    for j in range(LENGTHS[0]):
        page, slot = place(case, 0, j)
        case.k[page, :, slot, 0] = float("-inf")
    page, slot = place(case, 0, 333)
    case.v[page, :, slot, 7] = float("nan")
    cache, out, lse = run(case, GROUP, TOKENS, accumulate=True)
    assert (out[:9] == 0).all() and (lse[:9] == float("-inf")).all() and torch.equal(cache.weight[0].cpu(), case.weight[0])
    # the others have tokens of their own, and see the value
    rest = [d for d in range(dim) if d != 7]
    assert torch.isfinite(lse[9:]).all() and torch.isfinite(out[9:][..., rest]).all() and torch.isnan(out[9:13][..., 7]).all()
    assert torch.isfinite(out[13:]).all()
