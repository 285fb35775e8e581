"""Attention with shared prefixes whose groups' array descends: every sequence attends to what its own table
names, as if nothing were shared."""
import pytest
import torch

from cache_ref import Case
from test_gpu_cache_shared import check, run

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("group,tokens", [([0, 6, 2, 8, 1, 8], [64, 80, 48, 16, 96]), ([8, 0], [96]), ([4, 8, 0, 4], [64, 64, 64]),
                                          ([0, 8, 7], [80, 80]), ([0, 900, -5, 8], [96, 32, 64]), ([3, 2, 2, 8], [96, 96, 96])], ids=str)
def test_arrays_that_descend_share_nothing(dtype, group, tokens):
    """No two sequences hold the same keys here: whatever was shared would give another result."""
    case = Case(21, [100, 110, 120, 130, 105, 97, 140, 99], [1, 2, 1, 3, 1, 2, 1, 1], 4, 2, 64, 16, dtype)
    check(case, group, tokens, max_seqs=8, max_tokens=96)
    a, b = (run(case, group, tokens, max_seqs=8, max_tokens=96) for _ in range(2))
    assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])


def test_a_long_array_that_descends_at_its_end():
    """More groups than a wavefront has lanes; the last of them alone descends."""
    group, tokens = [2 * i for i in range(100)] + [100], [16] * 100
    check(Case(22, [40 + i % 30 for i in range(200)], [1] * 200, 4, 2, 64, 16, BF16), group, tokens, max_seqs=2, max_tokens=16)
