"""The rotation's angles in float32 against 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("far", [16, 1000, 100000])
def test_float32_turns_are_rounded_near_zero(far, interleaved):
    """Pairs (1, 0) and (0, 1) turn into the cosine and the sine themselves. The angle is a turn in
    64 bits, brought next to the nearest quarter: at most an eighth of a turn is rounded to 24 bits, by
    2^-28 of a turn at most (half a step below 1/8), 2 pi 2^-28 rad; the sine and cosine of a float are
    off by at most 2 of their steps (2^-24 below 1); the product with 1 and the sum with 0 are exact.
    The 64-bit angle itself: positions of 17 bits, two products, 2^-52 2 pi 17,000 turns."""
    import paper_2604_02945_amd as msao
    rows, D, page = 512, 256, 16
    g = torch.Generator().manual_seed(81)
    half = D // 2
    inv = (2.0 * torch.rand(half, generator=g)).float()
    pos = torch.randint(-far, far, (rows,), generator=g, dtype=torch.int32)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)  # noqa: E731
    pool = torch.zeros(1, 1, page, D, device=DEV)
    cache = msao.KvCache(pool, pool.clone(), i32(1, 1), i32(1))
    x = torch.zeros(rows, 2, D)
    i = torch.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    x[:, 0, a] = 1
    x[:, 1, b] = 1
    zero = torch.zeros(rows, 1, D, device=DEV)
    start = torch.tensor([0, rows], dtype=torch.int32, device=DEV)
    y = msao.msao_cache_append(cache, start, rows, zero, zero, q=x.to(DEV), positions=pos.to(DEV), inv_freq=inv.to(DEV),
                               interleaved=interleaved).double().cpu()
    t = pos.double()[:, None] * inv.double()[None]
    tol = 2 * math.pi * 2.0 ** -28 + 2 * 2.0 ** -24 + 2 * math.pi * 2 * far / 6 * 2.0 ** -52
    for got, want in ((y[:, 0, a], t.cos()), (y[:, 0, b], t.sin()), (y[:, 1, a], -t.sin()), (y[:, 1, b], t.cos())):
        assert (got - want).abs().max() <= tol


def test_whole_and_quarter_turns():
    """Angles next to multiples of a quarter turn, whose sines or cosines are next to 0, from both sides."""
    import paper_2604_02945_amd as msao
    D, half = 64, 32
    quarter = torch.tensor([math.pi / 2], dtype=torch.float32)
    inv = torch.cat([torch.nextafter(quarter, quarter * 0), quarter, torch.nextafter(quarter, quarter * 2),
                     torch.tensor([0.0])]).repeat(8)
    pos = torch.arange(-40, 41, dtype=torch.int32)
    rows = pos.numel()
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)  # noqa: E731
    pool = torch.zeros(1, 1, 16, D, device=DEV)
    cache = msao.KvCache(pool, pool.clone(), i32(1, 1), i32(1))
    x = torch.zeros(rows, 1, D)
    x[..., :half] = 1
    zero = torch.zeros(rows, 1, D, device=DEV)
    start = torch.tensor([0, rows], dtype=torch.int32, device=DEV)
    y = msao.msao_cache_append(cache, start, rows, zero, zero, q=x.to(DEV), positions=pos.to(DEV),
                               inv_freq=inv.to(DEV)).double().cpu()[:, 0]
    t = pos.double()[:, None] * inv.double()[None]
    tol = 2 * math.pi * 2.0 ** -28 + 2 * 2.0 ** -24
    assert (y[:, :half] - t.cos()).abs().max() <= tol and (y[:, half:] - t.sin()).abs().max() <= tol
    assert (y[:, 3] == 1).all() and (y[:, half + 3] == 0).all()
