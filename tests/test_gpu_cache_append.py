"""Append to a paged cache on the GPU (head norms, position rotation, keys and
values into their pages) against its definition in 64 bits."""
import numpy as np
import pytest
import torch

from cache_ref import Case

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-5


def turned(x, w, angle, interleaved):
    """The definition; and the magnitude that 32-bit rounding errors go by."""
    x = x.double().numpy()
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + EPS) * w.double().numpy()
    mag = np.abs(x)
    if angle is not None:
        half = angle.shape[1]
        i = np.arange(half)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        y = x.copy()
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
        m = np.abs(x[..., a]) + np.abs(x[..., b])
        mag = mag.copy()
        mag[..., a], mag[..., b] = m, m
        x = y
    return x, mag


def run(dtype, heads, kv_heads, dim, rot, axes=1, interleaved=False, norm=True, page=16, order="head", bad_page=None,
        new=(3, 0, 1, 40, 7), lengths=(20, 0, 1, 40, 100), positions=True, far=100000, in_place=False, extra=2, max_new=None):
    import paper_2604_02945_amd as msao
    case = Case(21, list(lengths), list(new), heads, kv_heads, dim, page, dtype, extra_rows=extra, order=order,
                bad_page=bad_page)
    g = case.g
    T = case.rows
    k_new, v_new = (torch.randn(T, kv_heads, dim, generator=g).to(dtype) * 2 for _ in range(2))
    qw, kw = ((1 + 0.3 * torch.randn(dim, generator=g)).to(dtype) if norm else None for _ in range(2))
    half = rot // 2
    inv = (10000.0 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))).float()
    pos = torch.randint(-far, far, (axes, T), generator=g, dtype=torch.int32) if positions else None
    sec = [half] if axes == 1 else [half // 4] * (axes - 1) + [half - half // 4 * (axes - 1)]
    cache, start = case.device(DEV)
    before_k, before_v, before_w = cache.k.clone(), cache.v.clone(), cache.weight.clone()
    q = case.q.to(DEV)
    q_out = q if in_place else torch.full_like(q, 7.0)
    d = lambda x: None if x is None else x.to(DEV)  # noqa: E731
    msao.msao_cache_append(cache, start, case.max_new, d(k_new), d(v_new), q=q, q_out=q_out, q_norm=d(qw), k_norm=d(kw),
                           eps=EPS, positions=d(pos), inv_freq=d(inv) if rot else None, sections=sec if rot else None,
                           interleaved=interleaved) if rot else \
        msao.msao_cache_append(cache, start, case.max_new, d(k_new), d(v_new), q=q, q_out=q_out, q_norm=d(qw),
                               k_norm=d(kw), eps=EPS)
    torch.cuda.synchronize()
    place = np.zeros((1, T), np.int64)
    for b in range(case.B):
        s, e = case.start[b], case.start[b + 1]
        place[0, s:e] = case.lengths[b] - (e - s) + np.arange(e - s)
    angle = None
    if rot:
        axis = np.repeat(np.arange(axes), sec)
        at = pos.numpy().astype(np.float64) if positions else np.repeat(place, axes, 0).astype(np.float64)
        angle = at[axis].T * inv.double().numpy()
    want_q, mag_q = turned(case.q, qw, angle, interleaved)
    want_k, mag_k = turned(k_new, kw, angle, interleaved)
    half_step = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24

    def near(got, want, mag):
        # 32 bits: the norm's sum, root and products (dim + 8 roundings at most), the angle as
        # a turn (2^-25 of one: 2^-22 rad) and its sine and cosine, two products and a sum
        tol = half_step * np.abs(want) * 1.01 + mag * ((dim + 8) * 2.0 ** -24 + 2.0 ** -21)
        return (np.abs(got.double().cpu().numpy() - want) <= tol).all()

    mine = np.arange(T) < case.start[-1]
    assert near(q_out[mine], want_q[mine], mag_q[mine])
    if not in_place:
        assert (q_out[~mine] == 7).all()
    wk, wv, ww = before_k.clone(), before_v.clone(), before_w.clone()
    for b in range(case.B):
        for r in range(case.start[b], case.start[b + 1]):
            j = int(place[0, r])
            if j < 0:
                continue
            ww[b, :, j] = 0
            p = case.pages[b, j // page]
            if not 0 <= p < case.n_pages:
                continue
            assert near(cache.k[p, :, j % page], want_k[r], mag_k[r])
            wk[p, :, j % page] = cache.k[p, :, j % page]
            wv[p, :, j % page] = v_new[r].to(DEV)
    bits = torch.int32 if dtype == F32 else torch.int16
    same = lambda a, b: torch.equal(a.contiguous().view(bits), b.contiguous().view(bits))  # noqa: E731
    assert same(cache.k, wk) and same(cache.v, wv)
    assert torch.equal(cache.weight, ww)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,dim,rot,axes,interleaved,norm", [
    (4, 2, 128, 128, 1, False, True), (28, 4, 128, 128, 3, False, True), (32, 8, 128, 64, 1, True, False),
    (3, 1, 96, 64, 2, True, True), (5, 5, 80, 80, 4, False, True), (8, 1, 256, 256, 1, False, True),
    (2, 2, 8, 0, 1, False, True), (6, 3, 72, 16, 1, False, True), (4, 4, 200, 176, 1, True, False),
    (7, 7, 64, 32, 1, False, False), (40, 8, 64, 64, 3, True, True)])
def test_heads_and_rotations(dtype, heads, kv_heads, dim, rot, axes, interleaved, norm):
    run(dtype, heads, kv_heads, dim, rot, axes, interleaved, norm)


@pytest.mark.parametrize("order", ["token", "mixed"])
def test_pool_layouts(order):
    run(BF16, 4, 2, 64, 64, order=order, page=32)
    run(F32, 4, 2, 64, 64, order=order, page=32)


def test_positions_are_places_without_an_array():
    run(BF16, 4, 2, 128, 128, positions=False)


def test_far_positions_are_as_exact_as_near_ones():
    run(F32, 4, 2, 128, 128, far=2 ** 31 - 1)


def test_queries_in_place():
    run(BF16, 4, 2, 128, 128, in_place=True)


@pytest.mark.parametrize("bad", [-1, 10 ** 6])
def test_no_page_nothing_stored(bad):
    run(BF16, 4, 2, 64, 64, bad_page=(3, 1, bad))


def test_a_chunk_longer_than_the_cache():
    run(BF16, 4, 2, 64, 64, lengths=(5, 0, 16), new=(9, 3, 16))


def test_many_rows_and_many_sequences():
    run(BF16, 8, 2, 64, 64, lengths=tuple(i % 50 + 1 for i in range(300)), new=tuple(i % 4 for i in range(300)),
        extra=70)
    run(BF16, 4, 1, 64, 64, lengths=(1500, 2700), new=(1500, 2600))


def test_keys_alone():
    """An encoder's states: no queries, no norm, no rotation: stored as they are."""
    import paper_2604_02945_amd as msao
    case = Case(22, [50, 33], [50, 33], 4, 4, 96, 16, BF16)
    cache, start = case.device(DEV, with_weight=False)
    k, v = (torch.randn(83, 4, 96).to(BF16).to(DEV) for _ in range(2))
    assert msao.msao_cache_append(cache, start, 50, k, v) is None
    torch.cuda.synchronize()
    at = 0
    for b, n in enumerate([50, 33]):
        j = torch.arange(n)
        p = torch.from_numpy(case.pages[b][j // 16].astype(np.int64)).to(DEV)
        assert torch.equal(cache.k[p, :, (j % 16).to(DEV)], k[at:at + n])
        assert torch.equal(cache.v[p, :, (j % 16).to(DEV)], v[at:at + n])
        at += n
