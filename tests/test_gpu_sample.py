"""Tokens drawn on the GPU against their definition in 64 bits. Indices have to be equal: both
sides compare 64-bit sums, which are off by about 1e-13 of a row's whole, and no running sum of the
inputs here lies that near to a number it is compared with by chance. ln p is a 64-bit value rounded
to 32 bits: off by 2^-24 of itself, and by the sums' 1e-13."""
import numpy as np
import pytest
import torch

import round_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
NAN, INF = float("nan"), float("inf")


def rows_of(seed, rows, vocab, dtype, sigma=2.0, boost=6.0):
    """[rows, vocab] logits, flat and confident ones, as a view of rows padded with NaN to 16 bytes."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, vocab, generator=g) * sigma * torch.rand(rows, 1, generator=g)
    at = torch.randint(vocab, (rows, 3), generator=g)
    x.scatter_add_(1, at, torch.rand(rows, 3, generator=g) * boost)
    return x.to(dtype)


def device_rows(x):
    """The rows on the device at a pitch of 16 bytes or more, and the tensor they are the first columns of."""
    pitch = -(-x.shape[1] // 8) * 8 + 8
    y = torch.full((x.shape[0], pitch), NAN, dtype=x.dtype)
    y[:, :x.shape[1]] = x
    return y.to(DEV)


def settings_of(seed, rows, kinds="tkpm"):
    g = np.random.default_rng(seed)
    pick = lambda v, t: torch.tensor(g.choice(v, rows), dtype=t)  # noqa: E731
    s = {"temperature": pick([0.0, 0.3, 0.7, 1.0, 1.3, 4.0], F32), "top_k": pick([-1, 0, 1, 2, 17, 50, 400, 10 ** 9], torch.int32),
         "top_p": pick([0.0, 0.1, 0.5, 0.9, 0.99, 1.0, 2.0], F32), "min_p": pick([0.0, 0.001, 0.05, 0.5, 1.0], F32)}
    return {k: v if k[0] in kinds or k[-1] in kinds else None for k, v in s.items()} if kinds != "tkpm" else s


def none():
    return {"temperature": None, "top_k": None, "top_p": None, "min_p": None}


def check(x, u, settings, **kw):
    import paper_2604_02945_amd as msao
    dev = {k: None if v is None else v.to(DEV) for k, v in settings.items()}
    got = msao.msao_sample(device_rows(x), u.to(DEV), vocab=x.shape[1], **dev, **kw)
    torch.cuda.synchronize()
    host = {k: None if v is None else v.numpy() for k, v in settings.items()}
    token, lp, kept = ref.sample(x.double().numpy(), u.numpy(), host)
    got = {k: v.cpu().numpy() for k, v in got.items()}
    assert np.array_equal(got["kept"], kept), (got["kept"], kept)
    assert np.array_equal(got["token"], token), (got["token"], token)
    bad = token < 0
    assert np.isnan(got["logprob"][bad]).all()
    assert (np.abs(got["logprob"][~bad] - lp[~bad]) <= 2.0 ** -24 * np.abs(lp[~bad]) + 1e-12).all()
    return got


def uniform(seed, rows):
    return torch.rand(rows, generator=torch.Generator().manual_seed(seed))


VOCABS = [1, 2, 3, 7, 8, 9, 64, 511, 1000, 4095, 4096, 4097, 8191, 8192, 8193, 20011]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("vocab", VOCABS)
def test_settings_of_every_kind_at_every_edge(dtype, vocab):
    check(rows_of(vocab, 40, vocab, dtype), uniform(vocab, 40), settings_of(vocab, 40))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("only", ["temperature", "top_k", "top_p", "min_p", None])
def test_one_setting_alone(dtype, only):
    s = {k: v if k == only else None for k, v in settings_of(3, 64).items()}
    check(rows_of(5, 64, 12345, dtype), uniform(6, 64), s)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_large_vocabularies(dtype):
    for vocab, rows in ((151936, 24), (152063, 5), (1 << 20, 3)):
        check(rows_of(7, rows, vocab, dtype), uniform(8, rows), settings_of(9, rows))
        check(rows_of(10, rows, vocab, dtype, sigma=0.5, boost=0.0), uniform(11, rows), {**none(), "top_p": torch.full((rows,), 0.9)})
        check(rows_of(12, rows, vocab, dtype), uniform(13, rows), none())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_equal_logits_stay_by_their_index(dtype):
    """Few different values, and rows of one value: sums are exact, numbers meet them."""
    g = torch.Generator().manual_seed(20)
    for vocab in (8, 1024, 9000):
        x = torch.randint(0, 3, (30, vocab), generator=g).to(dtype)
        s = {"temperature": None, "top_k": torch.randint(1, vocab, (30,), generator=g, dtype=torch.int32), "top_p": None, "min_p": None}
        check(x, uniform(21, 30), s)
        same = torch.full((9, vocab), -1.5, dtype=dtype)
        p = torch.tensor([0.0, 0.125, 0.25, 0.5, 0.75, 0.875, 1.0, 0.5, 0.5])
        u = torch.tensor([0.0, 0.125, 0.25, 0.5, 0.75, 0.875, 0.5, 0.25, 1.0])
        check(same, u, {**none(), "top_p": p})
        check(same, u, {**none(), "top_k": torch.arange(1, 10, dtype=torch.int32)})
        check(same, u, none())
        check(same * 0, u, {**none(), "min_p": torch.ones(9)})
    x = torch.tensor([[0.0, -0.0, 0.0, -1.0] * 4] * 6).to(dtype)  # zeros of both signs are one value
    check(x, torch.tensor([0.0, 0.3, 0.6, 0.9, 0.999, 0.1]), {**none(), "top_k": torch.arange(1, 7, dtype=torch.int32)})
    check(x, torch.tensor([0.0, 0.3, 0.6, 0.9, 0.999, 0.1]), {**none(), "temperature": torch.zeros(6)})


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_masked_logits(dtype):
    """-inf and the type's lowest value; rows with nothing left, with NaN, with +inf."""
    x = rows_of(30, 16, 5000, dtype)
    low = torch.finfo(dtype).min
    x[0, 10:] = -INF
    x[1, :-1] = -INF
    x[2] = -INF
    x[3, 100] = NAN
    x[4, 4999] = INF
    x[5, 5:] = low
    x[6] = low
    x[7, ::2] = -INF
    x[8, 1:] = -INF
    x[9, 4999] = NAN
    x[10] = -INF
    x[10, 77] = low
    x[11, :] = -INF
    x[11, 3] = x[11, 4] = torch.finfo(dtype).max
    x[12] = low
    x[12, 13] = torch.finfo(dtype).max
    for s in (none(), settings_of(31, 16), {**none(), "top_k": torch.full((16,), 50, dtype=torch.int32)},
              {**none(), "top_p": torch.full((16,), 0.9)}, {**none(), "temperature": torch.zeros(16)}):
        got = check(x, uniform(32, 16), s)
        assert (got["token"][[2, 3, 4, 9]] == -1).all() and got["token"][1] == 4999 and got["token"][8] == 0


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_numbers_and_settings_at_their_ends(dtype):
    u = torch.tensor([0.0, -1.0, NAN, 1.0, 2.0, INF, -INF, 1 - 2.0 ** -24, 2.0 ** -149, 1e-30])
    x = rows_of(40, 10, 3000, dtype)
    x[3:6, 2990:] = -INF
    check(x, u, none())
    check(x, u, {**none(), "top_k": torch.full((10,), 7, dtype=torch.int32)})
    t = torch.tensor([1e-45, 1e-38, 1e-4, 1e4, 3e38, INF, NAN, -1.0, -0.0, 0.05])
    for s in (none(), {"top_k": torch.full((10,), 20, dtype=torch.int32)}, {"top_p": torch.full((10,), 0.7)}, {"min_p": torch.full((10,), 0.2)}):
        check(x, uniform(41, 10), {**none(), **s, "temperature": t})
    p = torch.tensor([NAN, -1.0, 0.0, 1e-30, 1 - 2.0 ** -24, 1 - 2.0 ** -12, 1.0, INF, -INF, 0.5])
    check(x, uniform(42, 10), {**none(), "top_p": p})
    check(x, uniform(43, 10), {**none(), "min_p": p})
    k = torch.tensor([-2 ** 31, -1, 0, 1, 2, 2999, 3000, 3001, 2 ** 31 - 1, 1500], dtype=torch.int32)
    check(x, uniform(44, 10), {**none(), "top_k": k})
    check(x, uniform(45, 10), {**none(), "top_k": k, "top_p": torch.full((10,), 0.6)})


def test_a_draw_reaches_every_token_by_its_weight():
    """Numbers in the middle of each token's share give each token."""
    x = torch.tensor([[0.5, -1.0, 2.0, 0.0, -3.0, 1.0, 0.25, -0.5]])
    p = ref.distribution(x[0].double().numpy())[2]
    u = torch.from_numpy((np.cumsum(p) - p / 2).astype(np.float32))
    got = check(x.repeat(8, 1), u, none())
    assert got["token"].tolist() == list(range(8))


def families(seed, rows, vocab, dtype):
    """Rows of every kind of spread: even, two clusters, few values, values far apart and nearly equal, steps of the type,
    many masked, a heavy token in a flat row."""
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x = n(rows, vocab)
    low = torch.finfo(dtype).min
    for r in range(rows):
        k = r % 10
        if k == 1:
            x[r] = torch.where(torch.rand(vocab, generator=g) < 0.3, x[r] * 0.1, x[r] - 9)
        elif k == 2:
            x[r] = torch.randint(0, 5, (vocab,), generator=g) * 0.5
        elif k == 3:
            x[r] = x[r] * 10.0 ** torch.randint(-6, 30, (vocab,), generator=g)
        elif k == 4:
            x[r] = 1.0 + x[r] * 1e-6
        elif k == 5:
            x[r] = torch.rand(vocab, generator=g) * 0.01 - 0.005
        elif k == 6:
            x[r, torch.rand(vocab, generator=g) < 0.9] = low
        elif k == 7:
            x[r, torch.rand(vocab, generator=g) < 0.9] = -INF
        elif k == 8:
            x[r, int(torch.randint(vocab, (1,), generator=g))] = 11.0
        elif k == 9:
            x[r] *= 0.3
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1025, 2049, 6000, 17000, 70001])
def test_every_spread_with_every_setting(dtype, vocab):
    rows = 40
    x = families(vocab, rows, vocab, dtype)
    g = np.random.default_rng(vocab)
    f = lambda v: torch.tensor(g.choice(v, rows), dtype=F32)  # noqa: E731
    k = torch.tensor(g.choice([3, 300, 1000, 1024, 1025, 1500, vocab // 2, vocab - 1], rows), dtype=torch.int32)
    p, m, t = f([0.05, 0.5, 0.9, 0.99, 0.9999, 1 - 2.0 ** -20]), f([1e-9, 1e-4, 0.01, 0.3]), f([0.1, 0.7, 1.0, 3.0, 100.0])
    for i, s in enumerate(({"top_k": k}, {"top_p": p}, {"min_p": m}, {"top_k": k, "top_p": p}, {"top_p": p, "min_p": m},
                           {"top_k": k, "top_p": p, "min_p": m, "temperature": t}, {"top_p": p, "temperature": t}, {"temperature": t})):
        check(x, uniform(vocab + i, rows), {**none(), **s})


def test_logits_past_four_gigabytes():
    """Rows by offsets of 64 bits: the last rows of many are those of a call of their own."""
    import paper_2604_02945_amd as msao
    rows, vocab = 15000, 151936
    x = torch.zeros(rows, vocab, dtype=BF16, device=DEV)
    x[-6:] = rows_of(80, 6, vocab, BF16).to(DEV)
    x[:-6, 7::1000] = 20.0
    u = uniform(81, rows).to(DEV)
    s = {k: None if v is None else v.repeat(rows // 6).to(DEV) for k, v in settings_of(82, 6).items()}
    got = msao.msao_sample(x, u, **s)
    last = {k: None if v is None else v[-6:].clone() for k, v in s.items()}
    want = msao.msao_sample(x[-6:].clone(), u[-6:].clone(), **last)
    for k in want:
        assert torch.equal(got[k][-6:], want[k]), k
    start = torch.arange(0, rows + 1, 6, dtype=torch.int32, device=DEV)
    tokens = torch.full((rows,), 7, dtype=torch.int32, device=DEV)
    got = msao.msao_verify(start, 6, tokens, x, u, u, **s)
    want = msao.msao_verify(start[:2].clone(), 6, tokens[-6:].clone(), x[-6:].clone(), u[-6:].clone(), u[-6:].clone(), **last)
    assert torch.equal(got["next"][-6:], want["next"]) and torch.equal(got["accepted"][-1:], want["accepted"])


def test_outputs_one_by_one_streams_and_repeats():
    import paper_2604_02945_amd as msao
    x, u = device_rows(rows_of(50, 9, 40000, BF16)), uniform(51, 9).to(DEV)
    s = {k: v.to(DEV) for k, v in settings_of(52, 9).items()}
    want = msao.msao_sample(x, u, vocab=40000, **s)
    for k in ("token", "logprob", "kept"):
        o = {k: torch.zeros_like(want[k])}
        assert msao.msao_sample(x, u, vocab=40000, outputs=o, **s) is o and torch.equal(o[k], want[k])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = msao.msao_sample(x, u, vocab=40000, stream=side, **s)
    torch.cuda.synchronize()
    again = msao.msao_sample(x, u, vocab=40000, **s)
    for k in want:
        assert torch.equal(got[k], want[k]) and torch.equal(again[k], want[k])
    assert msao.msao_sample(x[:0], u[:0], vocab=40000)["token"].shape == (0,)
    one = msao.msao_sample(x[3:4], u[3:4], vocab=40000, **{k: v[3:4] for k, v in s.items()})
    assert torch.equal(one["token"], want["token"][3:4])


def test_replays_follow_their_inputs():
    import paper_2604_02945_amd as msao
    x, u = device_rows(rows_of(60, 12, 33333, BF16)), uniform(61, 12).to(DEV)
    s = {k: v.to(DEV) for k, v in settings_of(62, 12).items()}
    o = {"token": torch.zeros(12, dtype=torch.int32, device=DEV), "logprob": torch.zeros(12, device=DEV),
         "kept": torch.zeros(12, dtype=torch.int32, device=DEV)}
    msao.msao_sample(x, u, vocab=33333, outputs=o, **s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        msao.msao_sample(x, u, vocab=33333, outputs=o, **s)
    for i in range(4):
        x.copy_(device_rows(rows_of(63 + i, 12, 33333, BF16)))
        u.copy_(uniform(70 + i, 12))
        s["top_p"].fill_(0.3 + 0.2 * i)
        for t in o.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = {k: t.clone() for k, t in o.items()}
        want = msao.msao_sample(x, u, vocab=33333, **s)
        for k in want:
            assert torch.equal(got[k], want[k]), k
