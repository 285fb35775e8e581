"""Verification of drafts on the GPU against its definition in 64 bits. Counts and tokens have to be
equal (see test_gpu_sample.py for why they can be); ln p is a 64-bit value rounded to 32 bits."""
import numpy as np
import pytest
import torch

import round_ref as ref
from test_gpu_sample import device_rows, families, none, rows_of, settings_of, uniform

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
NAN, INF = float("nan"), float("inf")


def make(seed, counts, vocab, dtype, drawn, extra=0, boost=6.0):
    """Rows whose drafts stand about half of the time."""
    rows = sum(counts) + extra
    x = rows_of(seed, rows, vocab, dtype, boost=boost)
    g = torch.Generator().manual_seed(seed + 1)
    y = (x.float() + 0.5 * torch.randn(x.shape, generator=g)).to(dtype)
    tokens = torch.zeros(rows, dtype=torch.int32)
    for r in range(rows - 1):
        p = ref.distribution(y[r].double().numpy())[2]
        tokens[r + 1] = ref.pick(p, float(torch.rand((), generator=g))) if drawn else int(p.argmax())
    start = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32)
    length = torch.tensor([c + 11 * i for i, c in enumerate(counts)], dtype=torch.int32)
    return x, y if drawn else None, tokens, start, length, torch.rand(rows, generator=g), torch.rand(rows, generator=g)


def check(x, y, tokens, start, length, ua, u, settings, max_new):
    import paper_2604_02945_amd as msao
    rows, V = x.shape
    o = {"accepted": torch.full((len(start) - 1,), 77, dtype=torch.int32, device=DEV),
         "next": torch.full((rows,), 77, dtype=torch.int32, device=DEV), "logprob": torch.full((rows,), 77.0, device=DEV),
         "length": torch.full((len(start) - 1,), 77, dtype=torch.int32, device=DEV)}
    msao.msao_verify(start.to(DEV), max_new, tokens.to(DEV), device_rows(x), ua.to(DEV), u.to(DEV), vocab=V,
                     draft_logits=None if y is None else device_rows(y), length=length.to(DEV), outputs=o,
                     **{k: None if v is None else v.to(DEV) for k, v in settings.items()})
    torch.cuda.synchronize()
    host = {k: None if v is None else v.numpy() for k, v in settings.items()}
    accepted, nxt, lp, out = ref.verify(start.tolist(), max_new, tokens.tolist(), x.double().numpy(),
                                        None if y is None else y.double().numpy(), ua.numpy(), u.numpy(), host, length.tolist())
    got = {k: v.cpu().numpy() for k, v in o.items()}
    assert got["accepted"].tolist() == accepted
    assert got["next"].tolist() == [77 if t is None else t for t in nxt]
    assert got["length"].tolist() == out
    for g, w in zip(got["logprob"], lp):
        assert g == 77 if w is None else np.isnan(g) if np.isnan(w) else abs(g - w) <= 2.0 ** -24 * abs(w) + 1e-12
    return accepted


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("drawn", [False, True], ids=["greedy", "drawn"])
@pytest.mark.parametrize("vocab", [2, 9, 1000, 8193, 30011])
def test_rounds(dtype, drawn, vocab):
    counts = [6, 1, 0, 2, 3, 6, 5, 1, 4, 6, 6, 2]
    args = make(vocab, counts, vocab, dtype, drawn, extra=2)
    rows = args[0].shape[0]
    some = check(*args, none(), 6)
    # (of flat rows of many tokens no greedy draft stands)
    assert vocab not in (9, 1000) or (max(some) > 0 and any(a < c - 1 for a, c in zip(some, counts) if c > 1))
    check(*args, settings_of(vocab, rows), 6)
    check(*args, {**none(), "temperature": torch.zeros(rows)}, 6)


@pytest.mark.parametrize("drawn", [False, True], ids=["greedy", "drawn"])
def test_large_vocabulary_and_long_drafts(drawn):
    check(*make(3, [70, 1, 130], 500, BF16, drawn), none(), 130)
    check(*make(4, [6, 6], 151936, BF16, drawn), settings_of(5, 12), 6)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("drawn", [False, True], ids=["greedy", "drawn"])
def test_confident_rows(dtype, drawn):
    args = make(12, [6, 6, 3, 6, 2, 6, 6, 6], 60001, dtype, drawn, boost=24.0)
    some = check(*args, none(), 6)
    assert max(some) > 1 and min(some) == 0
    check(*args, settings_of(13, 41), 6)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("drawn", [False, True], ids=["greedy", "drawn"])
@pytest.mark.parametrize("vocab", [1025, 5000, 40001])
def test_every_spread_with_every_setting(dtype, drawn, vocab):
    """Drafts of the likeliest, of light and of removed tokens; the rows they were drawn from of the same spread or another."""
    counts = [6, 4, 6, 1, 5, 6, 6, 6]
    rows = sum(counts)
    x = families(vocab, rows, vocab, dtype)
    y = (x.float() * 0.9).to(dtype) if vocab == 5000 else families(vocab + 1, rows, vocab, dtype)
    g = np.random.default_rng(vocab)
    order = torch.argsort(x.double(), dim=1, descending=True, stable=True)
    tokens = order[torch.arange(rows), torch.from_numpy(g.choice([0, 0, 0, 1, 7, vocab // 2], rows))].roll(1).to(torch.int32)
    start = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32)
    length = torch.full((len(counts),), 100, dtype=torch.int32)
    f = lambda v: torch.tensor(g.choice(v, rows), dtype=F32)  # noqa: E731
    k = torch.tensor(g.choice([1, 3, 300, 1024, 1025, 1500, vocab // 2, vocab - 1], rows), dtype=torch.int32)
    p, m, t = f([0.05, 0.5, 0.9, 0.99, 0.9999]), f([1e-9, 1e-4, 0.01, 0.3]), f([0.1, 0.7, 1.0, 3.0, 100.0])
    for i, s in enumerate(({}, {"top_k": k}, {"top_p": p}, {"min_p": m, "temperature": t}, {"top_k": k, "top_p": p},
                           {"top_k": k, "top_p": p, "min_p": m, "temperature": t})):
        check(x, y if drawn else None, tokens, start, length, uniform(vocab + i, rows) ** 2, uniform(vocab + i + 10, rows), {**none(), **s}, 6)


@pytest.mark.parametrize("drawn", [False, True], ids=["greedy", "drawn"])
def test_more_rows_than_max_new(drawn):
    args = make(6, [9, 2, 5, 0], 700, F32, drawn)
    for most in (1, 2, 4, 9, 100):
        check(*args, none(), most)


def test_drafts_that_equal_the_models_own_all_stand():
    """q = p: every draft stands, whatever the numbers."""
    x, y, tokens, start, length, ua, u = make(7, [8] * 6, 5000, BF16, True)
    ua = torch.full_like(ua, 1 - 2.0 ** -24)
    for r in range(x.shape[0] - 1):
        tokens[r + 1] = ref.pick(ref.distribution(x[r].double().numpy())[2], float(u[r]))
    assert check(x, x.clone(), tokens, start, length, ua, u, none(), 8) == [7] * 6


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("vocab", [40, 1024, 5000, 40000])
def test_equal_distributions_leave_nothing_between_them(dtype, vocab):
    """A draft that is no token never stands; where the draft's logits are the row's and a number more, whose steps every one of
    them keeps, nothing of p is above q, and the token is one of p."""
    g = torch.Generator().manual_seed(vocab)
    rows, many = 36, torch.tensor([1, 1.5, 40, 0.25, 3, 0.7]).repeat(6)
    x = (torch.randint(0, 64, (rows, vocab), generator=g) / 64 + 1.0).to(dtype)
    x[::2, :5] += 1.0
    x[::2] = (x[::2].float() * 32).round().div(32).clamp(max=1.96875).to(dtype)
    y = (x.float() - 0.5).to(dtype)
    assert torch.equal(y.double() + 0.5, x.double())
    tokens = torch.full((rows,), -1, dtype=torch.int32)
    start = torch.arange(0, rows + 1, 6, dtype=torch.int32)
    length = torch.full((6,), 9, dtype=torch.int32)
    k = torch.tensor([2, 3, 30, 1024, 1300, vocab - 1], dtype=torch.int32).repeat(6)
    for i, s in enumerate(({}, {"temperature": many}, {"top_k": k}, {"top_k": k, "temperature": many}, {"top_p": torch.full((rows,), 0.7)})):
        for first in range(6):  # (each row of a sequence of six is once its first)
            one = torch.cat([torch.zeros(1), start[1:] - (6 - first)]).clamp(min=0).to(torch.int32)
            check(x, y, tokens, one, length, uniform(i, rows), uniform(i + 50, rows), {**none(), **s}, 6)


@pytest.mark.parametrize("drawn", [False, True], ids=["greedy", "drawn"])
def test_rows_that_have_no_distribution_and_tokens_that_are_none(drawn):
    x, y, tokens, start, length, ua, u = make(8, [6, 6, 6, 6, 6, 3], 900, BF16, drawn)
    ua *= 0  # what can stand stands
    x[0] = -INF
    x[8, 5] = NAN
    x[17, 0] = INF
    tokens[20], tokens[25], tokens[27] = -1, 900, 2 ** 31 - 1
    if drawn:
        y[30], y[31, 4] = -INF, NAN
    check(x, y, tokens, start, length, ua, u, none(), 6)
    x[30:33, 4:] = -INF  # a draft of no weight, and nothing beside it
    x[30:33, :3] = -INF
    tokens[31] = 3
    check(x, y, tokens, start, length, torch.ones_like(ua), u, none(), 6)


def test_numbers_at_their_ends():
    x, y, tokens, start, length, ua, u = make(9, [5] * 10, 333, F32, True)
    ends = torch.tensor([0.0, 1.0, NAN, -3.0, 2.0 ** -149, INF, 1 - 2.0 ** -24, 0.5, -INF, 2.0])
    check(x, y, tokens, start, length, ends.repeat(5), ends.flip(0).repeat(5), none(), 5)
    check(x, None, tokens, start, length, ends.repeat(5), ends.flip(0).repeat(5), none(), 5)


def test_starts_out_of_order_and_out_of_range():
    x, y, tokens, _, length, ua, u = make(10, [3] * 5, 250, BF16, False)
    start = torch.tensor([-4, 3, 3, 2, 9, 500], dtype=torch.int32)  # 0..3, none, none, 2..9 (rows 2 of two), 9..15
    import paper_2604_02945_amd as msao
    o = msao.msao_verify(start.to(DEV), 20, tokens.to(DEV), device_rows(x), ua.to(DEV), u.to(DEV), vocab=250, length=length.to(DEV))
    torch.cuda.synchronize()
    acc, nxt, _, out = ref.verify([0, 3, 3, 3, 9, 15], 20, tokens.tolist(), x.double().numpy(), None, ua.numpy(), u.numpy(), none(), length.tolist())
    assert o["accepted"].tolist()[0] == acc[0] and o["accepted"].tolist()[1:3] == [0, 0] and o["accepted"].tolist()[4] == acc[4]
    assert o["next"].tolist()[9:] == nxt[9:]


def test_replays_follow_their_inputs_and_lengths_in_place():
    import paper_2604_02945_amd as msao
    x, y, tokens, start, length, ua, u = make(11, [6, 2, 4, 6], 20000, BF16, True)
    dev = [t.to(DEV) for t in (start, tokens, device_rows(x), ua, u, device_rows(y))]
    o = {"accepted": torch.zeros(4, dtype=torch.int32, device=DEV), "next": torch.zeros(18, dtype=torch.int32, device=DEV),
         "logprob": torch.zeros(18, device=DEV), "length": length.to(DEV)}

    def call():
        msao.msao_verify(dev[0], 6, dev[1], dev[2], dev[3], dev[4], vocab=20000, draft_logits=dev[5], length=o["length"], outputs=o)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        a = make(20 + i, [[6, 2, 4, 6], [1, 6, 5, 6], [0, 6, 6, 6], [6, 6, 6, 0]][i], 20000, BF16, True)
        for d, t in zip(dev, (a[3], a[2], device_rows(a[0]), a[5], a[6], device_rows(a[1]))):
            d.copy_(t)
        o["length"].copy_(a[4])
        graph.replay()
        torch.cuda.synchronize()
        acc, nxt, _, out = ref.verify(a[3].tolist(), 6, a[2].tolist(), a[0].double().numpy(), a[1].double().numpy(), a[5].numpy(),
                                      a[6].numpy(), none(), a[4].tolist())
        assert o["accepted"].tolist() == acc and o["next"].tolist() == nxt and o["length"].tolist() == out
