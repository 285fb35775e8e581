"""Speculative rounds as a server runs them, on the device alone: room for the round's tokens, their keys and values
appended, attention behind a shared prefix, verification, and the pages of what does not stand given back. Against
host lists (pages), attention without sharing, and the definition of verification; eager, and as one
captured graph that is replayed round after round."""
import numpy as np
import pytest
import torch

import round_ref as ref
from resize_ref import State

pytestmark = pytest.mark.gpu
DEV = "cuda"
I32, BF16 = torch.int32, torch.bfloat16
HEADS, KV, DIM, PAGE, VOCAB, DRAFTS = 8, 2, 64, 16, 2000, 4
PREFIX = [96, 0, 160]  # tokens that each group of sequences shares
GROUP = [0, 4, 6, 11]
PER = 40


def ints(v):
    return torch.tensor(v, dtype=I32, device=DEV)


class Server:
    def __init__(self, seed):
        import paper_2604_02945_amd as msao
        self.msao = msao
        self.g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.B = GROUP[-1]
        n_pages = 16 * self.B * 2 + 30
        order = rng.permutation(n_pages).tolist()
        held, table = [], []
        for g, t in enumerate(PREFIX):
            mine = [order.pop() for _ in range(t // PAGE)]
            for _ in range(GROUP[g], GROUP[g + 1]):
                held.append(len(mine))
                table.append(mine + [-1] * (PER - len(mine)))
        self.lengths = [PAGE * h for h in held]
        self.host = State(table, self.lengths, held, order, PAGE)
        self.held_host = held
        self.k = torch.randn(n_pages, KV, PAGE, DIM, generator=self.g).to(BF16).to(DEV)
        self.v = torch.randn(n_pages, KV, PAGE, DIM, generator=self.g).to(BF16).to(DEV)
        self.cache = msao.KvCache(self.k, self.v, ints(table), ints(self.lengths))
        self.pool = msao.PagePool(ints(order + [-1] * (n_pages - len(order))), ints([len(order)]))
        self.held, self.columns = ints(held), ints(held)
        self.prefix = msao.SharedPrefix(ints(GROUP), ints(PREFIX), 5, 160)
        self.rows = self.B * (DRAFTS + 1)
        z = lambda *s, dtype=BF16: torch.zeros(*s, dtype=dtype, device=DEV)  # noqa: E731
        self.want, self.start, self.granted = z(self.B, dtype=I32), z(self.B + 1, dtype=I32), z(self.B, dtype=torch.uint8)
        self.slots, self.positions = z(self.rows, dtype=torch.int64), z(self.rows, dtype=I32)
        self.q, self.q_out, self.out = z(self.rows, HEADS, DIM), z(self.rows, HEADS, DIM), z(self.rows, HEADS, DIM)
        self.new_k, self.new_v = z(self.rows, KV, DIM), z(self.rows, KV, DIM)
        self.lse = z(self.rows, HEADS, dtype=torch.float32)
        self.logits, self.draft = z(self.rows, VOCAB), z(self.rows, VOCAB)
        self.tokens = z(self.rows, dtype=I32)
        self.ua, self.u = z(self.rows, dtype=torch.float32), z(self.rows, dtype=torch.float32)
        self.top_p = torch.full((self.rows,), 0.9, device=DEV)
        self.verdict = {"accepted": z(self.B, dtype=I32), "next": z(self.rows, dtype=I32), "logprob": z(self.rows, dtype=torch.float32),
                        "length": z(self.B, dtype=I32)}
        self.inv_freq = (1e4 ** (-torch.arange(DIM // 2) / (DIM // 2))).float().to(DEV)
        need = lambda n: torch.empty(n + 256, dtype=torch.uint8, device=DEV)  # noqa: E731
        m, st = msao, self.start
        sizes = (m.cache_resize_workspace(self.cache, self.rows),
                 m.cache_attention_shared_workspace(self.cache, self.prefix, st, self.rows, DRAFTS + 1, HEADS),
                 m.verify_workspace(st, DRAFTS + 1, self.rows, VOCAB, BF16))
        self.ws = [w[-w.data_ptr() % 256:][:w.numel() - 256] for w in map(need, sizes)]

    def fill(self):
        """The round's inputs."""
        r = lambda t, s=1.0: t.copy_((torch.randn(t.shape, generator=self.g) * s).to(t.dtype))  # noqa: E731
        for t in (self.q, self.new_k, self.new_v):
            r(t)
        for t in (self.ua, self.u):
            t.copy_(torch.rand(t.shape, generator=self.g))
        x = torch.randn(self.rows, VOCAB, generator=self.g) * 3
        self.logits.copy_(x.to(BF16))
        y = (x + 0.5 * torch.randn(x.shape, generator=self.g)).to(BF16)
        self.draft.copy_(y)
        tokens = [0] + [ref.pick(ref.distribution(y[i].double().numpy(), top_p=np.float32(0.9))[3], float(torch.rand((), generator=self.g)))
                        for i in range(self.rows - 1)]
        self.tokens.copy_(torch.tensor(tokens, dtype=I32))
        self.n_new = [1 + int(torch.randint(0, DRAFTS + 1, (), generator=self.g)) for _ in range(self.B)]
        self.before = list(self.host.length)
        self.want.copy_(torch.tensor([a + b for a, b in zip(self.before, self.n_new)], dtype=I32))

    def round(self):
        m = self.msao
        m.msao_cache_resize(self.cache, self.pool, self.want, held=self.held, columns=self.columns, start=self.start, slots=self.slots,
                            positions=self.positions, granted=self.granted, workspace=self.ws[0])
        m.msao_cache_append(self.cache, self.start, DRAFTS + 1, self.new_k, self.new_v, q=self.q, q_out=self.q_out, inv_freq=self.inv_freq)
        m.msao_cache_attention_shared(self.cache, self.prefix, self.start, DRAFTS + 1, self.q_out, out=self.out, lse=self.lse,
                                      workspace=self.ws[1])
        m.msao_verify(self.start, DRAFTS + 1, self.tokens, self.logits, self.ua, self.u, top_p=self.top_p, draft_logits=self.draft,
                      length=self.cache.length, outputs=self.verdict, workspace=self.ws[2])
        m.msao_cache_resize(self.cache, self.pool, self.verdict["length"], held=self.held, columns=self.columns, workspace=self.ws[0])

    def check(self):
        torch.cuda.synchronize()
        start, placed, granted = self.host.resize([a + b for a, b in zip(self.before, self.n_new)], self.held_host)
        assert granted == [1] * self.B == self.granted.tolist() and self.start.tolist() == start
        n = start[-1]
        assert self.slots[:n].tolist() == [a for a, _ in placed] and self.positions[:n].tolist() == [b for _, b in placed]
        grown = list(self.host.length)
        # the keys lie at their slots, turned by their positions; the values as they were
        at = self.slots[:n]
        assert torch.equal(self.v.transpose(1, 2)[at // PAGE, at % PAGE], self.new_v[:n])
        angle = self.positions[:n].double()[:, None] * self.inv_freq.double()
        a, b = self.new_k[:n].double().chunk(2, -1)
        c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        turned = torch.cat([a * c - b * s, a * s + b * c], -1)
        got = self.k.transpose(1, 2)[at // PAGE, at % PAGE].double()
        assert ((got - turned).abs() <= 2.0 ** -8 * turned.abs() + 1e-5).all()
        # attention over each sequence's own table, without sharing (its pages before anything was given back)
        pages = torch.tensor(self.host.pages)
        q = self.q_out.double().cpu()
        for s_ in range(self.B):
            L, m = grown[s_], self.n_new[s_]
            col = torch.arange(L)
            p, o = pages[s_][col // PAGE].to(DEV), (col % PAGE).to(DEV)
            k, v = self.k.transpose(1, 2)[p, o].double().cpu(), self.v.transpose(1, 2)[p, o].double().cpu()  # [L, KV, DIM]
            for i in range(m):
                r = start[s_] + i
                seen = L - m + i + 1
                for h in range(HEADS):
                    x = k[:seen, h // (HEADS // KV)] @ q[r, h] * DIM ** -0.5
                    z = torch.logsumexp(x, 0)
                    w = torch.exp(x - z)
                    vv = v[:seen, h // (HEADS // KV)]
                    want = w @ vv
                    # scores off by (64 + 2) 2^-24 of 80 at most, exponents and sums by 2^-24 a token; p and the result rounded to bf16
                    assert abs(float(self.lse[r, h]) - float(z)) < 1e-3
                    tol = 2.0 ** -8 * 1.01 * (w @ vv.abs() + want.abs()) + 2e-3 * (w @ vv.abs())
                    assert ((self.out[r, h].double().cpu() - want).abs() <= tol).all()
        acc, nxt, _, kept = ref.verify(start, DRAFTS + 1, self.tokens.tolist(), self.logits.double().cpu().numpy(), self.draft.double().cpu().numpy(),
                                       self.ua.cpu().numpy(), self.u.cpu().numpy(),
                                       {"temperature": None, "top_k": None, "top_p": self.top_p.cpu().numpy(), "min_p": None}, grown)
        assert self.verdict["accepted"].tolist() == acc and self.verdict["length"].tolist() == kept
        assert self.verdict["next"][:n].tolist() == nxt[:n]
        self.host.resize(kept, self.held_host)
        assert self.cache.length.tolist() == self.host.length and self.cache.pages.tolist() == self.host.pages
        assert self.columns.tolist() == self.host.columns
        count = int(self.pool.count)
        assert self.pool.free[:count].tolist() == self.host.free
        return acc


def test_rounds():
    s = Server(1)
    seen = []
    for _ in range(5):
        s.fill()
        s.round()
        seen += s.check()
    assert 0 in seen and max(seen) > 0 and max(s.host.length) > max(s.lengths)


def test_rounds_as_one_graph():
    s = Server(2)
    s.fill()
    s.round()
    s.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.round()
    for _ in range(5):
        s.fill()
        for w in s.ws:
            w.fill_(255)
        graph.replay()
        s.check()


def test_two_servers_on_two_streams():
    a, b = Server(3), Server(4)
    ctx = [a.msao.Context(0), a.msao.Context(0)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for s in (a, b):
            s.fill()
        torch.cuda.synchronize()
        for s, c, st in zip((a, b), ctx, streams):
            m = s.msao
            on = dict(ctx=c, stream=st)
            m.msao_cache_resize(s.cache, s.pool, s.want, held=s.held, columns=s.columns, start=s.start, slots=s.slots, positions=s.positions,
                                granted=s.granted, **on)
            m.msao_cache_append(s.cache, s.start, DRAFTS + 1, s.new_k, s.new_v, q=s.q, q_out=s.q_out, inv_freq=s.inv_freq, **on)
            m.msao_cache_attention_shared(s.cache, s.prefix, s.start, DRAFTS + 1, s.q_out, out=s.out, lse=s.lse, **on)
            m.msao_verify(s.start, DRAFTS + 1, s.tokens, s.logits, s.ua, s.u, top_p=s.top_p, draft_logits=s.draft, length=s.cache.length,
                          outputs=s.verdict, **on)
            m.msao_cache_resize(s.cache, s.pool, s.verdict["length"], held=s.held, columns=s.columns, **on)
        a.check()
        b.check()


def test_kernel_times():
    s = Server(5)
    ctx = s.msao.binding.default_context(0)
    s.fill()
    ctx.set_profiling(True)
    ctx.round_kernel_times()
    s.round()
    t = ctx.round_kernel_times()
    ctx.set_profiling(False)
    b = s.msao.binding
    for k in (b.ROUND_KERNEL_SCAN, b.ROUND_KERNEL_DISTRIBUTE, b.ROUND_KERNEL_VERIFY, b.ROUND_KERNEL_VERIFY_JOIN, b.ROUND_KERNEL_RESIZE,
              b.ROUND_KERNEL_SHARED, b.ROUND_KERNEL_SHARED_JOIN):
        assert t[k] > 0
    assert t[b.ROUND_KERNEL_SAMPLE] == 0 and ctx.round_kernel_times() == [0.0] * b.NUM_ROUND_KERNELS
    s.check()
