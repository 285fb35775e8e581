"""The paged cache's operators as a serving loop runs them: prompts, drafts verified
in one call, tokens taken back, eviction, more tokens; from captured graphs, on
other streams, two at once."""
import numpy as np
import pytest
import torch

from cache_ref import Case, evicted

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


class Toy:
    """One attention layer over embeddings and a head over a small vocabulary, float32."""

    def __init__(self, vocab=40, heads=4, kv_heads=2, dim=64, seed=0):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g).to(DEV)  # noqa: E731
        width = heads * dim
        self.emb = r(vocab, width)
        self.wq, self.wk, self.wv = (r(width, n * dim) * width ** -0.5 for n in (heads, kv_heads, kv_heads))
        self.head = r(width, vocab) * width ** -0.5
        self.inv = (100.0 ** (-torch.arange(dim // 2) / (dim // 2))).float().to(DEV)
        self.ones = torch.ones(dim, device=DEV)
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim

    def project(self, tokens):
        x = self.emb[tokens]
        n = tokens.shape[0]
        return x, (x @ self.wq).view(n, self.heads, self.dim), (x @ self.wk).view(n, self.kv_heads, self.dim), \
            (x @ self.wv).view(n, self.kv_heads, self.dim)

    def greedy(self, x, out):
        """Greedy token of each row, by the framework's own kernel."""
        import paper_2604_02945_amd as msao
        logits = (x + out.reshape(x.shape)) @ self.head
        return msao.msao_draft_entropy(logits.contiguous(), 0.5)["draft_token"].tolist()


def step(toy, cache, tokens, lengths):
    """Append each sequence's tokens (lengths: with them) and attend: greedy tokens of every row."""
    import paper_2604_02945_amd as msao
    new = [len(t) for t in tokens]
    start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=DEV)
    cache.length.copy_(torch.tensor(lengths, dtype=torch.int32))
    flat = torch.tensor([t for ts in tokens for t in ts], device=DEV)
    x, q, k, v = toy.project(flat)
    q = msao.msao_cache_append(cache, start, max(new), k, v, q=q, q_norm=toy.ones, k_norm=toy.ones, inv_freq=toy.inv)
    out = msao.msao_cache_attention(cache, start, max(new), q, accumulate=True)
    got = toy.greedy(x, out)
    return [got[a:a + n] for a, n in zip(np.cumsum([0] + new[:-1]), new)]


def make_cache(toy, seqs, per, page=16, seed=3):
    import paper_2604_02945_amd as msao
    g = torch.Generator().manual_seed(seed)
    n = seqs * per + 2
    k = torch.full((n, toy.kv_heads, page, toy.dim), float("nan"), device=DEV)
    pages = torch.randperm(n, generator=g)[:seqs * per].view(seqs, per).to(torch.int32).to(DEV)
    return msao.KvCache(k, k.clone(), pages, torch.zeros(seqs, dtype=torch.int32, device=DEV),
                        torch.full((seqs, toy.kv_heads, per * page), float("nan"), device=DEV))


def test_verified_drafts_are_the_tokens_of_one_at_a_time():
    """Speculative rounds with drafts right and wrong give the greedy tokens, the weight of the
    tokens that stayed included; rejected drafts are taken back by the length alone."""
    toy = Toy()
    rng = np.random.RandomState(0)
    prompts = [list(rng.randint(0, 40, n)) for n in (5, 33, 1)]
    plain = make_cache(toy, 3, 6)
    seqs = [list(p) for p in prompts]
    last = [r[-1] for r in step(toy, plain, prompts, [len(p) for p in prompts])]
    for _ in range(24):
        seqs = [s + [t] for s, t in zip(seqs, last)]
        last = [r[-1] for r in step(toy, plain, [[t] for t in last], [len(s) for s in seqs])]
    want = [s[len(p):] for s, p in zip(seqs, prompts)]

    spec = make_cache(toy, 3, 6, seed=4)
    done = [list(p) for p in prompts]
    last = [r[-1] for r in step(toy, spec, prompts, [len(p) for p in prompts])]
    while min(len(d) - len(p) for d, p in zip(done, prompts)) < 24:
        drafts = []
        for i, d in enumerate(done):
            # drafts copied from the truth, some spoilt; sequences have 0 .. 5 of them
            ahead = (want[i] + [0] * 40)[len(d) - len(prompts[i]) + 1:][:rng.randint(0, 6)]
            drafts.append([t if rng.rand() < 0.8 else int((t + 1) % 40) for t in ahead])
        tokens = [[t] + d for t, d in zip(last, drafts)]
        got = step(toy, spec, tokens, [len(d) + len(t) for d, t in zip(done, tokens)])
        for i in range(3):
            ok = 0
            while ok < len(drafts[i]) and drafts[i][ok] == got[i][ok]:
                ok += 1
            done[i] += tokens[i][:1 + ok]
            last[i] = got[i][ok]
    for d, p, w in zip(done, prompts, want):
        assert d[len(p):][:24] == w


def test_generation_goes_on_after_eviction():
    """Prompt, steps, eviction in place, more steps: every step against the 64-bit definition over
    the tokens that the definition keeps."""
    import paper_2604_02945_amd as msao
    rng = torch.Generator().manual_seed(5)
    H, K, D, page, B = 4, 2, 64, 16, 2
    n0 = [70, 41]
    cap_pages = 8
    n_pages = B * cap_pages + 1
    pool = torch.full((n_pages, K, page, D), float("nan"), device=DEV)
    pages = torch.randperm(n_pages, generator=rng)[:B * cap_pages].view(B, cap_pages).to(torch.int32).to(DEV)
    cache = msao.KvCache(pool, pool.clone(), pages, torch.zeros(B, dtype=torch.int32, device=DEV),
                         torch.zeros(B, K, cap_pages * page, device=DEV))
    keys = [[torch.zeros(0, D, dtype=torch.float64) for _ in range(K)] for _ in range(B)]
    vals = [[torch.zeros(0, D, dtype=torch.float64) for _ in range(K)] for _ in range(B)]
    wts = [[np.zeros(0) for _ in range(K)] for _ in range(B)]
    lengths = [0, 0]
    budget = torch.tensor([32, 50], dtype=torch.int32, device=DEV)
    for it in range(9):
        new = n0 if it == 0 else [1 + it % 3, 2]
        T = sum(new)
        q, k, v = (torch.randn(T, n, D, generator=rng) for n in (H, K, K))
        start = torch.tensor([0, new[0], T], dtype=torch.int32, device=DEV)
        lengths = [a + b for a, b in zip(lengths, new)]
        cache.length.copy_(torch.tensor(lengths, dtype=torch.int32))
        q2 = msao.msao_cache_append(cache, start, max(new), k.to(DEV), v.to(DEV), q=q.to(DEV))
        out = msao.msao_cache_attention(cache, start, max(new), q2, accumulate=True).double().cpu()
        at = 0
        for b in range(B):
            for h in range(K):
                keys[b][h] = torch.cat([keys[b][h], k[at:at + new[b], h].double()])
                vals[b][h] = torch.cat([vals[b][h], v[at:at + new[b], h].double()])
                wts[b][h] = np.concatenate([wts[b][h], np.zeros(new[b])])
            for i in range(new[b]):
                n = lengths[b] - new[b] + i + 1
                for hq in range(H):
                    h = hq // (H // K)
                    p = torch.softmax(keys[b][h][:n] @ q[at + i, hq].double() * D ** -0.5, 0)
                    assert (out[at + i, hq] - p @ vals[b][h][:n]).abs().max() < 2e-5
                    wts[b][h][:n] += p.numpy()
            at += new[b]
        if it % 3 == 0:
            got = cache.weight.cpu().numpy()
            for b in range(B):
                for h in range(K):
                    assert np.abs(got[b, h, :lengths[b]] - wts[b][h]).max() < 2e-5
                    wts[b][h] = got[b, h, :lengths[b]].astype(np.float64)  # (ranked by what the cache holds)
            r = msao.msao_cache_evict(cache, budget, n_first=2, n_recent=4)
            idx = r["kept_idx"].cpu().numpy()
            for b in range(B):
                for h in range(K):
                    kept = evicted(got[b, h], lengths[b], int(budget[b]), 128, 2, 4)
                    assert np.array_equal(idx[b, h, :len(kept)], kept)
                    keys[b][h], vals[b][h], wts[b][h] = keys[b][h][kept], vals[b][h][kept], wts[b][h][kept]
            lengths = cache.length.tolist()
            assert lengths == [min(n, x) for n, x in zip([len(w[0]) for w in wts], budget.tolist())]


def test_shared_pages_and_a_page_listed_twice():
    """Sequences over the same pages, and one whose table repeats a page."""
    import paper_2604_02945_amd as msao
    case = Case(41, [64, 64], [3, 3], 4, 2, 64, 16, BF16)
    cache, start = case.device(DEV)
    cache.pages[1] = cache.pages[0]
    q = case.q.to(DEV)
    q[3:] = q[:3]
    out = msao.msao_cache_attention(cache, start, 3, q, causal=False, accumulate=True)
    assert torch.equal(out[:3], out[3:])
    w = cache.weight.cpu()
    assert torch.allclose(w[0] - case.weight[0], w[1] - case.weight[1], atol=1e-6)
    cache.pages[0] = cache.pages[0, 0]
    one = torch.tensor([16, 16], dtype=torch.int32, device=DEV)
    many = msao.msao_cache_attention(cache, start, 3, q, causal=False)
    cache.length.copy_(one)
    cache.pages[1] = cache.pages[0]
    few = msao.msao_cache_attention(cache, start, 3, q, causal=False)
    assert torch.allclose(many[:3].float(), few[:3].float(), rtol=2 ** -7, atol=2 ** -7)


def all_outputs(case, dtype, seed, n_first=2, n_recent=5, stream=None, ctx=None):
    """One append, attention and eviction into other pages: everything they write."""
    import paper_2604_02945_amd as msao
    g = torch.Generator().manual_seed(seed)
    cache, start = case.device(DEV)
    T = case.rows
    k, v = (torch.randn(T, case.kv_heads, case.dim, generator=g).to(dtype).to(DEV) for _ in range(2))
    inv = (0.5 ** torch.arange(case.dim // 2)).float().to(DEV)
    to = msao.KvCache(torch.zeros_like(cache.k), torch.zeros_like(cache.v), cache.pages.clone(),
                      torch.zeros_like(cache.length), torch.zeros_like(cache.weight))
    budget = torch.tensor([max(1, n // 2) for n in case.lengths], dtype=torch.int32, device=DEV)
    s = {"cache": cache, "to": to, "start": start, "k": k, "v": v, "q": case.q.to(DEV), "inv": inv, "budget": budget,
         "out": torch.zeros(T, case.heads, case.dim, dtype=dtype, device=DEV), "lse": torch.zeros(T, case.heads, device=DEV),
         "q2": torch.zeros(T, case.heads, case.dim, dtype=dtype, device=DEV),
         "idx": torch.zeros(case.B, case.kv_heads, cache.capacity, dtype=torch.int32, device=DEV),
         "max_new": case.max_new}

    def run():
        msao.msao_cache_append(cache, s["start"], s["max_new"], s["k"], s["v"], q=s["q"], q_out=s["q2"],
                               inv_freq=s["inv"], ctx=ctx, stream=stream)
        msao.msao_cache_attention(cache, s["start"], s["max_new"], s["q2"], out=s["out"], lse=s["lse"], accumulate=True,
                                  ctx=ctx, stream=stream)
        msao.msao_cache_evict(cache, s["budget"], n_first, n_recent, to=to, kept_idx=s["idx"], ctx=ctx, stream=stream)
    s["run"] = run
    return s


def snapshot(s):
    bits = lambda t: t.contiguous().view(torch.uint8).clone()  # noqa: E731
    return [bits(t) for t in (s["q2"], s["out"], s["lse"], s["cache"].k, s["cache"].v, s["cache"].weight, s["to"].k, s["to"].v,
                              s["to"].weight, s["to"].length, s["idx"])]


CASES = [dict(lengths=[300, 17, 0, 2000], new=[5, 1, 0, 6], heads=14, kv_heads=2, dim=128, page=16, dtype=BF16),
         dict(lengths=[400, 170], new=[200, 90], heads=4, kv_heads=2, dim=64, page=32, dtype=BF16),
         dict(lengths=[130, 90], new=[50, 1], heads=4, kv_heads=4, dim=96, page=16, dtype=F32)]


@pytest.mark.parametrize("case", CASES, ids=["round", "prompts", "f32"])
def test_the_same_call_gives_the_same_bits(case):
    a, b = (all_outputs(Case(51, **case), case["dtype"], 1) for _ in range(2))
    for s in (a, b):
        s["run"]()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(snapshot(a), snapshot(b)))


@pytest.mark.parametrize("case", CASES, ids=["round", "prompts", "f32"])
def test_replays_of_a_graph_follow_the_arrays(case):
    """Captured once; replayed with other lengths, starts, pages, inputs and eager work between."""
    graph_s, eager = (all_outputs(Case(52, **case), case["dtype"], 2) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph_s["run"]()
    torch.cuda.current_stream().wait_stream(side)
    eager["run"]()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graph_s["run"]()
    g = torch.Generator().manual_seed(9)
    c = Case(52, **case)
    for it in range(4):
        q = torch.randn(c.q.shape, generator=g).to(c.dtype).to(DEV)
        used = -(-c.lengths[0] // c.page)
        pages = torch.from_numpy(c.pages[0, :used])[torch.randperm(used, generator=g)].to(DEV)
        lengths = torch.tensor([int(n * f) for n, f in zip(c.lengths, torch.rand(c.B, generator=g) * 0.5 + 0.5)], dtype=torch.int32)
        for s in (graph_s, eager):
            s["q"].copy_(q)
            s["cache"].length.copy_(lengths)
            if it > 1:
                s["cache"].pages[0, :used].copy_(pages)
        x = torch.randn(1000, 1000, device=DEV)
        graph.replay()
        y = (x @ x).sum()
        eager["run"]()
        torch.cuda.synchronize()
        assert torch.isfinite(y)
        assert all(torch.equal(a, b) for a, b in zip(snapshot(graph_s), snapshot(eager))), it


def test_two_graphs_share_a_workspace():
    """Replayed in turn on one stream: each call writes what it reads of its workspace."""
    import paper_2604_02945_amd as msao
    cases = [Case(53, [900, 300], [2, 4], 8, 2, 128, 16, BF16), Case(54, [700], [90], 4, 1, 64, 32, BF16)]
    made, need = [], 0
    for c in cases:
        cache, start = c.device(DEV)
        need = max(need, msao.cache_attention_workspace(cache, start, c.rows, c.max_new, c.heads, accumulate=True))
        made.append((c, cache, start, c.q.to(DEV), torch.zeros(c.rows, c.heads, c.dim, dtype=BF16, device=DEV)))
    ws = torch.empty(need + 256, dtype=torch.uint8, device=DEV)
    ws = ws[(-ws.data_ptr()) % 256:][:need]
    want, graphs = [], []
    for c, cache, start, q, out in made:
        msao.msao_cache_attention(cache, start, c.max_new, q, out=out, accumulate=True, workspace=ws)
        want.append(out.clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            msao.msao_cache_attention(cache, start, c.max_new, q, out=out, accumulate=True, workspace=ws)
        graphs.append(graph)
    for _ in range(3):
        for (c, cache, start, q, out), graph, w in zip(made, graphs, want):
            out.zero_()
            ws.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, w)


def test_two_streams_at_once():
    """Calls on two streams with a context each, and memory that the calls allocate for themselves."""
    import paper_2604_02945_amd as msao
    cases = [CASES[0], CASES[1]]
    want = [all_outputs(Case(55, **c), c["dtype"], 3) for c in cases]
    for s in want:
        s["run"]()
    torch.cuda.synchronize()
    streams, ctxs = [torch.cuda.Stream() for _ in cases], [msao.Context(0) for _ in cases]
    got = [all_outputs(Case(55, **c), c["dtype"], 3, stream=st, ctx=x) for c, st, x in zip(cases, streams, ctxs)]
    torch.cuda.synchronize()
    for s in got:
        s["run"]()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(snapshot(a), snapshot(b)))
    # outputs allocated by the call belong to its stream
    s, st = got[0], streams[0]
    out = msao.msao_cache_attention(s["cache"], s["start"], s["max_new"], s["q2"], stream=st, ctx=ctxs[0])
    st.synchronize()
    assert torch.equal(out, s["out"])


def test_nothing_to_do():
    import paper_2604_02945_amd as msao
    k = torch.zeros(2, 2, 16, 64, device=DEV)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)  # noqa: E731
    none = msao.KvCache(k, k.clone(), i32(0, 3), i32(0), torch.zeros(0, 2, 48, device=DEV))
    q = torch.zeros(0, 4, 64, device=DEV)
    msao.msao_cache_append(none, i32(1), 0, q[:, :2], q[:, :2], q=q)
    msao.msao_cache_attention(none, i32(1), 0, q, accumulate=True)
    msao.msao_cache_evict(none, i32(0))
    empty = msao.KvCache(k, k.clone(), i32(3, 0), i32(3) + 5, torch.zeros(3, 2, 0, device=DEV))  # no capacity
    start = torch.tensor([0, 1, 1, 3], dtype=torch.int32, device=DEV)
    q = torch.ones(3, 4, 64, device=DEV)
    lse = torch.zeros(3, 4, device=DEV)
    msao.msao_cache_append(empty, start, 2, q[:, :2], q[:, :2], q=q.clone())
    out = msao.msao_cache_attention(empty, start, 2, q, lse=lse, accumulate=True)
    r = msao.msao_cache_evict(empty, i32(3) + 2)
    torch.cuda.synchronize()
    assert (out == 0).all() and (lse == -np.inf).all() and r["kept_count"].tolist() == [0, 0, 0]
    assert (k == 0).all()


@pytest.mark.parametrize("start", [[5, 2, 9], [-4, 3, 3], [0, 100, 4], [3, 3, -1], [7, 8, 1000]])
def test_starts_out_of_order_stay_in_bounds(start):
    """Entries are taken into [0, rows]; a sequence that ends before its start has no rows."""
    import paper_2604_02945_amd as msao
    case = Case(56, [40, 33], [4, 5], 4, 2, 64, 16, BF16)
    cache, _ = case.device(DEV)
    st = torch.tensor(start, dtype=torch.int32, device=DEV)
    b = np.clip(start, 0, case.rows)
    q = case.q.to(DEV)
    out = torch.full_like(q, 7.0)
    q2 = torch.full_like(q, 7.0)
    kv = torch.randn(case.rows, 2, 64, device=DEV).to(BF16)
    msao.msao_cache_append(cache, st, case.rows, kv, kv, q=q, q_out=q2)
    msao.msao_cache_attention(cache, st, case.rows, q, out=out, accumulate=True)
    torch.cuda.synchronize()
    mine = np.zeros(case.rows, bool)
    for s in range(2):
        mine[b[s]:max(b[s], b[s + 1])] = True
    assert (out[~torch.from_numpy(mine).to(DEV)] == 7).all()
    assert ((out != 7).any(-1).any(-1).cpu().numpy() == mine).all()


def test_lengths_past_the_capacity_count_as_it():
    import paper_2604_02945_amd as msao
    case = Case(57, [48, 48], [2, 2], 4, 2, 64, 16, BF16)
    cache, start = case.device(DEV)
    q = case.q.to(DEV)
    want = msao.msao_cache_attention(cache, start, 2, q)
    cache.length.copy_(torch.tensor([2 ** 31 - 1, 49], dtype=torch.int32))
    assert torch.equal(msao.msao_cache_attention(cache, start, 2, q), want)
    cache.length.copy_(torch.tensor([-5, -2 ** 31], dtype=torch.int32))
    assert (msao.msao_cache_attention(cache, start, 2, q) == 0).all()


def test_pages_past_4_gib():
    """A pool whose pages lie further apart than 32 bits of bytes reach."""
    import paper_2604_02945_amd as msao
    far = (5 << 30) // 2  # elements
    if torch.cuda.mem_get_info()[0] < 14 << 30:
        pytest.skip("needs 14 GiB of free device memory")
    pool = torch.empty(far + (1 << 20), dtype=BF16, device=DEV)
    shape, stride = (2, 2, 16, 64), (far, 16 * 64, 64, 1)
    k, v = (torch.as_strided(pool, shape, stride, o) for o in (0, 1 << 16))
    small = Case(58, [30, 16], [3, 2], 4, 2, 64, 16, BF16, spare_pages=0)
    near, start = small.device(DEV)
    pages = torch.tensor([[1, 0], [1, -1]], dtype=torch.int32, device=DEV)
    near_k, near_v = (torch.zeros(2, 2, 16, 64, dtype=BF16, device=DEV) for _ in range(2))
    w = [torch.zeros(2, 2, 32, device=DEV) for _ in range(2)]
    caches = [msao.KvCache(a, b, pages, torch.tensor([30, 16], dtype=torch.int32, device=DEV), x)
              for a, b, x in ((k, v, w[0]), (near_k, near_v, w[1]))]
    whole = torch.tensor([0, 30, 30], dtype=torch.int32, device=DEV)
    kv = torch.randn(30, 2, 64, device=DEV).to(BF16)
    got = []
    for c in caches:
        msao.msao_cache_append(c, whole, 30, kv, kv.flip(0))
        got.append(msao.msao_cache_attention(c, start, 3, small.q.to(DEV), accumulate=True))
        msao.msao_cache_evict(c, torch.tensor([20, 16], dtype=torch.int32, device=DEV), 1, 2)
    torch.cuda.synchronize()
    assert torch.equal(got[0], got[1]) and torch.equal(w[0], w[1])
    assert torch.equal(k, near_k) and torch.equal(v, near_v)


def test_kernel_times():
    import paper_2604_02945_amd as msao
    ctx = msao.Context(0)
    s = all_outputs(Case(59, **CASES[1]), BF16, 4, ctx=ctx)
    ctx.set_profiling(True)
    s["run"]()
    ms = ctx.cache_kernel_times()
    B = msao.binding
    assert all(ms[i] > 0 for i in (B.CACHE_KERNEL_APPEND, B.CACHE_KERNEL_ATTEND, B.CACHE_KERNEL_WEIGHT, B.CACHE_KERNEL_SELECT,
                                   B.CACHE_KERNEL_MOVE))
    assert ctx.cache_kernel_times() == [0.0] * B.NUM_CACHE_KERNELS and sum(ctx.kernel_times()) == 0
    ctx.close()
