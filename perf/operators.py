"""Timed calls of the paged cache's operators: append (norms of queries and keys
per head and the position rotation, into the pages), attention of a chunk of new
tokens over the pages, and eviction by accumulated attention weight. The plain
forms are elementary torch operations in 32 bits (64 for the angles)."""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6
BASE = 1e6  # of the rotation's frequencies


def _case(op, name=None, **kw):
    case = {"op": op, "dtype": "bf16", "seqs": 1, "heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64,
            "len_lo": 1, "len_hi": 1}
    if op != "evict":
        case.update({"new_lo": 1, "new_hi": 1})
    if op == "append":
        case.update({"rot": 128, "axes": 1, "interleaved": False, "norm": True})
    elif op == "attend":
        case.update({"causal": True, "weight": False})
    else:
        case.update({"budget": 1024, "first": 4, "recent": 64})
    assert set(kw) <= set(case)
    case.update(kw)
    return dict(case, name=name) if name else case


def listed():
    return [
        # one generated token of one request: the smallest call, bound by latency
        _case("append", "append_step", len_lo=1500, len_hi=1500),
        # a speculative round: 256 requests, each with its accepted token and up to five drafts
        _case("append", "append_round", seqs=256, len_lo=40, len_hi=500, new_lo=2, new_hi=6),
        # prompts of images and text, positions in time, row and column
        _case("append", "append_prompts", seqs=12, len_lo=300, len_hi=4000, new_lo=300, new_hi=4000, axes=3),
        # float32 prompts behind cached ones, part of each head rotated, neighbouring pairs
        _case("append", "append_prompts_f32", dtype="f32", seqs=3, heads=12, kv_heads=4, head_dim=96, page=16, rot=64,
              interleaved=True, len_lo=900, len_hi=2500, new_lo=700, new_hi=1300),
        # one generated token of one request
        _case("attend", "attend_step", len_lo=2000, len_hi=2000),
        # verification of a speculative round of ragged requests, with the weight that eviction goes by
        _case("attend", "attend_round", seqs=64, heads=28, kv_heads=4, len_lo=200, len_hi=16000, new_lo=2, new_hi=6,
              weight=True),
        # generation steps of two long documents
        _case("attend", "attend_long", seqs=2, page=256, len_lo=120000, len_hi=131072),
        # chunks of two long prompts
        _case("attend", "attend_chunk", seqs=2, len_lo=9000, len_hi=12288, new_lo=2000, new_hi=2048),
        # short prompts as they arrive, with the weight, narrow heads
        _case("attend", "attend_prompts", seqs=8, heads=16, kv_heads=2, head_dim=64, page=16, len_lo=77, len_hi=1500,
              new_lo=77, new_hi=1500, weight=True),
        # text tokens over an encoder's states, float32, all of them visible
        _case("attend", "attend_encoder_f32", dtype="f32", seqs=4, heads=12, kv_heads=12, head_dim=96, page=32,
              len_lo=577, len_hi=1500, new_lo=20, new_hi=200, causal=False),
        # one request over its budget
        _case("evict", "evict_request", len_lo=2900, len_hi=2900, budget=1450),
        # a batch of requests cut back together
        _case("evict", "evict_batch", seqs=32, len_lo=3000, len_hi=8000, budget=2048, first=8, recent=256),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(["append", "attend", "attend", "attend", "evict"])
        kv = rng.choice([1, 2, 4, 8])
        c = {"dtype": rng.choice(["bf16", "bf16", "f32"]), "seqs": _log(rng, 1, 256), "kv_heads": kv,
             "heads": kv * rng.choice([1, 2, 4, 5, 7, 8]), "head_dim": rng.choice([64, 64, 80, 96, 128, 128, 128, 256]),
             "page": rng.choice([16, 32, 64, 128, 256])}
        c["len_hi"] = _log(rng, 64, 131072)
        c["len_lo"] = _log(rng, 1, c["len_hi"])
        if op != "evict":
            c["new_hi"] = min(c["len_hi"], rng.choice([1, _log(rng, 1, 8), _log(rng, 8, 4096)]))
            c["new_lo"] = _log(rng, 1, min(c["new_hi"], c["len_lo"]))
        if op == "append":
            c["len_hi"] = max(c["new_hi"], min(c["len_hi"], 4096))  # (the whole pool is compared)
            c["len_lo"] = min(c["len_lo"], c["len_hi"])
            c["rot"] = rng.choice([c["head_dim"], c["head_dim"] // 2 // 16 * 16])
            c["axes"] = rng.choice([1, 3])
            c["interleaved"], c["norm"] = rng.random() < 0.3, rng.random() < 0.7
        elif op == "attend":
            c["causal"], c["weight"] = rng.random() < 0.8, rng.random() < 0.4
        else:
            c["budget"] = _log(rng, 16, c["len_hi"])
            c["first"], c["recent"] = rng.choice([0, 1, 4]), min(c["budget"] // 2, rng.choice([0, 16, 128]))
        case = _case(op, **c)
        w = work(case)
        cells = case["seqs"] * case["len_hi"] * case["kv_heads"] * case["head_dim"]
        scores = case["seqs"] * case["len_hi"] * case["heads"] * case.get("new_hi", 1)
        fp32 = case["dtype"] == "f32"
        if w["bytes"] > 1.0e9 or w["flops"] > (4e10 if fp32 else 2e11) or cells > 1.2e9 or scores > 6e8:
            continue
        return case


# ---- sizes that a case stands for --------------------------------------------

def _spread(n, lo, hi, by=0.6180339887):
    """n whole numbers from lo to hi, hi first, most of them nearer to lo."""
    return [hi if i == 0 else lo + int((hi - lo) * ((i * by) % 1.0) ** 2) for i in range(n)]


def _lengths(case):
    """Cached tokens of each sequence, the new ones among them, and the new ones."""
    length = _spread(case["seqs"], case["len_lo"], case["len_hi"])
    if case["op"] == "evict":
        return length, [0] * len(length)
    new = _spread(case["seqs"], case["new_lo"], case["new_hi"], 0.7548776662)
    return [max(a, b) for a, b in zip(length, new)], new


def _size(case):
    return 4 if case["dtype"] == "f32" else 2


def work(case):
    length, new = _lengths(case)
    es, H, K, D = _size(case), case["heads"], case["kv_heads"], case["head_dim"]
    T, L = sum(new), sum(length)
    if case["op"] == "append":
        return {"bytes": 2 * T * (H + 2 * K) * D * es, "flops": 8 * T * (H + K) * D}
    if case["op"] == "evict":
        kept = sum(min(n, case["budget"]) for n in length)
        return {"bytes": 4 * K * L + kept * K * (2 * 2 * D * es + 4 + 4), "flops": K * L}
    seen = sum(m * n - (m * (m - 1) // 2 if case["causal"] else 0) for n, m in zip(length, new))
    more = 1 if case["weight"] else 0
    return {"bytes": 2 * L * K * D * es + 2 * T * H * D * es + 4 * T * H + more * 8 * K * L,
            "flops": (4 + 2 * more) * seen * H * D}


# ---- what a serving program has in hand ----------------------------------------

def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    length, new = _lengths(case)
    dt, B, H, K, D = DTYPES[case["dtype"]], case["seqs"], case["heads"], case["kv_heads"], case["head_dim"]
    page = case["page"]
    per = -(-max(length) // page)
    used = [-(-n // page) for n in length]
    n_pages = sum(used) + 3

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dt)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32).to(DEV)

    # a sequence's pages lie anywhere in the pool; entries past its own name none
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    first = torch.tensor([sum(used[:i]) for i in range(B)])[:, None] + torch.arange(per)[None, :]
    mine = torch.arange(per)[None, :] < torch.tensor(used)[:, None]
    first, mine = first.to(DEV), mine.to(DEV)
    pages = torch.where(mine, order[first.clamp(max=n_pages - 1)], torch.full_like(first, -1, dtype=torch.int32))
    s = {"case": case, "pages": pages.contiguous(), "length": ints(length), "handle": None,
         "k": normal(n_pages, K, page, D), "v": normal(n_pages, K, page, D), "weight": None}
    cap = per * page
    if case["op"] == "evict":
        # weight gathered over many steps: a few tokens hold most of it, some none
        w = torch.exp(2.0 * torch.randn(B, K, cap, generator=g, device=DEV))
        w = w * (torch.rand(B, K, cap, generator=g, device=DEV) > 0.05)
        s["weight"] = w * (torch.arange(cap, device=DEV) < s["length"][:, None, None])
        keep = min(case["budget"], max(length))
        to = -(-keep // page)
        s["to_pages"] = torch.randperm(B * to, generator=g, device=DEV).to(torch.int32).view(B, to)
        s["to_k"] = torch.zeros(B * to, K, page, D, dtype=dt, device=DEV)
        s["to_v"] = torch.zeros_like(s["to_k"])
        s["to_weight"] = torch.zeros(B, K, to * page, device=DEV)
        s["to_length"] = torch.zeros(B, dtype=torch.int32, device=DEV)
        s["budget"] = torch.full((B,), case["budget"], dtype=torch.int32, device=DEV)
        s["to_handle"] = None
        return s
    T = sum(new)
    s["start"] = ints([sum(new[:i]) for i in range(B + 1)])
    s["max_new"] = max(new)
    # projections of the heads: queries and keys with a common part, as trained heads have
    s["q"] = normal(T, H, D, scale=1.5)
    s["out"] = torch.zeros(T, H, D, dtype=dt, device=DEV)
    if case["op"] == "append":
        s["new_k"], s["new_v"] = normal(T, K, D, scale=3.0), normal(T, K, D)
        s["q_norm"] = (1 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(dt) if case["norm"] else None
        s["k_norm"] = (1 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(dt) if case["norm"] else None
        half = case["rot"] // 2
        s["inv_freq"] = (BASE ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))).float().to(DEV)
        far = torch.randint(0, 100000, (case["axes"], B), generator=g, device=DEV)
        seq = torch.repeat_interleave(torch.arange(B), torch.tensor(new)).to(DEV)
        at = torch.arange(T, device=DEV) - s["start"][seq.long()]
        step = torch.stack([at, at // 24, at % 24])[:case["axes"]]
        s["positions"] = (far[:, seq] + step).to(torch.int32).contiguous()
        s["sections"] = [half] if case["axes"] == 1 else [half // 4, half // 4, half - 2 * (half // 4)]
    else:
        if case["weight"]:
            w = torch.rand(B, K, cap, generator=g, device=DEV) * 4
            s["weight"] = w * (torch.arange(cap, device=DEV) < s["length"][:, None, None])
        s["lse"] = torch.zeros(T, H, device=DEV)
    return s


# ---- the plain forms -------------------------------------------------------------

def _slots(s, pos):
    """Page and slot of positions [B, n] of each sequence (page -1: none)."""
    page = s["k"].shape[2]
    col = torch.div(pos, page, rounding_mode="floor").clamp(0, s["pages"].shape[1] - 1)
    return torch.gather(s["pages"].long(), 1, col), pos % page


def _new_tokens(s):
    """[B, max_new]: row of each new token, which of them exist, and their positions in the cache."""
    a = torch.arange(s["max_new"], device=DEV)[None, :]
    start = s["start"].long()
    n = (start[1:] - start[:-1])[:, None]
    return start[:-1, None] + a, a < n, s["length"].long()[:, None] - n + a


def _normed(x, w):
    x = x.float()
    if w is None:
        return x
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()


def _rotated(x, cos, sin, rot, interleaved):
    """x [T, heads, D] in 32 bits with its first `rot` values turned by pairs."""
    y = x[..., :rot]
    cos, sin = cos[:, None, :], sin[:, None, :]
    if interleaved:
        a, b = y[..., 0::2], y[..., 1::2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_append(s):
    c = s["case"]
    axis = torch.repeat_interleave(torch.arange(len(s["sections"])), torch.tensor(s["sections"])).to(DEV)
    angle = s["positions"][axis].double().t() * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    s["out"].copy_(_rotated(_normed(s["q"], s["q_norm"]), cos, sin, c["rot"], c["interleaved"]))
    k = _rotated(_normed(s["new_k"], s["k_norm"]), cos, sin, c["rot"], c["interleaved"]).to(s["k"].dtype)
    row, there, pos = _new_tokens(s)
    page, slot = _slots(s, pos.clamp(min=0))
    T = k.shape[0]
    seq = torch.searchsorted(s["start"].long(), torch.arange(T, device=DEV), right=True) - 1
    at = torch.arange(T, device=DEV) - s["start"].long()[seq]
    s["k"][page[seq, at], :, slot[seq, at]] = k
    s["v"][page[seq, at], :, slot[seq, at]] = s["new_v"]
    return [s["out"], s["k"], s["v"]]


def _gathered(s, x, pages):
    """[B, kv heads, capacity, D] in 32 bits of the pages of each sequence."""
    y = x[pages.clamp(min=0).long()]  # [B, pages, kv heads, page, D]
    y = y.permute(0, 2, 1, 3, 4).flatten(2, 3).float()
    there = torch.arange(y.shape[2], device=DEV)[None, :] < s["length"][:, None]
    return torch.where(there[:, None, :, None], y, torch.zeros((), device=DEV))


def _plain_attend(s):
    c = s["case"]
    B, K, D = c["seqs"], c["kv_heads"], c["head_dim"]
    G, N, T = c["heads"] // K, s["max_new"], s["q"].shape[0]
    row, there, pos = _new_tokens(s)
    k, v = _gathered(s, s["k"], s["pages"]), _gathered(s, s["v"], s["pages"])
    cap = k.shape[2]
    q = s["q"][row.clamp(max=T - 1)].float().view(B, N, K, G, D).permute(0, 2, 1, 3, 4).reshape(B, K, N * G, D)
    score = torch.matmul(q, k.transpose(2, 3)).view(B, K, N, G, cap) * D ** -0.5
    j = torch.arange(cap, device=DEV)
    last = pos if c["causal"] else (s["length"].long() - 1)[:, None].expand(B, N)
    seen = (j <= last[..., None]) & there[..., None]  # [B, N, cap]
    score = torch.where(seen[:, None, :, None, :], score, torch.full((), -math.inf, device=DEV))
    most = score.amax(-1, keepdim=True)
    most = torch.where(most == -math.inf, torch.zeros_like(most), most)
    p = torch.exp(score - most)
    total = p.sum(-1, keepdim=True)
    lse = (most + torch.log(total)).squeeze(-1)  # [B, K, N, G]
    p = torch.where(total > 0, p / total, torch.zeros_like(p))
    o = torch.matmul(p.view(B, K, N * G, cap), v).view(B, K, N, G, D)
    # rows of no token land behind the last one
    to = torch.where(there, row, torch.full_like(row, T)).flatten()
    out = torch.zeros(T + 1, c["heads"], D, device=DEV)
    out[to] = o.permute(0, 2, 1, 3, 4).reshape(B * N, c["heads"], D)
    s["out"].copy_(out[:T])
    of = torch.zeros(T + 1, c["heads"], device=DEV)
    of[to] = lse.permute(0, 2, 1, 3).reshape(B * N, c["heads"])
    s["lse"].copy_(of[:T])
    if not c["weight"]:
        return [s["out"], s["lse"]]
    s["weight"] += p.sum((2, 3))
    return [s["out"], s["lse"], s["weight"]]


def _plain_evict(s):
    c = s["case"]
    B, K, page, cap = c["seqs"], c["kv_heads"], c["page"], s["weight"].shape[2]
    j = torch.arange(cap, device=DEV)
    L = s["length"].long()[:, None]
    kept = torch.minimum(L, s["budget"].long()[:, None])  # [B, 1]
    always = (j < c["first"]) | ((j >= L - c["recent"]) & (j < L))
    w = s["weight"]
    key = torch.where(w > 0, w, torch.zeros_like(w))
    key = torch.where(always[:, None], torch.full_like(key, math.inf), key)
    key = torch.where((j < L)[:, None], key, torch.full_like(key, -1.0))
    rank = torch.sort(key, dim=-1, descending=True, stable=True).indices  # equal weights: the lower index first
    width = s["to_weight"].shape[2]
    n = torch.arange(width, device=DEV)
    there = (n < kept)[:, None, :].expand(B, K, width)
    width_rank = torch.nn.functional.pad(rank, (0, max(0, width - cap)))[..., :width]
    idx = torch.where(there, width_rank, torch.full_like(width_rank, cap))
    idx = torch.sort(idx, dim=-1).values  # ascending, the absent ones last
    safe = idx.clamp(max=cap - 1)
    src_page = torch.gather(s["pages"].long()[:, None].expand(B, K, -1), 2, safe // page)
    head = torch.arange(K, device=DEV)[None, :, None]
    to_page = s["to_pages"].long()[:, None, n // page]  # [B, 1, width]
    for x, y in ((s["k"], s["to_k"]), (s["v"], s["to_v"])):
        old = y[to_page, head, n % page]
        new = x[src_page, head, safe % page]
        y[to_page.expand(B, K, width), head.expand(B, K, width), (n % page).expand(B, K, width)] = torch.where(
            there[..., None], new, old)
    s["to_weight"].copy_(torch.where(there, torch.gather(w, 2, safe), s["to_weight"]))
    s["to_length"].copy_(kept[:, 0].to(torch.int32))
    kept_idx = torch.full((B, K, cap), -1, dtype=torch.int32, device=DEV)
    part = min(width, cap)
    kept_idx[..., :part] = torch.where(there, idx, torch.full_like(idx, -1))[..., :part].to(torch.int32)
    return [s["to_k"], s["to_v"], s["to_weight"], s["to_length"], kept_idx]


# ---- one pass --------------------------------------------------------------------

def run(s):
    c = s["case"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "evict": _plain_evict}[c["op"]](s)
    import paper_2604_02945_amd as msao
    if s["handle"] is None:
        s["handle"] = msao.KvCache(s["k"], s["v"], s["pages"], s["length"], s["weight"])
        if c["op"] == "evict":
            s["to_handle"] = msao.KvCache(s["to_k"], s["to_v"], s["to_pages"], s["to_length"], s["to_weight"])
    if c["op"] == "append":
        msao.msao_cache_append(s["handle"], s["start"], s["max_new"], s["new_k"], s["new_v"], q=s["q"], q_out=s["out"],
                               q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS, positions=s["positions"],
                               inv_freq=s["inv_freq"], sections=s["sections"], interleaved=c["interleaved"])
        return [s["out"], s["k"], s["v"]]
    if c["op"] == "attend":
        msao.msao_cache_attention(s["handle"], s["start"], s["max_new"], s["q"], causal=c["causal"], out=s["out"],
                                  lse=s["lse"], accumulate=c["weight"])
        return [s["out"], s["lse"]] + ([s["weight"]] if c["weight"] else [])
    sel = msao.msao_cache_evict(s["handle"], s["budget"], n_first=c["first"], n_recent=c["recent"], to=s["to_handle"])
    return [s["to_k"], s["to_v"], s["to_weight"], s["to_length"], sel["kept_idx"]]


# ---- the definitions in 64 bits, sequence by sequence -------------------------------

def _rows(x, pages, n):
    """Rows 0 .. n-1 of one sequence: [kv heads, n, D]."""
    page = x.shape[2]
    y = x[pages[:-(-n // page)].long()].transpose(0, 1)
    return y.reshape(x.shape[1], -1, x.shape[3])[:, :n]


def _exact_append(s, length, new):
    c = s["case"]
    half, D = c["rot"] // 2, c["head_dim"]
    bounds = [sum(s["sections"][:i + 1]) for i in range(len(s["sections"]))]
    axis = [sum(i >= b for b in bounds) for i in range(half)]
    angle = torch.stack([s["positions"][a].double() for a in axis], 1) * s["inv_freq"].double() if half else None

    def turned(x, w):
        x = x.double()
        if w is not None:
            x = x / ((x * x).sum(-1, keepdim=True) / D + EPS).sqrt() * w.double()
        if half:
            i = torch.arange(half, device=DEV)
            lo, hi = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
            z = torch.complex(x[..., lo], x[..., hi]) * torch.polar(torch.ones_like(angle), angle)[:, None, :]
            x = x.clone()
            x[..., lo], x[..., hi] = z.real, z.imag
        return x

    q, k = turned(s["q"], s["q_norm"]), turned(s["new_k"], s["k_norm"])
    K, V = s["k"].double(), s["v"].double()
    at = 0
    for b, (n, m) in enumerate(zip(length, new)):
        pos = torch.arange(n - m, n, device=DEV)
        page = s["pages"][b].long()[pos // c["page"]]
        K[page, :, pos % c["page"]] = k[at:at + m]
        V[page, :, pos % c["page"]] = s["new_v"][at:at + m].double()
        at += m
    return [q, K, V]


def _exact_attend(s, length, new):
    c = s["case"]
    G = c["heads"] // c["kv_heads"]
    outs, lses, at = [], [], 0
    weight = s["weight"].double() if c["weight"] else None
    for b, (n, m) in enumerate(zip(length, new)):
        k, v = _rows(s["k"], s["pages"][b], n).double(), _rows(s["v"], s["pages"][b], n).double()
        out, lse = [], []
        for h in range(c["heads"]):
            q = s["q"][at:at + m, h].double() / math.sqrt(c["head_dim"])
            x = q @ k[h // G].t().contiguous()
            if c["causal"]:
                x = x + torch.full_like(x, -math.inf).triu(n - m + 1)
            z = torch.logsumexp(x, -1)
            p = torch.exp(x - z[:, None])
            out.append(p @ v[h // G])
            lse.append(z)
            if weight is not None:
                weight[b, h // G, :n] += p.sum(0)
        outs.append(torch.stack(out, 1))
        lses.append(torch.stack(lse, 1))
        at += m
    return [torch.cat(outs), torch.cat(lses)] + ([weight] if weight is not None else [])


def _exact_evict(s, length):
    c = s["case"]
    K, V, W = s["to_k"].double(), s["to_v"].double(), s["to_weight"].double()
    for b, n in enumerate(length):
        kept = min(n, c["budget"])
        a = min(n, c["first"])
        z = max(a, n - c["recent"])
        w = s["weight"][b, :, a:z].double()
        w = torch.where(w > 0, w, torch.zeros_like(w))
        take = kept - a - (n - z)
        best = torch.sort(-w, dim=-1, stable=True).indices[:, :take] + a
        ends = torch.cat([torch.arange(a, device=DEV), torch.arange(z, n, device=DEV)]).expand(c["kv_heads"], -1)
        idx = torch.sort(torch.cat([best, ends], 1), dim=1).values  # [kv heads, kept]
        k, v = _rows(s["k"], s["pages"][b], n).double(), _rows(s["v"], s["pages"][b], n).double()
        pos = torch.arange(kept, device=DEV)
        page = s["to_pages"][b].long()[pos // c["page"]]
        for h in range(c["kv_heads"]):
            K[page, h, pos % c["page"]] = k[h, idx[h]]
            V[page, h, pos % c["page"]] = v[h, idx[h]]
            W[b, h, :kept] = s["weight"][b, h, idx[h]].double()
    return [K, V, W, None, None]


def exact(case, seed):
    s = prepare(case, seed)
    length, new = _lengths(case)
    if case["op"] == "append":
        return _exact_append(s, length, new)
    if case["op"] == "attend":
        return _exact_attend(s, length, new)
    return _exact_evict(s, length)
