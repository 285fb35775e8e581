"""Plain 64-bit forms of the paged cache's operators on host arrays, token by
token from their definitions, and cases for them."""
import numpy as np
import torch


class Case:
    """A cache of ragged sequences with a chunk of new tokens, as host float64
    arrays of exactly the values that the device tensors hold. Memory that no token
    owns (the rest of a sequence's last page, pages of none) holds NaN."""

    def __init__(self, seed, lengths, new, heads, kv_heads, dim, page, dtype, extra_rows=0, spare_pages=3, device="cpu",
                 order="head", bad_page=None, scale_q=1.5):
        g = torch.Generator().manual_seed(seed)
        self.lengths, self.new, self.heads, self.kv_heads, self.dim, self.page = lengths, new, heads, kv_heads, dim, page
        self.dtype, self.B, self.order = dtype, len(lengths), order
        self.per = max(1, max(-(-n // page) for n in lengths) if lengths else 1)
        self.cap = self.per * page
        used = [-(-n // page) for n in lengths]
        n_pages = sum(used) + spare_pages
        perm = torch.randperm(n_pages, generator=g).tolist()
        self.pages = np.full((self.B, self.per), -7, np.int32)
        at = 0
        for b, u in enumerate(used):
            self.pages[b, :u] = perm[at:at + u]
            at += u
        if bad_page is not None:  # (sequence, column, what it names)
            self.pages[bad_page[0], bad_page[1]] = bad_page[2]
        self.n_pages = n_pages
        self.k = torch.full((n_pages, kv_heads, page, dim), float("nan"), dtype=dtype)
        self.v = self.k.clone()
        for b, n in enumerate(lengths):
            for j in range(0, n, page):
                p = self.pages[b, j // page]
                if 0 <= p < n_pages:
                    m = min(page, n - j)
                    self.k[p, :, :m] = torch.randn(kv_heads, m, dim, generator=g).to(dtype)
                    self.v[p, :, :m] = torch.randn(kv_heads, m, dim, generator=g).to(dtype)
        self.start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.rows = int(self.start[-1]) + extra_rows
        self.q = (torch.randn(self.rows, heads, dim, generator=g) * scale_q).to(dtype)
        self.weight = torch.rand(self.B, kv_heads, self.cap, generator=g)
        self.max_new = max(new) if new else 0
        self.g = g

    def tokens(self, b):
        """k, v [kv_heads, length, dim] of sequence b in float64, and which of its tokens have a page."""
        n = self.lengths[b]
        j = np.arange(n)
        p = self.pages[b, j // self.page]
        there = (p >= 0) & (p < self.n_pages)
        safe = torch.from_numpy(np.where(there, p, 0).astype(np.int64))
        slot = torch.from_numpy(j % self.page)
        k, v = (x[safe, :, slot].transpose(0, 1).double().numpy() for x in (self.k, self.v))
        return k, v, there

    def attention(self, scale, causal):
        """out [rows, heads, dim] (NaN rows: not written), lse, weight, and for tolerances
        per row sum p|v| and the largest sum |q||k| scale."""
        out = np.full((self.rows, self.heads, self.dim), np.nan)
        mag = np.full((self.rows, self.heads, self.dim), np.nan)
        lse = np.full((self.rows, self.heads), np.nan)
        weight = self.weight.double().numpy().copy()
        span = 0.0
        q = self.q.double().numpy()
        G = self.heads // self.kv_heads
        for b in range(self.B):
            n, m = self.lengths[b], self.new[b]
            k, v, there = self.tokens(b)
            for i in range(m):
                row = self.start[b] + i
                seen = there & (np.arange(n) <= (n - m + i if causal else n))
                for h in range(self.heads):
                    kk, vv = k[h // G][seen], v[h // G][seen]
                    s = scale * (kk @ q[row, h])
                    if s.size == 0:
                        out[row, h], mag[row, h], lse[row, h] = 0, 0, -np.inf
                        continue
                    if np.isfinite(kk).all():
                        span = max(span, scale * (np.abs(kk) @ np.abs(q[row, h])).max())
                    z = s.max() + np.log(np.exp(s - s.max()).sum())
                    p = np.exp(s - z)
                    out[row, h], mag[row, h], lse[row, h] = p @ vv, p @ np.abs(vv), z
                    weight[b, h // G, np.flatnonzero(seen)] += p
        return out, lse, weight, mag, span

    def device(self, dev, with_weight=True):
        """KvCache and chunk tensors on the device. `order`: the pool's layout in memory."""
        import paper_2604_02945_amd as msao
        k, v = self.k.to(dev), self.v.to(dev)
        if self.order == "token":  # pages of tokens of heads
            k, v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
        elif self.order == "mixed":  # k and v of a token side by side
            both = torch.stack([k.transpose(1, 2), v.transpose(1, 2)], 3).contiguous()  # [pages, slot, heads, 2, dim]
            k, v = both[:, :, :, 0].transpose(1, 2), both[:, :, :, 1].transpose(1, 2)
        cache = msao.KvCache(k, v, torch.from_numpy(self.pages).to(dev),
                             torch.tensor(self.lengths, dtype=torch.int32, device=dev),
                             self.weight.to(dev) if with_weight else None)
        return cache, torch.from_numpy(self.start).to(dev)


def tolerances(case, mag, span, out):
    """Bounds on |error| of lse and out. A score is a sum of dim products in 32 bits, off
    by at most (dim + 2) 2^-24 sum |q||k| scale = d; the exponent function and the sums
    over L tokens add (L + 8) 2^-24 relative. With d' = d + (L + 8) 2^-24, lse is off by
    at most d', and out by 2 d' sum p|v|; bf16 rounds each p that multiplies v (2^-8) and
    the result (2^-8 of it), float32 the result (2^-24)."""
    L = max(case.lengths) if case.lengths else 0
    d = (case.dim + 2) * 2.0 ** -24 * span + (L + 8) * 2.0 ** -24
    bf = case.dtype == torch.bfloat16
    half = 2.0 ** -8 if bf else 2.0 ** -24
    tol = 2 * d * mag + half * np.abs(out) * 1.01 + (half * mag * 1.01 if bf else 0) + 1e-30
    # ln 2 times the base-2 sum: two more roundings of lse itself
    return d + 2.0 ** -22 * (np.abs(span) + np.log(L + 2)), tol


def evicted(weight, length, budget, cap_to, n_first, n_recent):
    """Kept tokens (ascending) of one (sequence, kv head)."""
    k = min(length, max(budget, 0), cap_to)
    a = min(n_first, k)
    r = min(n_recent, k - a)
    w = weight[:length].astype(np.float64)
    key = np.where(w > 0, w, 0.0)
    mid = np.arange(a, length - r)
    best = mid[np.argsort(-key[mid], kind="stable")][:k - a - r]
    return np.sort(np.concatenate([np.arange(a), best, np.arange(length - r, length)])).astype(np.int64)
