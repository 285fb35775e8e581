"""Plain 64-bit forms, on host arrays and from their definitions, of what draws tokens and
verifies drafts."""
import math

import numpy as np


def distribution(x, temperature=None, top_k=None, top_p=None, min_p=None):
    """(which tokens stay, ln p of them, p, the weights p is a share of) of one row of logits, None of a row
    without a distribution."""
    x = np.asarray(x, np.float64)
    if np.isnan(x).any() or (x == np.inf).any() or not np.isfinite(x).any():
        return None
    t = 1.0 if temperature is None else float(temperature)
    order = np.argsort(-x, kind="stable")
    order = order[np.isfinite(x[order])]
    if not t > 0:
        order = order[:1]
        t = 1.0
    if top_k is not None and top_k > 0:
        order = order[:top_k]
    with np.errstate(over="ignore", under="ignore"):
        z = (x[order] - x.max()) / t
        w = np.where(z >= -1000 * math.log(2), np.exp(z), 0.0)
    if top_p is not None and float(top_p) < 1:
        n = 1 + int((np.cumsum(w)[:-1] < float(top_p) * math.fsum(w)).sum())
        order, z, w = order[:n], z[:n], w[:n]
    if min_p is not None and float(min_p) > 0:
        n = int((z >= min(0.0, math.log(float(min_p)))).sum())
        order, z, w = order[:n], z[:n], w[:n]
    stays = np.zeros(x.shape, bool)
    stays[order] = True
    total = math.fsum(w)
    lp = np.full(x.shape, -np.inf)
    lp[order] = z - math.log(total)
    p, weight = np.zeros(x.shape), np.zeros(x.shape)
    p[order] = w / total
    weight[order] = w
    return stays, lp, p, weight


def pick(p, u):
    """The first index whose running sum passes u times the whole, None where there is nothing."""
    u = float(u) if u > 0 else 0.0
    run = np.cumsum(p)
    if not run.size or not run[-1] > 0:
        return None
    over = np.flatnonzero((run > u * run[-1]) & (p > 0))
    return int(over[0]) if over.size else int(np.flatnonzero(p > 0)[-1])


def row_settings(settings, r):
    return {k: None if v is None else v[r] for k, v in settings.items()}


def sample(x, u, settings):
    token, lp, kept = [], [], []
    for r in range(len(u)):
        d = distribution(x[r], **row_settings(settings, r))
        if d is None:
            token.append(-1), lp.append(np.nan), kept.append(0)
            continue
        t = pick(d[3], u[r])
        token.append(t), lp.append(d[1][t]), kept.append(int(d[0].sum()))
    return np.array(token), np.array(lp), np.array(kept)


def verify(start, max_new, tokens, x, y, ua, u, settings, length):
    """accepted, next, logprob, length; rows that are not written hold None."""
    rows, V = x.shape
    nxt, lps = [None] * rows, [None] * rows
    accepted, out = [], []
    for s in range(len(start) - 1):
        n_all = max(0, start[s + 1] - start[s])
        n, a = min(n_all, max_new), 0
        alive = n > 0
        for i in range(n):
            r = start[s] + i
            if not alive:
                nxt[r], lps[r] = -1, np.nan
                continue
            d = distribution(x[r], **row_settings(settings, r))
            alive = False
            if d is None:
                nxt[r], lps[r] = -1, np.nan
                continue
            p = d[2]
            if i == n - 1:
                t = pick(d[3], u[r])
            else:
                draft = int(tokens[r + 1])
                known = 0 <= draft < V
                e = None if y is None else distribution(y[r], **row_settings(settings, r))
                v = float(ua[r]) if ua[r] > 0 else 0.0
                if e is None:
                    alive = known and v < p[draft]
                    rest = d[3].copy()
                    if known:
                        rest[draft] = 0
                else:
                    alive = known and v * e[2][draft] < p[draft]
                    rest = np.maximum(p - e[2], 0)
                if alive:
                    a += 1
                    t = draft
                else:
                    t = pick(rest, u[r])
                    t = pick(d[3], u[r]) if t is None else t
            nxt[r], lps[r] = t, d[1][t]
        accepted.append(a)
        out.append(None if length is None else int(length[s]) - (n_all - 1 - a if n > 0 else 0))
    return accepted, nxt, lps, out
