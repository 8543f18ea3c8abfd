"""Plain 64-bit numpy forms of the operators over a model's answers: token
log-probabilities, scores per answer, routing, and their gradients. Loops over
rows and positions, straight from the definitions."""
import numpy as np

U = 2.0 ** -24  # half a unit in the last place of fp32


def token_row(x, scale, target, k):
    """(logprob, entropy, lse, top_idx, top_logprob) of one row; x: the stored values."""
    z = (x.astype(np.float32) * np.float32(scale)).astype(np.float64)  # one rounding, by definition
    V = len(z)
    if np.isnan(z).any() or (z == np.inf).any():
        lp = 0.0 if target < 0 else np.nan
        return lp, np.nan, np.nan, [-1] * k, [np.nan] * k
    m = z.max()
    if m == -np.inf:
        lp = 0.0 if target < 0 else np.nan if target >= V else -np.inf
        return lp, 0.0, -np.inf, [-1] * k, [-np.inf] * k
    e = np.exp(z - m)
    ls = np.log(e.sum())  # (kept apart from m, beside which it can vanish)
    p = e / e.sum()
    on = p > 0
    H = -(p[on] * (z[on] - m - ls)).sum()
    lp = 0.0 if target < 0 else np.nan if target >= V else z[target] - m - ls
    order = np.lexsort((np.arange(V), -z))[:k]
    idx = [int(j) if z[j] > -np.inf else -1 for j in order]
    return lp, H, m + ls, idx, [z[j] - m - ls for j in order]


def token_grad_row(x, scale, target, g, gh):
    """The gradient of one row for the outputs' gradients g and gh."""
    z = x.astype(np.float64) * float(np.float32(scale))
    V = len(z)
    if target >= V or np.isnan(z).any() or (z == np.inf).any():
        return np.full(V, np.nan)
    if target < 0:
        g = 0.0
    m = z.max()
    if m == -np.inf:
        return np.zeros(V)
    p = np.exp(z - m)
    ls = np.log(p.sum())
    p /= p.sum()
    lp = np.where(p > 0, z - m - ls, 0.0)
    H = -(p * lp).sum()
    d = -p * (g + gh * (lp + H))
    if target >= 0:
        d[target] += g
    return d * float(np.float32(scale))


def answer_rows(lp, ent, targets, offsets):
    Q = len(offsets) - 1
    out, cnt = np.zeros((Q, 4)), np.zeros(Q, np.int64)
    for q in range(Q):
        t = np.arange(offsets[q], offsets[q + 1])
        t = t[targets[t] >= 0] if targets is not None else t
        cnt[q] = len(t)
        if len(t):
            a, b = lp[t].astype(np.float64), ent[t].astype(np.float64)
            out[q] = a.mean(), a.min(), b.mean(), b.max()
    return out, cnt


def answer_grad(lp, ent, targets, offsets, g):
    gl, gh = np.zeros(len(lp)), np.zeros(len(lp))
    for q in range(len(offsets) - 1):
        t = np.arange(offsets[q], offsets[q + 1])
        t = t[targets[t] >= 0] if targets is not None else t
        if len(t) == 0:
            continue
        gl[t] = g[q, 0] / len(t)
        gh[t] = g[q, 2] / len(t)
        gl[t[np.argmin(lp[t])]] += g[q, 1]
        gh[t[np.argmax(ent[t])]] += g[q, 3]
    return gl, gh


def scores(x, mode):
    """softmax (mode 0) or logistic scores of one row, None without a distribution. What fp32
    cannot hold is 0, by definition."""
    x = x.astype(np.float64)
    if np.isnan(x).any() or (mode == 0 and (x == np.inf).any()):
        return None
    with np.errstate(over="ignore"):
        if mode == 1:
            s = 1.0 / (1.0 + np.exp(-x))
            return np.where(s < 2.0 ** -149, 0.0, s)
    m = x.max()
    if m == -np.inf:
        return np.zeros(len(x))
    e = np.exp(x - m)
    e /= e.sum()
    return np.where(e < 2.0 ** -149, 0.0, e)


def _gaps(v, n):
    v = np.sort(v)[::-1][:n + 1]
    with np.errstate(invalid="ignore"):
        d = v[:-1] - v[1:]
    d = d[(d > 0)]
    return d.min() if len(d) else np.inf


def route_row(x, bias, mode, G, keep, gtop, k, renorm, factor):
    """(idx, weight, gap): gap is the smallest nonzero difference that the choice hangs on."""
    E = len(x)
    s = scores(x, mode)
    if s is None:
        return [-1] * k, [np.nan] * k, np.inf
    with np.errstate(invalid="ignore"):
        c = s + (0.0 if bias is None else bias.astype(np.float64))
    c = np.where(np.isneginf(x.astype(np.float64)) | np.isnan(c), -np.inf, c)
    gap, per = np.inf, E // G
    if keep < G:
        gs = np.full(G, -np.inf)
        for g in range(G):
            top = np.sort(c[g * per:(g + 1) * per])[::-1][:gtop]
            top = top[top > -np.inf]
            if len(top):
                gs[g] = top.sum()
        order = np.lexsort((np.arange(G), -gs))[:keep]
        gap = _gaps(gs, keep)
        kept = [g for g in order if gs[g] > -np.inf]
        c = np.where(np.isin(np.arange(E) // per, kept), c, -np.inf)
    order = np.lexsort((np.arange(E), -c))[:k]
    gap = min(gap, _gaps(c, k))
    idx = [int(e) if c[e] > -np.inf else -1 for e in order]
    w = np.array([s[e] if e >= 0 else 0.0 for e in idx])
    if renorm:
        w = w / w.sum() if w.sum() > 0 else w * 0
    return idx, list(factor * w), gap


def route_grad_row(x, mode, idx, g, renorm, factor):
    E = len(x)
    s = scores(x, mode)
    on = [r for r, e in enumerate(idx) if e >= 0]
    if s is None or not on:
        return np.zeros(E)
    e = np.array([idx[r] for r in on])
    g = np.array([g[r] for r in on], np.float64) * factor
    if renorm:
        S = s[e].sum()
        g = (g - (g * s[e]).sum() / S) / S if S > 0 else g * 0
    ds = np.zeros(E)
    ds[e] += g
    return ds * s * (1 - s) if mode == 1 else s * (ds - (g * s[e]).sum())
