"""Work cases of the operators that read a model's answers and route queries.

A case is a plain dict; ``kind`` says which call it stands for:

  logprobs     log-probabilities of given tokens from the vocabulary's logits,
               with the entropy and the top alternatives of every position
  logprobs_grad  its gradient with respect to the logits
  scores       tokens reduced to one row of scores per answer
  scores_grad  its gradient with respect to the tokens' values
  route        queries to experts (models, replicas): scores, a bias for
               balance, groups, the k best, their weights, and the load
  route_grad   the gradient of the weights with respect to the logits

``run`` computes a case in elementary torch operations in 32 bits, or, where
``own`` is set, through this library's entry points.
"""
import math

import torch

own = False

F32, F64 = torch.float32, torch.float64
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
INF = float("inf")


def _lp(name, T, V, dtype, k, scale=1.0, masked=0, pitch=0, grad=False, ent=True):
    """masked: columns at the row's end that are -inf; pitch: elements between rows beyond V."""
    c = dict(kind="logprobs_grad" if grad else "logprobs", T=T, V=V, dtype=dtype, k=k, scale=scale,
             masked=masked, pitch=pitch, ent=ent)
    return dict(c, name=name) if name else c


def _sc(name, Q, mean, grad=False):
    c = dict(kind="scores_grad" if grad else "scores", Q=Q, mean=mean)
    return dict(c, name=name) if name else c


def _rt(name, T, E, dtype, mode, k, G=1, keep=1, gtop=1, renorm=True, bias=False, masked=0,
        factor=1.0, grad=False):
    """masked: in every 16th query, that many experts are out of service (-inf)."""
    c = dict(kind="route_grad" if grad else "route", T=T, E=E, dtype=dtype, mode=mode, k=k, G=G,
             keep=keep, gtop=gtop, renorm=renorm, bias=bias, masked=masked, factor=factor)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one answer while it is generated: latency alone
        _lp("logprobs-one", 1, 50021, "bf16", 5),
        # a step of sixty-four answers that are generated together, logits in 32 bits
        _lp("logprobs-decode", 64, 131072, "f32", 20, scale=1.25),
        # a few finished answers, an odd vocabulary (rows start anywhere), fp16
        _lp("logprobs-answers-odd", 2039, 50021, "f16", 8, scale=1.0 / 0.7),
        # a batch of long answers scored at once, a padded vocabulary
        _lp("logprobs-largest", 8192, 131072, "bf16", 20, masked=321),
        # a small training step in 32 bits, likelihood and entropy
        _lp("logprobs-grad-small", 48, 32768, "f32", 0, grad=True),
        # a large training step on 16-bit logits
        _lp("logprobs-grad-largest", 8192, 131072, "bf16", 0, scale=1.25, masked=321, grad=True),
        # the answers of a benchmark's questions, ragged
        _sc("scores-ragged", 4096, 200),
        # long answers, the training direction
        _sc("scores-grad-long", 96, 16384, grad=True),
        # the queries of one scheduling tick over one fleet
        _rt("route-tick", 32, 64, "f32", "softmax", 2),
        # model types as groups, replicas as experts, a bias that evens out the load
        _rt("route-groups", 4099, 192, "bf16", "sigmoid", 6, G=8, keep=4, gtop=2, bias=True,
            masked=9, factor=2.5),
        # a day of queries replayed for one evaluation of a configuration
        _rt("route-largest", 262144, 256, "bf16", "softmax", 4),
        # the router's training step
        _rt("route-grad-large", 131072, 160, "f32", "sigmoid", 6, bias=True, grad=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("logprobs", "logprobs", "logprobs_grad", "scores", "scores_grad", "route",
                       "route", "route_grad"))
    dtype = rng.choice(("f32", "f16", "bf16", "bf16"))
    if kind.startswith("logprobs"):
        grad = kind.endswith("grad")
        V = _log(rng, 500, 131072)
        if rng.random() < 0.5:
            V = max(512, V // 256 * 256)
        most = (1 << 31) // (V * BYTES[dtype])  # 2 GiB of logits, as the largest listed case
        T = _log(rng, 1, min(8192, most))
        return _lp(None, T, V, dtype, 0 if grad else rng.randint(1, 32),
                   scale=rng.choice((1.0, 1.25, 1.0 / 0.7)),
                   masked=rng.choice((0, 0, rng.randint(1, V // 4))),
                   pitch=rng.choice((0, 0, rng.randint(1, 64))), grad=grad,
                   ent=not grad or rng.random() < 0.7)
    if kind.startswith("scores"):
        Q = _log(rng, 1, 16384)
        return _sc(None, Q, _log(rng, 4, min(16384, (1 << 21) // Q)), grad=kind.endswith("grad"))
    grad = kind.endswith("grad")
    G = rng.choice((1, 1, 2, 4, 8))
    E = G * rng.randint(max(2, 8 // G), 320 // G)
    T = _log(rng, 1, 131072)
    keep = rng.randint(max(1, G // 4), G)
    k = rng.randint(1, min(10, keep * (E // G)))
    mode = rng.choice(("softmax", "sigmoid"))
    return _rt(None, T, E, dtype, mode, k, G=G, keep=keep,
               gtop=rng.randint(1, 2) if G > 1 else 1, renorm=rng.random() < 0.7,
               bias=mode == "sigmoid" or rng.random() < 0.3,
               masked=rng.choice((0, rng.randint(1, E // 2))), factor=rng.choice((1.0, 2.5)),
               grad=grad)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)


def _vocab_logits(c, g):
    """Most of a vocabulary is noise; a few tokens of each position stand out, now and then one."""
    T, V = c["T"], c["V"]
    buf = torch.empty((T, V + c["pitch"]), dtype=DTYPES[c["dtype"]], device="cuda")
    x = buf[:, :V]
    for r0 in range(0, T, 1024):
        r1 = min(T, r0 + 1024)
        z = torch.randn((r1 - r0, V), generator=g, device="cuda") * 1.7
        n = min(24, V)  # one of each n-th of the vocabulary
        at = torch.randint(0, V // n, (r1 - r0, n), generator=g, device="cuda")
        at += torch.arange(n, device="cuda") * (V // n)
        up = 4.0 + 12.0 * torch.rand((r1 - r0, n), generator=g, device="cuda") ** 2
        z.scatter_(1, at, up)
        x[r0:r1] = z.to(x.dtype)
        if c["masked"]:
            x[r0:r1, V - c["masked"]:] = -INF
    # the given tokens: mostly likely ones, some any; a few positions hold no token
    t = torch.randint(0, V - c["masked"], (T,), generator=g, device="cuda")
    best = x.argmax(1)
    pick = torch.rand((T,), generator=g, device="cuda")
    t = torch.where(pick < 0.6, best, t)
    if T > 8:
        t = torch.where(pick > 0.97, torch.full_like(t, -1), t)
    return x, t


def _lse_entropy(c, x):
    """What the forward pass left for the backward pass."""
    lse, ent = [], []
    for r in x.split(512):
        z = r.float() * c["scale"]
        m = z.amax(1, keepdim=True)
        e = torch.exp(z - m)
        s = e.sum(1, keepdim=True)
        d = torch.where(e > 0, z - m, torch.zeros_like(z))
        lse.append((m + torch.log(s))[:, 0])
        ent.append((torch.log(s) - (e * d).sum(1, keepdim=True) / s)[:, 0])
    return torch.cat(lse), torch.cat(ent)


def _offsets(c, g):
    """Q mean tokens in answers of log-normal lengths, now and then an empty one."""
    w = torch.exp(0.8 * torch.randn((c["Q"],), generator=g, device="cuda")).double()
    if c["Q"] > 50:
        w *= torch.rand((c["Q"],), generator=g, device="cuda") > 0.01
    off = torch.zeros((c["Q"] + 1,), dtype=torch.int64, device="cuda")
    off[1:] = (w.cumsum(0) / w.sum() * (c["Q"] * c["mean"])).round()
    off[-1] = c["Q"] * c["mean"]
    return off


def _near_ties(c, x, b):
    """Queries whose choice hangs on the last bits of a 32-bit score."""
    s = _scores64(c, x)
    v = s if b is None else s + b.double()
    v = torch.where(torch.isinf(x), torch.full_like(v, -INF), v)
    T, E, G = x.shape[0], c["E"], c["G"]
    tol = 1e-6 * (s.amax(1, keepdim=True) + (0.0 if b is None else b.abs().max().double()))

    def close(w, n):
        w = w.sort(1, descending=True).values[:, :n + 1]
        gap = w[:, :-1] - w[:, 1:]
        return ((gap > 0) & (gap < tol)).any(1)

    bad = torch.zeros((T,), dtype=torch.bool, device=x.device)
    if G > 1:
        gv = v.view(T, G, E // G).sort(2, descending=True).values[:, :, :c["gtop"]]
        gs = torch.where(torch.isinf(gv), torch.zeros_like(gv), gv).sum(2)
        gs = torch.where(torch.isinf(gv[:, :, 0]), torch.full_like(gs, -INF), gs)
        bad |= close(gs, c["keep"])
        kept = gs.sort(1, descending=True).values[:, c["keep"] - 1:c["keep"]]
        v = torch.where((gs < kept).repeat_interleave(E // G, 1), torch.full_like(v, -INF), v)
    return bad | close(v, c["k"])


def _route_inputs(c, g):
    T, E = c["T"], c["E"]
    dt = DTYPES[c["dtype"]]
    lean = torch.randn((E,), generator=g, device="cuda") * 0.7  # some experts are liked more

    def draw_rows(n):
        return (torch.randn((n, E), generator=g, device="cuda") * 1.5 + lean).to(dt)

    x = draw_rows(T)
    # the bias moved in fixed steps against the load
    b = None
    if c["bias"]:
        b = -(lean * 100).round() * 1e-3 if c["mode"] == "sigmoid" else -(lean * 20).round() * 1e-3
    # near ties are drawn again: there the formulas leave the choice to the last bit
    off = torch.zeros((T, E), dtype=torch.bool, device="cuda")
    if c["masked"]:
        order = torch.rand((E,), generator=g, device="cuda").argsort()[:c["masked"]]
        off[::16, order] = True
    x = x.masked_fill(off, -INF)
    for _ in range(30):
        rows = _near_ties(c, x, b).nonzero()[:, 0]
        if rows.numel() == 0:
            break
        x[rows] = draw_rows(rows.numel()).masked_fill(off[rows], -INF)
    return x, b


def prepare(case, seed):
    c, g = case, _gen(seed)
    dev = dict(device="cuda")
    st = dict(c=c)
    if c["kind"].startswith("logprobs"):
        T, k = c["T"], c["k"]
        x, t = _vocab_logits(c, g)
        st |= dict(x=x, t=t)
        if c["kind"] == "logprobs":
            st |= dict(logprob=torch.empty((T,), **dev), entropy=torch.empty((T,), **dev),
                       lse=torch.empty((T,), **dev),
                       ti=torch.empty((T, k), dtype=torch.int64, **dev),
                       tv=torch.empty((T, k), **dev))
        else:
            lse, ent = _lse_entropy(c, x)
            st |= dict(lse=lse, ent=ent, glp=torch.randn((T,), generator=g, **dev),
                       gent=0.05 * torch.randn((T,), generator=g, **dev) if c["ent"] else None,
                       dx=torch.empty((T, c["V"]), dtype=x.dtype, **dev))
    elif c["kind"].startswith("scores"):
        off, T = _offsets(c, g), c["Q"] * c["mean"]
        lp = torch.log(torch.rand((T,), generator=g, **dev).clamp_min(1e-6)) * 0.7
        ent = -0.8 * torch.log(torch.rand((T,), generator=g, **dev).clamp_min(1e-6))
        t = torch.randint(0, 50021, (T,), generator=g, **dev)
        t = torch.where(torch.rand((T,), generator=g, **dev) < 0.02, torch.full_like(t, -1), t)
        st |= dict(lp=lp, ent=ent, t=t, off=off)
        if c["kind"] == "scores":
            st |= dict(scores=torch.empty((c["Q"], 4), **dev),
                       counts=torch.empty((c["Q"],), dtype=torch.int32, **dev))
        else:
            st |= dict(gs=torch.randn((c["Q"], 4), generator=g, **dev),
                       glp=torch.empty((T,), **dev), gent=torch.empty((T,), **dev))
    else:
        x, b = _route_inputs(c, g)
        T, k = c["T"], c["k"]
        st |= dict(x=x, b=b)
        if c["kind"] == "route":
            st |= dict(idx=torch.empty((T, k), dtype=torch.int32, **dev),
                       w=torch.empty((T, k), **dev),
                       load=torch.empty((c["E"],), dtype=torch.int32, **dev))
        else:
            s = _plain_scores(c, x)
            st |= dict(idx=_plain_choice(c, x, b, s), gw=torch.randn((T, k), generator=g, **dev),
                       dx=torch.empty_like(x))
    return st


# ---------------------------------------------------------------- plain forms
def _keys(v):
    """64-bit keys that order by value descending, then index ascending; -0 as +0."""
    u = torch.where(v == 0, torch.zeros_like(v), v).view(torch.int32).long()
    u = torch.where(u >= 0, u, -(u & 0x7FFFFFFF) - 1)
    return (u << 32) + (0x7FFFFFFF - torch.arange(v.shape[-1], device=v.device))


def _best(v, k):
    """Indices of the k largest, ties to the lowest index; -1 where there is none above -inf."""
    i = 0x7FFFFFFF - (torch.topk(_keys(v), k, dim=-1).values & 0xFFFFFFFF)
    return torch.where(torch.gather(v, -1, i) > -INF, i, torch.full_like(i, -1))


def _plain_logprobs(st):
    c, t = st["c"], st["t"]
    z = st["x"].float() * c["scale"]
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    s = e.sum(1, keepdim=True)
    ls = torch.log(s)
    d = torch.where(e > 0, z - m, torch.zeros_like(z))
    entropy = (ls - (e * d).sum(1, keepdim=True) / s)[:, 0]
    logprob = torch.gather(z, 1, t.clamp_min(0)[:, None]) - m - ls
    logprob = torch.where(t >= 0, logprob[:, 0], torch.zeros_like(entropy))
    ti = _best(z, c["k"])
    tv = torch.gather(z, 1, ti.clamp_min(0)) - m - ls
    tv = torch.where(ti >= 0, tv, torch.full_like(tv, -INF))
    return dict(logprob=logprob, entropy=entropy, lse=(m + ls)[:, 0], top_idx=ti, top_logprob=tv)


def _plain_logprobs_grad(st):
    c, t = st["c"], st["t"]
    g = torch.where(t >= 0, st["glp"], torch.zeros_like(st["glp"]))[:, None]
    lp = st["x"].float() * c["scale"] - st["lse"][:, None]
    p = torch.exp(lp)
    d = -g * p
    if st["gent"] is not None:
        lp = torch.where(p > 0, lp, torch.zeros_like(lp))
        d -= st["gent"][:, None] * p * (lp + st["ent"][:, None])
    d.scatter_add_(1, t.clamp_min(0)[:, None], g)
    return dict(dlogits=(d * c["scale"]).to(st["x"].dtype))


def _segments(st):
    off = st["off"]
    Q = off.numel() - 1
    seg = torch.searchsorted(off, torch.arange(st["lp"].numel(), device=off.device), right=True) - 1
    return seg.clamp(0, Q - 1), Q, st["t"] >= 0


def _extremes(st, seg, Q, on):
    full = lambda v: torch.full((Q,), v, device=seg.device)
    lo = full(INF).scatter_reduce(0, seg, torch.where(on, st["lp"], torch.full_like(st["lp"], INF)),
                                  "amin")
    hi = full(-INF).scatter_reduce(0, seg,
                                   torch.where(on, st["ent"], torch.full_like(st["ent"], -INF)),
                                   "amax")
    return lo, hi


def _plain_scores_of_answers(st):
    seg, Q, on = _segments(st)
    zero = torch.zeros((Q,), device=seg.device)
    cnt = zero.index_add(0, seg, on.float())
    some = cnt > 0
    mean = lambda v: torch.where(some, zero.index_add(0, seg, torch.where(on, v, torch.zeros_like(
        v))) / cnt.clamp_min(1), zero)
    lo, hi = _extremes(st, seg, Q, on)
    scores = torch.stack([mean(st["lp"]), torch.where(some, lo, zero), mean(st["ent"]),
                          torch.where(some, hi, zero)], 1)
    return dict(scores=scores, counts=cnt.to(torch.int32))


def _plain_scores_grad(st):
    seg, Q, on = _segments(st)
    n = torch.zeros((Q,), device=seg.device).index_add(0, seg, on.float()).clamp_min(1)
    lo, hi = _extremes(st, seg, Q, on)
    at = torch.arange(seg.numel(), device=seg.device)

    def first(hit):
        none = torch.full((Q,), seg.numel(), dtype=torch.int64, device=seg.device)
        return none.scatter_reduce(0, seg, torch.where(hit, at, torch.full_like(at, seg.numel())),
                                   "amin")[seg] == at

    gs, z = st["gs"][seg], torch.zeros_like(st["lp"])
    glp = gs[:, 0] / n[seg] + torch.where(first(on & (st["lp"] == lo[seg])), gs[:, 1], z)
    gent = gs[:, 2] / n[seg] + torch.where(first(on & (st["ent"] == hi[seg])), gs[:, 3], z)
    return dict(g_logprob=torch.where(on, glp, z), g_entropy=torch.where(on, gent, z))


def _plain_scores(c, x):
    x = x.float()
    if c["mode"] == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-x))
    e = torch.exp(x - x.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _plain_choice(c, x, b, s):
    T, E, G = x.shape[0], c["E"], c["G"]
    v = s if b is None else s + b
    v = torch.where(x > -INF, v, torch.full_like(v, -INF))
    if G > 1:
        top = torch.topk(v.view(T, G, E // G), c["gtop"], dim=2).values
        gs = torch.where(top > -INF, top, torch.zeros_like(top)).sum(2)
        gs = torch.where(top[:, :, 0] > -INF, gs, torch.full_like(gs, -INF))
        kept = _best(gs, c["keep"])
        on = torch.zeros((T, G + 1), dtype=torch.bool, device=x.device)
        on.scatter_(1, torch.where(kept < 0, torch.full_like(kept, G), kept), True)
        v = torch.where(on[:, :G].repeat_interleave(E // G, 1), v, torch.full_like(v, -INF))
    return _best(v, c["k"]).to(torch.int32)


def _plain_route(st):
    c = st["c"]
    s = _plain_scores(c, st["x"])
    idx = _plain_choice(c, st["x"], st["b"], s)
    i = idx.long()
    w = torch.where(i >= 0, torch.gather(s, 1, i.clamp_min(0)), torch.zeros_like(s[:, :1]))
    if c["renorm"]:
        S = w.sum(1, keepdim=True)
        w = torch.where(S > 0, w / S, torch.zeros_like(w))
    at = torch.where(i >= 0, i, torch.full_like(i, c["E"])).reshape(-1)
    load = torch.zeros((c["E"] + 1,), dtype=torch.int32, device=at.device)
    load.index_add_(0, at, torch.ones_like(at, dtype=torch.int32))
    return dict(idx=idx, weight=w * c["factor"], load=load[:c["E"]])


def _plain_route_grad(st):
    c, i = st["c"], st["idx"].long()
    s = _plain_scores(c, st["x"])
    on = i >= 0
    z = torch.zeros_like(st["gw"])
    si = torch.where(on, torch.gather(s, 1, i.clamp_min(0)), z)
    g = torch.where(on, st["gw"], z) * c["factor"]
    if c["renorm"]:
        S = si.sum(1, keepdim=True)
        g = torch.where(S > 0, (g - (g * si).sum(1, keepdim=True) / S) / S, z)
    g = torch.where(on, g, z)
    ds = torch.zeros_like(s).scatter_add_(1, i.clamp_min(0), g)
    if c["mode"] == "sigmoid":
        dx = ds * s * (1 - s)
    else:
        dx = s * (ds - (g * si).sum(1, keepdim=True))
    return dict(dlogits=dx.to(st["x"].dtype))


# ---------------------------------------------------------------- the library
def _own(st):
    from paper_2602_10729_gb300 import boute as bt
    c, kind = st["c"], st["c"]["kind"]
    if kind == "logprobs":
        bt.boute_token_logprobs(st["x"], st["t"], c["scale"], st["logprob"], st["entropy"],
                                st["lse"], st["ti"], st["tv"])
        return dict(logprob=st["logprob"], entropy=st["entropy"], lse=st["lse"],
                    top_idx=st["ti"], top_logprob=st["tv"])
    if kind == "logprobs_grad":
        bt.boute_token_logprobs_grad(st["x"], st["t"], c["scale"], st["lse"], st["ent"],
                                     st["glp"], st["gent"], st["dx"])
        return dict(dlogits=st["dx"])
    if kind == "scores":
        bt.boute_answer_scores(st["lp"], st["ent"], st["t"], st["off"], st["scores"],
                               st["counts"])
        return dict(scores=st["scores"], counts=st["counts"])
    if kind == "scores_grad":
        bt.boute_answer_scores_grad(st["lp"], st["ent"], st["t"], st["off"], st["gs"], st["glp"],
                                    st["gent"])
        return dict(g_logprob=st["glp"], g_entropy=st["gent"])
    mode = bt.BOUTE_ROUTE_SIGMOID if c["mode"] == "sigmoid" else bt.BOUTE_ROUTE_SOFTMAX
    if kind == "route":
        bt.boute_route(st["x"], st["b"], mode, c["G"], c["keep"], c["gtop"], c["renorm"],
                       c["factor"], st["idx"], st["w"], st["load"])
        return dict(idx=st["idx"], weight=st["w"], load=st["load"])
    bt.boute_route_grad(st["x"], mode, c["renorm"], c["factor"], st["idx"], st["gw"], st["dx"])
    return dict(dlogits=st["dx"])


PLAIN = dict(logprobs=_plain_logprobs, logprobs_grad=_plain_logprobs_grad,
             scores=_plain_scores_of_answers, scores_grad=_plain_scores_grad,
             route=_plain_route, route_grad=_plain_route_grad)


def run(state):
    return _own(state) if own else PLAIN[state["c"]["kind"]](state)


def work(case):
    """Each input read once, each output written once; a floating operation per step of the formulas."""
    c, kind = case, case["kind"]
    if kind.startswith("logprobs"):
        n = c["T"] * c["V"]
        if kind == "logprobs":
            return dict(bytes=n * BYTES[c["dtype"]] + c["T"] * (8 + 12 + 12 * c["k"]),
                        flops=6.0 * n)
        return dict(bytes=2 * n * BYTES[c["dtype"]] + c["T"] * 24, flops=(8.0 if c["ent"] else 5.0) * n)
    if kind.startswith("scores"):
        T = c["Q"] * c["mean"]
        if kind == "scores":
            return dict(bytes=16 * T + 28 * c["Q"], flops=4.0 * T)
        return dict(bytes=24 * T + 24 * c["Q"], flops=8.0 * T)
    n = c["T"] * c["E"]
    if kind == "route":
        return dict(bytes=n * BYTES[c["dtype"]] + 8 * c["T"] * c["k"] + 8 * c["E"], flops=8.0 * n)
    return dict(bytes=2 * n * BYTES[c["dtype"]] + 8 * c["T"] * c["k"], flops=8.0 * n)


# ---------------------------------------------------------------- 64 bits
def _scores64(c, x):
    x = x.double()
    if c["mode"] == "sigmoid":
        return torch.sigmoid(x)
    return torch.softmax(x, 1)


def _exact_logprobs(st):
    c, out = st["c"], []
    scale = torch.tensor(c["scale"], dtype=F32).double().item()
    for r0 in range(0, c["T"], 256):
        x, t = st["x"][r0:r0 + 256].double() * scale, st["t"][r0:r0 + 256]
        lp = torch.log_softmax(x, 1)
        p = torch.exp(lp)
        H = -torch.special.xlogy(p, p).sum(1)
        at = torch.take_along_dim(lp, t.clamp_min(0)[:, None], 1)[:, 0]
        # (by value alone: equal values have equal log-probabilities)
        out.append((at.masked_fill(t < 0, 0.0), H, torch.logsumexp(x, 1),
                    torch.topk(lp, c["k"], 1).values))
    lp, H, lse, tv = (torch.cat(v) for v in zip(*out))
    return dict(logprob=lp, entropy=H, lse=lse, top_idx=None, top_logprob=tv)


def _exact_logprobs_grad(st):
    c = st["c"]
    scale = torch.tensor(c["scale"], dtype=F32).double().item()
    dx = torch.empty((c["T"], c["V"]), dtype=F64, device="cuda")
    for r0 in range(0, c["T"], 256):
        r = slice(r0, min(c["T"], r0 + 256))
        t = st["t"][r]
        lp = st["x"][r].double() * scale - st["lse"][r].double()[:, None]
        p = torch.exp(lp)
        one = torch.arange(c["V"], device="cuda")[None] == t[:, None]
        g = st["glp"][r].double().masked_fill(t < 0, 0.0)[:, None]
        d = g * (one.double() - p)
        if st["gent"] is not None:
            d = d - st["gent"][r].double()[:, None] * (torch.special.xlogy(p, p) +
                                                       p * st["ent"][r].double()[:, None])
        dx[r] = scale * d
    return dict(dlogits=dx)


def _answer_parts(st):
    off = st["off"].tolist()
    lp, ent, t = st["lp"].double().cpu(), st["ent"].double().cpu(), st["t"].cpu()
    for q in range(len(off) - 1):
        s = slice(off[q], off[q + 1])
        yield q, s, lp[s], ent[s], t[s] >= 0


def _exact_scores(st):
    out = torch.zeros((st["c"]["Q"], 4), dtype=F64)
    for q, _, lp, ent, on in _answer_parts(st):
        if bool(on.any()):
            lp, ent = lp[on], ent[on]
            out[q] = torch.stack([lp.mean(), lp.min(), ent.mean(), ent.max()])
    return dict(scores=out, counts=None)


def _exact_scores_grad(st):
    T = st["lp"].numel()
    glp, gent = torch.zeros((T,), dtype=F64), torch.zeros((T,), dtype=F64)
    gs = st["gs"].double().cpu()
    for q, s, lp, ent, on in _answer_parts(st):
        at = on.nonzero()[:, 0] + s.start
        if at.numel() == 0:
            continue
        glp[at] = gs[q, 0] / at.numel()
        gent[at] = gs[q, 2] / at.numel()
        lo = (on & (lp == lp[on].min())).nonzero()[0, 0] + s.start
        hi = (on & (ent == ent[on].max())).nonzero()[0, 0] + s.start
        glp[lo] += gs[q, 1]
        gent[hi] += gs[q, 3]
    return dict(g_logprob=glp, g_entropy=gent)


def _exact_weights(c, s, i):
    w = torch.take_along_dim(s, i.clamp_min(0), 1) * (i >= 0)
    return w / w.sum(1, keepdim=True).clamp_min(1e-300) if c["renorm"] else w


def _exact_route(st):
    c, x = st["c"], st["x"]
    s = _scores64(c, x)
    v = s if st["b"] is None else s + st["b"].double()
    v = v.masked_fill(x == -INF, -INF)
    T, E, G = c["T"], c["E"], c["G"]
    if G > 1:
        m = v.reshape(T, G, E // G).sort(2, descending=True).values[:, :, :c["gtop"]]
        gs = m.masked_fill(m == -INF, 0.0).sum(2).masked_fill(m[:, :, 0] == -INF, -INF)
        rank = torch.argsort(gs, dim=1, descending=True, stable=True).argsort(1)
        v = v.masked_fill((rank >= c["keep"]).repeat_interleave(E // G, 1), -INF)
    val, i = torch.sort(v, dim=1, descending=True, stable=True)
    val, i = val[:, :c["k"]], i[:, :c["k"]]
    i = i.masked_fill(val == -INF, -1)
    return dict(idx=None, weight=_exact_weights(c, s, i) * c["factor"], load=None)


def _exact_route_grad(st):
    c, i = st["c"], st["idx"].long()
    out = []
    for r in range(0, c["T"], 8192):
        x = st["x"][r:r + 8192].double().requires_grad_(True)
        w = _exact_weights(c, _scores64(c, x), i[r:r + 8192]) * c["factor"]
        (d,) = torch.autograd.grad((w * st["gw"][r:r + 8192].double()).sum(), x)
        out.append(torch.nan_to_num(d))
    return dict(dlogits=torch.cat(out))


EXACT = dict(logprobs=_exact_logprobs, logprobs_grad=_exact_logprobs_grad, scores=_exact_scores,
             scores_grad=_exact_scores_grad, route=_exact_route, route_grad=_exact_route_grad)


def exact(case, seed):
    return EXACT[case["kind"]](prepare(case, seed))
