"""Work cases of the operators between a router and a model's answers.

A case is a plain dict; ``kind`` says which calls it stands for:

  sort         the choices of a routing put in the order of their experts, and the
               queries' rows copied to the places of their choices
  combine      the experts' rows back to the queries, summed with the routing's weights
  expert_grad  the backward pass of both: the gradients of the experts' rows and of the
               weights, and (from the gradient of what the experts read) of the queries
  hidden       log-probabilities of given tokens and entropies from the last hidden
               states and the vocabulary's weight, without the logits
  hidden_grad  its gradient with respect to the hidden states and the weight

``run`` computes a case in elementary torch operations in 32 bits, or, where
``own`` is set, through this library's entry points.
"""
import math

import torch

own = False

F32, F64 = torch.float32, torch.float64
I32, I64 = torch.int32, torch.int64
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def _ex(kind, name, T, k, E, D, dtype, pitch=0, none=0.0):
    """pitch: elements between rows beyond D; none: the share of queries without a choice."""
    c = dict(kind=kind, T=T, k=k, E=E, D=D, dtype=dtype, pitch=pitch, none=none)
    return dict(c, name=name) if name else c


def _hd(kind, name, T, V, D, dtype, scale=1.0, ent=True, pitch=0):
    c = dict(kind=kind, T=T, V=V, D=D, dtype=dtype, scale=scale, ent=ent, pitch=pitch)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the queries of one scheduling tick, their features to the replicas: latency alone
        _ex("sort", "sort-tick", 32, 2, 64, 64, "f32"),
        # a batch of odd sizes, rows that start anywhere, some queries unserved
        _ex("sort", "sort-odd", 4099, 6, 61, 1001, "f16", pitch=3, none=0.05),
        # a day of queries replayed: many short rows, the sorting itself
        _ex("sort", "sort-replay", 262144, 4, 256, 24, "f32"),
        # the hidden states of a prompt batch to a layer's experts
        _ex("sort", "sort-largest", 65536, 8, 256, 2048, "bf16"),
        # one token each of sixty-four answers that are generated together
        _ex("combine", "combine-decode", 64, 8, 128, 4096, "bf16"),
        # the prompt batch's rows back
        _ex("combine", "combine-largest", 65536, 8, 256, 2048, "bf16"),
        # a small training step of odd sizes
        _ex("expert_grad", "expert-grad-odd", 4099, 3, 61, 1001, "f16", pitch=3, none=0.05),
        # a training batch
        _ex("expert_grad", "expert-grad-large", 32768, 8, 128, 4096, "bf16"),
        # one token of one answer while it is generated, an odd vocabulary
        _hd("hidden", "hidden-one", 1, 50021, 2048, "bf16"),
        # a batch of finished answers
        _hd("hidden", "hidden-largest", 4096, 131072, 4096, "bf16", scale=1.25),
        # a small training step, an odd vocabulary, likelihood and entropy
        _hd("hidden_grad", "hidden-grad-odd", 515, 50021, 1000, "f16", scale=1.0 / 0.7),
        # a large training step
        _hd("hidden_grad", "hidden-grad-largest", 4096, 131072, 2048, "bf16", ent=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("sort", "combine", "expert_grad", "hidden", "hidden_grad"))
    if kind.startswith("hidden"):
        V, D = _log(rng, 500, 131072), _log(rng, 32, 4096)
        if rng.random() < 0.5:
            V = max(512, V // 256 * 256)
        if rng.random() < 0.8:  # (a head's rows are whole vectors, as a rule)
            D = max(32, D // 32 * 32)
        most = (4096 * 131072 * (4096 if kind == "hidden" else 2048)) // (V * D)
        return _hd(kind, None, _log(rng, 1, min(4096, most)), V, D,
                   rng.choice(("f16", "bf16", "bf16")), scale=rng.choice((1.0, 1.25, 1.0 / 0.7)),
                   ent=kind == "hidden" or rng.random() < 0.5,
                   pitch=rng.choice((0, 0, 8 * rng.randint(1, 8))))
    E = _log(rng, 2, 512)
    k = rng.randint(1, min(E, 10))
    D = _log(rng, 8, 8192)
    if rng.random() < 0.7:
        D = max(8, D // 8 * 8)
    dtype = rng.choice(("f32", "f16", "bf16", "bf16"))
    # 1 GiB of experts' rows, half of the largest listed cases' (three arrays of that in the gradient)
    T = _log(rng, 1, max(1, min(65536, (1 << 30) // (k * D * BYTES[dtype]))))
    return _ex(kind, None, T, k, E, D, dtype, pitch=rng.choice((0, 0, rng.randint(1, 32))),
               none=rng.choice((0.0, 0.05, 0.3)))


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 6007 + 29)


def _matrix(rows, c, values=None):
    """rows x D of the case's type and pitch, zeros or the given values."""
    buf = torch.zeros((rows, c["D"] + c["pitch"]), dtype=DTYPES[c["dtype"]], device="cuda")
    m = buf[:, :c["D"]]
    if values is not None:
        m.copy_(values)
    return m


def _choices(c, g):
    """k different experts of each query, some liked more; -1 where a query has no choice."""
    T, E = c["T"], c["E"]
    lean = torch.randn((E,), generator=g, device="cuda")
    u = torch.rand((T, E), generator=g, device="cuda").clamp_min(1e-20)
    idx = torch.topk(lean - torch.log(-torch.log(u)), c["k"], dim=1).indices.to(I32)
    w = torch.rand((T, c["k"]), generator=g, device="cuda") + 0.05
    w /= w.sum(1, keepdim=True)
    if c["none"]:
        off = torch.rand((T,), generator=g, device="cuda") < c["none"]
        idx[off], w[off] = -1, 0.0
    return idx, w


def _vocabulary(c, g):
    """Hidden states that point to a token, more or less, and the vocabulary's weight."""
    T, V, D = c["T"], c["V"], c["D"]
    w = _matrix(V, c, torch.randn((V, D), generator=g, device="cuda") * (1.5 / math.sqrt(D)))
    t = torch.randint(0, V, (T,), generator=g, device="cuda")
    h = torch.randn((T, D), generator=g, device="cuda")
    h += (3.5 * torch.rand((T, 1), generator=g, device="cuda")) * w[t].float()
    h = _matrix(T, c, h)
    # the given tokens: mostly those, some any; a few positions hold no token
    pick = torch.rand((T,), generator=g, device="cuda")
    t = torch.where(pick < 0.75, t, torch.randint(0, V, (T,), generator=g, device="cuda"))
    if T > 8:
        t = torch.where(pick > 0.97, torch.full_like(t, -1), t)
    return h, w, t


def prepare(case, seed):
    c, g = case, _gen(seed)
    T, D = c["T"], c["D"]
    dev = dict(device="cuda")
    new = lambda *s: torch.empty(s, **dev)
    if c["kind"].startswith("hidden"):
        h, w, t = _vocabulary(c, g)
        st = dict(c=c, h=h, w=w, t=t)
        if c["kind"] == "hidden":
            return dict(st, logprob=new(T), entropy=new(T), lse=new(T))
        lp = _plain_hidden(st)  # what the forward pass left for the backward pass
        return dict(st, lse=lp["lse"], ent=lp["entropy"],
                    glp=torch.randn((T,), generator=g, **dev) / T,
                    gent=0.05 * torch.randn((T,), generator=g, **dev) / T if c["ent"] else None,
                    dh=torch.empty((T, D), dtype=h.dtype, **dev),
                    dw=torch.empty((c["V"], D), dtype=h.dtype, **dev))
    N = T * c["k"]
    idx, weight = _choices(c, g)
    st = dict(c=c, idx=idx, weight=weight)
    if c["kind"] == "sort":
        ints = lambda *s: torch.empty(s, dtype=I32, **dev)
        return dict(st, x=_matrix(T, c, torch.randn((T, D), generator=g, **dev)), rows=_matrix(N, c),
                    offsets=ints(c["E"] + 1), source=ints(N), place=ints(T, c["k"]))
    st["place"] = _plain_order(c, idx)[2]
    randn = lambda rows: _matrix(rows, c, torch.randn((rows, D), generator=g, **dev))
    if c["kind"] == "combine":
        return dict(st, rows=randn(N), out=_matrix(T, c))
    return dict(st, g_out=randn(T), rows=randn(N), g_rows=_matrix(N, c), g_weight=new(T, c["k"]),
                g_read=randn(N), dx=_matrix(T, c))


# ---------------------------------------------------------------- plain forms
def _plain_order(c, idx):
    """(offsets, source, place) of the choices in the order of their experts."""
    E, e = c["E"], idx.reshape(-1).long()
    key = torch.where(e >= 0, e, torch.full_like(e, E))
    order = torch.sort(key, stable=True).indices
    offsets = torch.searchsorted(key[order].contiguous(), torch.arange(E + 1, device=e.device))
    at = torch.arange(e.numel(), device=e.device)
    valid = at < offsets[E]
    source = torch.where(valid, order, torch.full_like(order, -1))
    place = torch.empty_like(order).scatter_(0, order, torch.where(valid, at, torch.full_like(at, -1)))
    return offsets.to(I32), source.to(I32), place.to(I32).view(idx.shape)


def _plain_sort(st):
    c = st["c"]
    offsets, source, place = _plain_order(c, st["idx"])
    s = source.long()
    rows = st["x"][s.clamp_min(0) // c["k"]]
    rows = torch.where((s >= 0)[:, None], rows, torch.zeros_like(rows))
    return dict(offsets=offsets, source=source, place=place, rows=rows)


def _taken(rows, place):
    """T x k x D: the row of each choice in 32 bits, 0 where there is none."""
    v = rows[place.long().clamp_min(0)].float()
    return torch.where((place >= 0)[:, :, None], v, torch.zeros_like(v))


def _plain_combine(st):
    v = _taken(st["rows"], st["place"])
    return dict(out=(v * st["weight"][:, :, None]).sum(1).to(st["rows"].dtype))


def _plain_expert_grad(st):
    place, go = st["place"], st["g_out"].float()[:, None]
    dt = st["rows"].dtype
    on = (place >= 0)[:, :, None]
    g_weight = (_taken(st["rows"], place) * go).sum(2)
    v = torch.where(on, go * st["weight"][:, :, None], torch.zeros_like(go)).to(dt)
    N = place.numel()
    at = torch.where(place >= 0, place.long(), torch.full_like(place, N, dtype=I64)).reshape(-1)
    g_rows = torch.zeros((N + 1, v.shape[2]), dtype=dt, device=v.device)
    g_rows.index_copy_(0, at, v.reshape(N, -1))
    return dict(g_rows=g_rows[:N], g_weight=g_weight, dx=_taken(st["g_read"], place).sum(1).to(dt))


def _plain_logits(st):
    return (st["h"].float() @ st["w"].float().t()) * st["c"]["scale"]


def _plain_hidden(st):
    z, t = _plain_logits(st), st["t"]
    at = torch.gather(z, 1, t.clamp_min(0)[:, None])
    m = z.amax(1, keepdim=True)
    z -= m
    e = torch.exp(z)
    s = e.sum(1, keepdim=True)
    ls = torch.log(s)
    entropy = (ls - e.mul_(z).sum(1, keepdim=True) / s)[:, 0]
    logprob = torch.where(t >= 0, (at - m - ls)[:, 0], torch.zeros_like(entropy))
    return dict(logprob=logprob, entropy=entropy, lse=(m + ls)[:, 0])


def _plain_hidden_grad(st):
    c, t = st["c"], st["t"]
    g = torch.where(t >= 0, st["glp"], torch.zeros_like(st["glp"]))[:, None]
    lp = _plain_logits(st).sub_(st["lse"][:, None])
    p = torch.exp(lp)
    if st["gent"] is not None:
        d = p * (-g - st["gent"][:, None] * (lp + st["ent"][:, None]))
    else:
        d = p.mul_(-g)
    d.scatter_add_(1, t.clamp_min(0)[:, None], g)
    d *= c["scale"]
    return dict(dhidden=(d @ st["w"].float()).to(st["h"].dtype),
                dweight=(d.t() @ st["h"].float()).to(st["w"].dtype))


# ---------------------------------------------------------------- the library
def _workspace(st, bt, grad):
    if "ws" not in st:  # kept, as a program's loop keeps it
        n = bt.boute_hidden_logprobs_workspace(st["h"], st["w"], grad)
        st["ws"] = torch.empty((n,), dtype=torch.uint8, device="cuda")
    return st["ws"]


def _own(st):
    from paper_2602_10729_gb300 import boute as bt
    c, kind = st["c"], st["c"]["kind"]
    if kind == "sort":
        bt.boute_expert_sort(st["idx"], st["offsets"], st["source"], st["place"])
        bt.boute_expert_dispatch(st["x"], st["place"], st["rows"])
        return dict(offsets=st["offsets"], source=st["source"], place=st["place"], rows=st["rows"])
    if kind == "combine":
        bt.boute_expert_combine(st["rows"], st["place"], st["weight"], st["out"])
        return dict(out=st["out"])
    if kind == "expert_grad":
        bt.boute_expert_combine_grad(st["g_out"], st["rows"], st["place"], st["weight"],
                                     st["g_rows"], st["g_weight"])
        bt.boute_expert_dispatch_grad(st["g_read"], st["place"], st["dx"])
        return dict(g_rows=st["g_rows"], g_weight=st["g_weight"], dx=st["dx"])
    if kind == "hidden":
        bt.boute_hidden_logprobs(st["h"], st["w"], st["t"], c["scale"], st["logprob"],
                                 st["entropy"], st["lse"], _workspace(st, bt, False))
        return dict(logprob=st["logprob"], entropy=st["entropy"], lse=st["lse"])
    bt.boute_hidden_logprobs_grad(st["h"], st["w"], st["t"], c["scale"], st["lse"], st["ent"],
                                  st["glp"], st["gent"], st["dh"], st["dw"],
                                  _workspace(st, bt, True))
    return dict(dhidden=st["dh"], dweight=st["dw"])


PLAIN = dict(sort=_plain_sort, combine=_plain_combine, expert_grad=_plain_expert_grad,
             hidden=_plain_hidden, hidden_grad=_plain_hidden_grad)


def run(state):
    return _own(state) if own else PLAIN[state["c"]["kind"]](state)


def work(case):
    """Each input read once, each output written once; a floating operation per step of the formulas."""
    c, kind = case, case["kind"]
    T, D, b = c["T"], c["D"], BYTES[c["dtype"]]
    if kind.startswith("hidden"):
        V = c["V"]
        if kind == "hidden":
            return dict(bytes=(T + V) * D * b + 20 * T, flops=2.0 * T * V * D + 6.0 * T * V)
        return dict(bytes=2 * (T + V) * D * b + 24 * T, flops=6.0 * T * V * D + 8.0 * T * V)
    N = T * c["k"]
    n = round(N * (1.0 - c["none"]))  # the choices that there are
    if kind == "sort":
        return dict(bytes=12 * N + 4 * c["E"] + (T + n) * D * b, flops=0.0)
    if kind == "combine":
        return dict(bytes=8 * N + (T + n) * D * b, flops=2.0 * n * D)
    return dict(bytes=12 * N + (2 * T + 3 * n) * D * b, flops=4.0 * n * D)


# ---------------------------------------------------------------- 64 bits
def _exact_sort(st):
    c, idx = st["c"], st["idx"].cpu()
    x = st["x"].double()
    flat = idx.reshape(-1)
    order = torch.cat([(flat == e).nonzero()[:, 0] for e in range(c["E"])])
    rows = torch.zeros((flat.numel(), c["D"]), dtype=F64, device="cuda")
    rows[:order.numel()] = x[(order // c["k"]).cuda()]
    return dict(offsets=None, source=None, place=None, rows=rows)


def _exact_combine(st):
    out = torch.zeros((st["c"]["T"], st["c"]["D"]), dtype=F64, device="cuda")
    for i in range(st["c"]["k"]):
        p, w = st["place"][:, i].long(), st["weight"][:, i].double()
        on = p >= 0
        out[on] += w[on, None] * st["rows"][p[on]].double()
    return dict(out=out)


def _exact_expert_grad(st):
    c = st["c"]
    go = st["g_out"].double()
    g_rows = torch.zeros((c["T"] * c["k"], c["D"]), dtype=F64, device="cuda")
    g_weight = torch.zeros((c["T"], c["k"]), dtype=F64, device="cuda")
    dx = torch.zeros_like(go)
    for i in range(c["k"]):
        p, w = st["place"][:, i].long(), st["weight"][:, i].double()
        on = p >= 0
        g_rows[p[on]] = w[on, None] * go[on]
        g_weight[on, i] = (go[on] * st["rows"][p[on]].double()).sum(1)
        dx[on] += st["g_read"][p[on]].double()
    return dict(g_rows=g_rows, g_weight=g_weight, dx=dx)


def _exact_hidden(st):
    c, out, w = st["c"], [], st["w"].double()
    scale = torch.tensor(c["scale"], dtype=F32).double().item()
    for h, t in zip(st["h"].split(512), st["t"].split(512)):
        z = scale * (h.double() @ w.t())
        lse = torch.logsumexp(z, 1)
        z -= lse[:, None]
        at = torch.take_along_dim(z, t.clamp_min(0)[:, None], 1)[:, 0]
        out.append((at.masked_fill(t < 0, 0.0), -(z * torch.exp(z)).sum(1), lse))
    return dict(zip(("logprob", "entropy", "lse"), (torch.cat(v) for v in zip(*out))))


def _exact_hidden_grad(st):
    c, w = st["c"], st["w"].double()
    scale = torch.tensor(c["scale"], dtype=F32).double().item()
    dw, dh = torch.zeros_like(w), []
    for r in range(0, c["T"], 512):
        r = slice(r, min(c["T"], r + 512))
        h, t = st["h"][r].double(), st["t"][r]
        lp = scale * (h @ w.t()) - st["lse"][r].double()[:, None]
        p = torch.exp(lp)
        g = st["glp"][r].double().masked_fill(t < 0, 0.0)
        d = -g[:, None] * p
        if st["gent"] is not None:
            d -= st["gent"][r].double()[:, None] * p * (lp + st["ent"][r].double()[:, None])
        at = (t >= 0).nonzero()[:, 0]
        d[at, t[at]] += g[at]
        d *= scale
        dh.append(d @ w)
        dw += d.t() @ h
    return dict(dhidden=torch.cat(dh), dweight=dw)


EXACT = dict(sort=_exact_sort, combine=_exact_combine, expert_grad=_exact_expert_grad,
             hidden=_exact_hidden, hidden_grad=_exact_hidden_grad)


def exact(case, seed):
    return EXACT[case["kind"]](prepare(case, seed))
