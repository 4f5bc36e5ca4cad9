"""The scored router, its gradient and the int8 experts as measurable cases.

``op`` names the operator of a case:

* "route": routing by scores.  Z = X W_r + bias in 32 bits, the score s of an
  expert is sigmoid(Z) or the softmax of Z, experts are chosen by s + balance
  (held in 64 bits) within the best groups of experts, and weighted by
  scale * s, renormalised over the chosen ones or not.
* "route_grad": the gradient of a loss with respect to the router's logits from
  its gradient with respect to the chosen experts' weights.
* "experts": the expert FFNs of a planned batch in 8-bit integers, one scale
  per token (activations) and per channel (weights).

Field names follow the C ABI: T tokens, d hidden, E local experts, k routes per
token, f routed intermediate width, fs shared-expert width (0: none).
``balance`` is the std of the selection bias, ``bias`` that of the bias of the
logits (0: none), ``off`` the number of experts whose logits are masked,
``hot`` the share of tokens that take expert 0, ``skew`` the std of the
experts' popularity.
"""
import math

import torch

own = False

DEV = "cuda"
BF, F32, F64, I32, I64 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64
MASKED = -1e38   # a logit or selection bias below this takes its expert out


def _route(name, op, T, d, E, k, score, G=1, topg=1, pair=False, norm=True, scale=1.0,
           balance=0.0, bias=0.0, off=0):
    return dict(name=name, op=op, T=T, d=d, E=E, k=k, score=score, groups=G, top_groups=topg,
                group_pair=pair, renormalise=norm, scale=scale, balance=balance, bias=bias, off=off)


def _experts(name, T, d, E, k, f, fs=0, skew=0.0, hot=0.0):
    return dict(name=name, op="experts", T=T, d=d, E=E, k=k, f=f, fs=fs, skew=skew, hot=hot)


def listed():
    return [
        # decoding one sequence with the router of a layer of 256 experts in 8
        # groups, four of them kept: latency
        _route("route 1, 256 in 8 groups", "route", 1, 7168, 256, 8, "sigmoid", 8, 4, True,
               scale=2.5, balance=0.1),
        # prefill of a ragged batch with the same router
        _route("route 4099, 256 in 8 groups", "route", 4099, 7168, 256, 8, "sigmoid", 8, 4, True,
               scale=2.5, balance=0.1),
        # a training batch routed by softmax scores that are not renormalised
        _route("route 16384, 128 softmax", "route", 16384, 2048, 128, 8, "softmax", norm=False,
               balance=0.01, bias=0.5),
        # the router's gradient in a training step, renormalised sigmoid
        # scores: k of a row's E logits have one
        _route("gradient 16384, 256 sigmoid", "route_grad", 16384, 7168, 256, 8, "sigmoid", 8, 4,
               True, scale=2.5, balance=0.1),
        # softmax scores without renormalisation: every logit has a gradient
        _route("gradient 6001, 96 softmax", "route_grad", 6001, 2048, 96, 6, "softmax",
               norm=False, balance=0.01),
        # decoding one sequence: the reached experts' weights are streamed
        _experts("int8 decode 1, 128 experts", 1, 2048, 128, 8, 768, skew=0.5),
        # decoding a small batch: most experts see a few rows
        _experts("int8 decode 16, 32 experts", 16, 4096, 32, 8, 1536, hot=0.1),
        # every token takes every local expert and the shared one
        _experts("int8 decode 61, dense + shared", 61, 7168, 8, 8, 2048, fs=2048),
        # prefill of one short prompt
        _experts("int8 prefill 1000, 32 experts", 1000, 4096, 32, 8, 1536, hot=0.1),
        # prefill over many small experts with skewed load
        _experts("int8 prefill 8192, 128 experts", 8192, 2048, 128, 8, 768, skew=0.5),
        # a ragged batch on the dense share with a shared expert
        _experts("int8 prefill 4099, dense + shared", 4099, 7168, 8, 8, 2048, fs=2048),
        # a large batch with one hot expert
        _experts("int8 prefill 16384, 32 experts", 16384, 4096, 32, 8, 1536, hot=0.1),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    """1 to 16384 tokens, hidden sizes to 7168, 8 to 256 experts (counts that
    are no power of two among them), every kind of score and group."""
    if rng.random() < 0.5:
        most = max(work(c)["flops"] for c in listed() if c["op"] == "experts")
        while True:
            E = rng.choice([8, 12, 16, 24, 32, 48, 64, 96, 128, 200])
            k = min(rng.choice([1, 2, 4, 6, 8]), E)
            c = _experts("", _log_int(rng, 1, 16384), 256 * rng.randint(1, 28), E, k,
                         256 * rng.randint(1, 8), rng.choice([0, 0, 0, 1, 2]) * 1024,
                         rng.choice([0.0, 0.5]), rng.choice([0.0, 0.0, 0.1]))
            if work(c)["flops"] <= most and 3 * E * c["d"] * c["f"] <= 2_000_000_000:
                break
    else:
        E = rng.choice([8, 20, 32, 60, 64, 96, 128, 160, 256])
        G = rng.choice([g for g in (1, 1, 2, 4, 5, 8) if E % g == 0])
        k = rng.choice([n for n in (1, 2, 4, 6, 8, 16) if n <= E])
        topg = rng.randint(-(-k * G // E), G)
        op = rng.choice(["route", "route", "route_grad"])
        T = _log_int(rng, 1 if op == "route" else 64, 16384)
        norm = rng.random() < 0.6 and (k > 1 or op == "route")   # one renormalised weight is constant
        c = _route("", op, T, 256 * rng.randint(1, 28), E, k, rng.choice(["sigmoid", "softmax"]), G,
                   topg, rng.random() < 0.5, norm, rng.choice([1.0, 2.5]),
                   rng.choice([0.0, 0.01, 0.1]), rng.choice([0.0, 0.5]), rng.choice([0, 0, 2]))
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _normal(g, shape, std, dtype=F32):
    return torch.empty(shape, dtype=F32, device=DEV).normal_(0.0, std, generator=g).to(dtype)


def _quantised(W):
    """A weight [E, n, K]: int8 codes and one fp32 scale per channel n."""
    s = W.abs().amax(-1) / torch.full((), 127.0, device=DEV)
    return torch.round(W / s[..., None]).to(torch.int8), s


def _prepare_route(c, g):
    T, d, E, k = c["T"], c["d"], c["E"], c["k"]
    # Normal values on a grid (X on multiples of 1/16 up to 6, W_r of std
    # 1/sqrt(d) on 8 bits): every partial sum of a logit is then exact in 32
    # bits, so the logits, and with them the chosen experts, do not depend on
    # the order of summation.
    X = (_normal(g, (T, d), 16.0).round_().clamp_(-96, 96) / 16).to(BF)
    unit = 2.0 ** math.floor(math.log2(d ** -0.5 / 24))
    W_r = (_normal(g, (d, E), d ** -0.5 / unit).round_().clamp_(-240, 240) * unit).to(BF)
    bias = _normal(g, (E,), c["bias"]) if c["bias"] or c["off"] else None
    if c["off"]:
        bias[torch.randperm(E, device=DEV, generator=g)[:c["off"]]] = -math.inf
    s = dict(c=c, X=X, W_r=W_r, bias=bias,
             balance=_normal(g, (E,), c["balance"]) if c["balance"] else None)
    if c["op"] == "route_grad":
        s["logits"] = _normal(g, (T, E), 1.0)
        if bias is not None:
            s["logits"] += bias
        s["topk_idx"] = _choose(c, s["logits"], s["balance"])[0]
        s["dw"] = _normal(g, (T, k), 1.0)
        del s["X"], s["W_r"]
    return s


def _prepare_experts(c, g):
    T, d, E, k, f, fs = (c[n] for n in ("T", "d", "E", "k", "f", "fs"))
    X = _normal(g, (T, d), 1.0, BF)
    # k different experts per token, popular ones more often
    score = torch.empty((T, E), device=DEV).exponential_(generator=g).log_().neg_()
    if c["skew"]:
        score += _normal(g, (E,), c["skew"])
    n_hot = int(c["hot"] * T)
    if n_hot:
        score[torch.randperm(T, device=DEV, generator=g)[:n_hot], 0] = math.inf
    idx = score.argsort(dim=1, descending=True)[:, :k].sort(dim=1).values
    w = torch.softmax(_normal(g, (T, k), 1.0), dim=1)
    flat = idx.reshape(-1)
    perm = flat.argsort(stable=True)
    counts = torch.bincount(flat, minlength=E)
    offsets = torch.zeros(E + 1, dtype=I64, device=DEV)
    offsets[1:] = counts.cumsum(0)
    pos = torch.empty_like(perm)
    pos[perm] = torch.arange(T * k, device=DEV)
    s = dict(c=c, X=X, topk_idx=idx.to(I32), topk_w=w, counts=counts.to(I32), offsets=offsets.to(I32),
             perm=perm.to(I32), route_pos=pos.to(I32), most=int(counts.max()))
    for name, n, rows, K in (("g", E, f, d), ("u", E, f, d), ("d", E, d, f),
                             ("gs", 1, fs, d), ("us", 1, fs, d), ("ds", 1, d, fs)):
        if rows and K:
            s["W" + name], s["S" + name] = _quantised(_normal(g, (n, rows, K), K ** -0.5, BF).float())
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    return _prepare_experts(case, g) if case["op"] == "experts" else _prepare_route(case, g)


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------

def _scores(c, z):
    """Scores of the logits z, in their type; masked logits score 0."""
    live = z >= MASKED
    z = torch.where(live, z, -math.inf)
    if c["score"] == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-z)), live
    e = torch.exp(z - z.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True), live


def _choose(c, logits, balance):
    """Chosen experts in ascending id, all scores and who is not masked."""
    T, E = logits.shape
    G, k = c["groups"], c["k"]
    s, live = _scores(c, logits.double())
    v = s if balance is None else s + balance.double()
    v = torch.where(live, v, -math.inf)
    kept = torch.ones_like(live)
    if G > 1:
        best = v.view(T, G, E // G).sort(dim=2, descending=True).values
        gs = best[:, :, 0]
        if c["group_pair"] and E // G > 1:
            gs = gs + torch.where(best[:, :, 1] == -math.inf, 0.0, best[:, :, 1])
        order = gs.sort(dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        kept = torch.zeros(T, G, dtype=torch.bool, device=logits.device).scatter_(1, order, True)
        kept = kept[:, :, None].expand(T, G, E // G).reshape(T, E)
    order = v.sort(dim=1, descending=True, stable=True).indices
    out = (~kept).gather(1, order).to(torch.int8)
    order = order.gather(1, out.sort(dim=1, stable=True).indices)
    idx = order[:, :k].sort(dim=1).values
    return idx.to(I32), s, live


def _weights(c, s, live, idx):
    w = torch.where(live, s, 0.0).gather(1, idx.long())
    if c["renormalise"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, 0.0)
    return c["scale"] * w


def _plain_route(st):
    c = st["c"]
    logits = st["X"].float() @ st["W_r"].float()
    if st["bias"] is not None:
        logits = logits + st["bias"]
    idx, s, live = _choose(c, logits, st["balance"])
    return dict(logits=logits, topk_idx=idx, topk_w=_weights(c, s, live, idx).float())


def _plain_route_grad(st):
    c, idx, dw = st["c"], st["topk_idx"].long(), st["dw"]
    s, live = _scores(c, st["logits"])
    w = _weights(c, s, live, idx)
    if c["renormalise"]:
        dw = dw - (dw * w).sum(1, keepdim=True) / c["scale"]
    g = w * dw
    if c["score"] == "sigmoid":
        g = g / (1.0 + torch.exp(st["logits"].gather(1, idx)))
    dZ = torch.zeros_like(st["logits"]).scatter_(1, idx, g)
    if c["score"] == "softmax" and not c["renormalise"]:
        dZ = dZ - s * g.sum(1, keepdim=True)
    return dict(dZ=dZ)


def _quantise_rows(x):
    s = x.abs().amax(-1, keepdim=True) / torch.full((), 127.0, device=x.device)
    return torch.where(s > 0, torch.round(x / s), 0.0), s


def _ffn(xq, xs, W, S):
    """[n, rows, d] codes and [n, rows, 1] scales through n experts."""
    up = [torch.bmm(xq, W[i].mT.contiguous().float()) * xs * S[i][:, None, :] for i in (0, 1)]
    h = up[0] / (1.0 + torch.exp(-up[0])) * up[1]
    hq, hs = _quantise_rows(h)
    return torch.bmm(hq, W[2].mT.contiguous().float()) * hs * S[2][:, None, :]


def _plain_experts(st):
    c = st["c"]
    T, d, E, k, R = c["T"], c["d"], c["E"], c["k"], c["T"] * c["k"]
    xq, xs = _quantise_rows(st["X"].float())
    perm, offsets = st["perm"].long(), st["offsets"].long()
    p = torch.arange(R, device=DEV)
    e = st["topk_idx"].reshape(-1)[perm].long()
    W, S = [st["Wg"], st["Wu"], st["Wd"]], [st["Sg"], st["Su"], st["Sd"]]
    if R <= E:       # few routes: each with its expert's weights
        y = _ffn(xq[perm // k][:, None], xs[perm // k][:, None], [w[e] for w in W], [s[e] for s in S])[:, 0]
    else:            # each expert's rows, padded to the longest
        at = e * st["most"] + p - offsets[e]
        xp = torch.zeros(E * st["most"], d, device=DEV)
        sp = torch.zeros(E * st["most"], 1, device=DEV)
        xp[at], sp[at] = xq[perm // k], xs[perm // k]
        y = _ffn(xp.view(E, -1, d), sp.view(E, -1, 1), W, S).view(-1, d)[at]
    y = y[st["route_pos"].long()].view(T, k, d)
    Y = (st["topk_w"][:, :, None] * y).sum(1)
    if c["fs"]:
        Y = Y + _ffn(xq[None], xs[None], [st[n] for n in ("Wgs", "Wus", "Wds")],
                     [st[n] for n in ("Sgs", "Sus", "Sds")])[0]
    return dict(Y=Y.to(BF))


# ---------------------------------------------------------------------------
# The framework's calls
# ---------------------------------------------------------------------------

class _Layer:
    """Outputs, workspace and argument structures that a program keeps."""

    def __init__(self, st):
        from paper_2609_36070_amd import binding as B
        self.B, c = B, st["c"]
        T, E, k = c["T"], c["E"], c["k"]
        self.shape = B.make_shape(T, c["d"], E, k, c.get("f", 256), c.get("fs", 0))
        if c["op"] == "experts":
            self.plan = B.plan_bufs(*(st[n] for n in ("counts", "offsets", "perm", "route_pos")))
            self.weights = B.int_weights_struct(*(st.get(a + n) for a in ("W", "S") for n in ("g", "u", "d")),
                                               *(st.get(a + n) for a in ("W", "S") for n in ("gs", "us", "ds")))
            self.ws = torch.empty(B.moe_int_workspace_bytes(self.shape), dtype=torch.uint8, device=DEV)
            self.Y = torch.empty(T, c["d"], dtype=BF, device=DEV)
            return
        self.routing = B.routing(c["score"], groups=c["groups"], top_groups=c["top_groups"],
                                 group_score="pair" if c["group_pair"] else "max",
                                 renormalise=c["renormalise"], scale=c["scale"])
        if c["op"] == "route":
            self.ws = torch.empty(B.moe_workspace_bytes(self.shape, False), dtype=torch.uint8, device=DEV)
            self.logits = torch.empty(T, E, device=DEV)
            self.topk_idx = torch.empty(T, k, dtype=I32, device=DEV)
            self.topk_w = torch.empty(T, k, device=DEV)
        else:
            self.dZ = torch.empty(T, E, device=DEV)


def _own(st):
    if "layer" not in st:
        st["layer"] = _Layer(st)
    m = st["layer"]
    op = st["c"]["op"]
    if op == "route":
        m.B.moe_route_scored(m.shape, m.routing, st["X"], st["W_r"], st["bias"], st["balance"], m.logits,
                             m.topk_idx, m.topk_w, m.ws)
        return dict(logits=m.logits, topk_idx=m.topk_idx, topk_w=m.topk_w)
    if op == "route_grad":
        m.B.moe_score_backward(m.shape, m.routing, st["logits"], st["balance"], st["topk_idx"], st["dw"], m.dZ)
        return dict(dZ=m.dZ)
    m.B.moe_forward_int(m.shape, st["X"], m.weights, st["topk_idx"], st["topk_w"], m.plan, m.Y, m.ws)
    return dict(Y=m.Y)


def run(state):
    if own:
        return _own(state)
    plain = {"route": _plain_route, "route_grad": _plain_route_grad, "experts": _plain_experts}
    return plain[state["c"]["op"]](state)


def work(case):
    T, d, E, k = case["T"], case["d"], case["E"], case["k"]
    if case["op"] == "experts":
        reached = E * (1.0 - (1.0 - k / E) ** T)
        return {"bytes": 3 * d * (reached * case["f"] + case["fs"]) + 4 * T * d + 8 * T * k,
                "flops": 6.0 * T * (k * case["f"] + case["fs"]) * d}
    if case["op"] == "route":
        return {"bytes": 2 * T * d + 2 * d * E + 4 * T * E + 8 * T * k, "flops": 2.0 * T * d * E}
    dense = case["score"] == "softmax" and not case["renormalise"]
    return {"bytes": 4 * T * E * (2 if dense else 1) + (8 if dense else 12) * T * k,
            "flops": (8.0 * E if dense else 16.0 * k) * T}


# ---------------------------------------------------------------------------
# From the definitions, in 64 bits
# ---------------------------------------------------------------------------

def _exact_scores(c, z):
    dead = ~(z > MASKED)
    z = z.masked_fill(dead, -math.inf)
    logp = -torch.logaddexp(torch.zeros_like(z), -z) if c["score"] == "sigmoid" else \
        z - torch.logsumexp(z, 1, keepdim=True)
    return logp.exp().masked_fill(dead, 0.0), dead


def _exact_ffn(x, Wg, Wu, Wd, Sg, Su, Sd):
    def rows(v):
        s = (v.abs().max(1, keepdim=True).values / 127).float().double()
        # a code is the quotient rounded to 32 bits, then to an integer, ties to even
        return torch.round((v / s.clamp_min(1e-300)).float()).double(), s
    q, s = rows(x)
    a, b = s * (q @ Wg.double().T) * Sg, s * (q @ Wu.double().T) * Su
    q, s = rows(a * torch.sigmoid(a) * b)
    return s * (q @ Wd.double().T) * Sd


def exact(case, seed):
    c, st = case, prepare(case, seed)
    T, E, k = c["T"], c["E"], c["k"]
    if c["op"] == "experts":
        X, Y = st["X"].double(), torch.zeros(T, c["d"], dtype=F64, device=DEV)
        for e in range(E):
            t, slot = (st["topk_idx"] == e).nonzero(as_tuple=True)
            if len(t):
                y = _exact_ffn(X[t], st["Wg"][e], st["Wu"][e], st["Wd"][e], st["Sg"][e].double(),
                               st["Su"][e].double(), st["Sd"][e].double())
                Y[t] += st["topk_w"][t, slot].double()[:, None] * y
        if c["fs"]:
            Y += _exact_ffn(X, st["Wgs"][0], st["Wus"][0], st["Wds"][0], st["Sgs"][0].double(),
                            st["Sus"][0].double(), st["Sds"][0].double())
        return dict(Y=Y)
    if c["op"] == "route":
        z = st["X"].double() @ st["W_r"].double()
        if st["bias"] is not None:   # the logits are 32-bit values
            z = (z.float() + st["bias"]).double()
        p, dead = _exact_scores(c, z)
        v = p if st["balance"] is None else p + st["balance"].double()
        v = v.masked_fill(dead, -math.inf)
        G, n = c["groups"], E // c["groups"]
        allowed = torch.ones(T, G, dtype=torch.bool, device=DEV)
        if G > 1:
            gv = v.view(T, G, n)
            first = gv.max(2)
            gs = first.values.clone()
            if c["group_pair"] and n > 1:
                second = gv.scatter(2, first.indices[..., None], -math.inf).max(2).values
                gs += second.masked_fill(second == -math.inf, 0.0)
            ids = torch.arange(G, device=DEV)
            better = (gs[:, None, :] > gs[:, :, None]) | \
                ((gs[:, None, :] == gs[:, :, None]) & (ids[None, None, :] < ids[None, :, None]))
            allowed = better.sum(2) < c["top_groups"]
        free = allowed.repeat_interleave(n, dim=1)
        chosen = torch.zeros(T, E, dtype=torch.bool, device=DEV)
        for _ in range(k):           # the best one left; argmax of a 0/1 row is its first 1
            left = free & ~chosen
            top = torch.where(left, v, -math.inf).max(1, keepdim=True).values
            first = (left & (v == top)).to(torch.int8).argmax(1, keepdim=True)
            chosen.scatter_(1, first, True)
        idx = chosen.nonzero()[:, 1].view(T, k)
        w = p.gather(1, idx)
        if c["renormalise"]:
            w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
        return dict(logits=z, topk_idx=idx.to(I32), topk_w=c["scale"] * w)
    z = st["logits"].double().requires_grad_()
    p, _ = _exact_scores(c, z)
    w = p.gather(1, st["topk_idx"].long())
    if c["renormalise"]:
        w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
    (c["scale"] * w * st["dw"].double()).sum().backward()
    return dict(dZ=z.grad)
