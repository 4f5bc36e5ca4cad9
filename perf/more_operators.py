"""What stands around the layer and the whole layer for a few tokens, as measurable cases.

``op`` names the operator of a case:

* "join": a block's output y goes back into the residual stream x: an optional
  norm of y, dropout, a gate per channel and per token and a scale, then the sum
  r, and the norm of r that the next block reads, h.  ``block`` is false for the
  norm before the first block alone (no y: h is the norm of x).
* "join_grad": its gradient: of x, y, the norms' weights and biases and the gates.
* "few": a whole layer for a few tokens: router, selection, experts, sum.

Dropout keeps an element by 16 bits of Philox4x32-10 (Salmon, Moraes, Dror, Shaw,
"Parallel random numbers: as easy as 1, 2, 3", 2011): the key is the seed, the
counter of the 8 elements 8 j .. 8 j + 7 of row t is (j, t, offset), its four
words hold their 16 bits in order, lower halves first; an element is kept where
they are at least drop * 2^16, and divided by the share that is kept.

Field names follow the C ABI: T tokens, d hidden, E local experts, k routes per
token, f routed intermediate width, fs shared-expert width (0: none).  ``stream``
is the residual stream's type.
"""
import math

import torch

own = False

DEV = "cuda"
BF, F32, F64, I32, I64 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64
EPS = 1e-6
MASKED = -1e38   # a logit or selection bias below this takes its expert out


def _join(name, op, T, d, stream="bf16", y_norm="none", r_norm="rms", gate=False, token_gate=False,
          scale=1.0, drop=0.0, block=True, train=True):
    return dict(name=name, op=op, T=T, d=d, stream=stream, y_norm=y_norm, r_norm=r_norm, gate=gate,
                token_gate=token_gate, scale=scale, drop=drop, block=block, train=train)


def _few(name, T, d, E, k, f, fs=0, score="softmax", G=1, topg=1, pair=False, norm=True, scale=1.0,
         balance=0.0, bias=0.0):
    return dict(name=name, op="few", T=T, d=d, E=E, k=k, f=f, fs=fs, score=score, groups=G, top_groups=topg,
                group_pair=pair, renormalise=norm, scale=scale, balance=balance, bias=bias)


def listed():
    return [
        # decoding one sequence: between two layers, norms on either side
        _join("join 1 x 7168", "join", 1, 7168, y_norm="rms", train=False),
        # the norm before the first block of a ragged prefill batch
        _join("norm 4099 x 4096", "join", 4099, 4096, block=False, train=False),
        # a training batch: the residual stream in fp32, dropout and layer norms
        _join("join 6001 x 2048, fp32", "join", 6001, 2048, "f32", "none", "layer", gate=True, drop=0.1),
        # a large training batch with norms on either side, a gate per channel and dropout
        _join("join 16384 x 7168", "join", 16384, 7168, "bf16", "rms", "rms", gate=True, scale=0.5, drop=0.1),
        # gradients of a short micro-batch
        _join("gradient 500 x 1000", "join_grad", 500, 1000, "f32", "layer", "layer", token_gate=True),
        _join("gradient 6001 x 2048, fp32", "join_grad", 6001, 2048, "f32", "none", "layer", gate=True, drop=0.1),
        # of the large training batch
        _join("gradient 16384 x 7168", "join_grad", 16384, 7168, "bf16", "rms", "rms", gate=True, scale=0.5,
              drop=0.1),
        # decoding one sequence with many small experts: latency
        _few("few 1, 128 experts", 1, 2048, 128, 8, 768),
        # four sequences, 256 experts in groups, a shared expert
        _few("few 4, 256 in 8 groups + shared", 4, 7168, 256, 8, 512, 512, "sigmoid", 8, 4, True, scale=2.5,
             balance=0.1),
        # every token takes every local expert and the shared one
        _few("few 7, dense + shared", 7, 7168, 8, 8, 2048, 2048),
        # the largest batch of the path, most experts reached
        _few("few 16, 32 experts", 16, 4096, 32, 8, 1536),
        # two tokens to few experts, one of them each
        _few("few 2, 8 experts, top 1", 2, 1024, 8, 1, 512, 0, "sigmoid", norm=False, bias=0.5),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    """Rows of 8 to 8192 values, 1 to 16384 of them, every kind of norm; layers
    for 1 to 16 tokens, 4 to 256 experts (counts that are no power of two too)."""
    if rng.random() < 0.5:
        most = max(work(c)["bytes"] for c in listed() if c["op"] == "few")
        while True:
            E = rng.choice([4, 8, 12, 20, 32, 60, 64, 96, 128, 160, 256])
            G = rng.choice([g for g in (1, 1, 2, 4, 8) if E % g == 0])
            k = rng.choice([n for n in (1, 2, 4, 6, 8, 16) if n <= E])
            topg = rng.randint(-(-k * G // E), G)
            c = _few("", rng.randint(1, 16), 256 * rng.randint(1, 28), E, k, 256 * rng.randint(1, 8),
                     rng.choice([0, 0, 1, 2]) * 1024, rng.choice(["sigmoid", "softmax"]), G, topg,
                     rng.random() < 0.5, rng.random() < 0.6, rng.choice([1.0, 2.5]),
                     rng.choice([0.0, 0.1]), rng.choice([0.0, 0.5]))
            if work(c)["bytes"] <= most and E * c["d"] * c["f"] <= 1_000_000_000:
                break
    else:
        op = rng.choice(["join", "join_grad"])
        block = rng.random() < 0.75
        norms = ["none", "rms", "layer"]
        c = _join("", op, _log_int(rng, 1, 16384), 8 * _log_int(rng, 1, 896), rng.choice(["bf16", "f32"]),
                  rng.choice(norms) if block else "none", rng.choice(norms if block else norms[1:]),
                  block and rng.random() < 0.4, block and rng.random() < 0.3,
                  rng.choice([1.0, 0.25]) if block else 1.0, rng.choice([0.0, 0.1, 0.5]) if block else 0.0,
                  block, op == "join_grad" or rng.random() < 0.5)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _normal(g, shape, std, dtype=F32):
    return torch.empty(shape, dtype=F32, device=DEV).normal_(0.0, std, generator=g).to(dtype)


def _stats(c, y, r):
    """Mean and reciprocal deviation of y's rows and of r's, as the forward keeps them."""
    out = torch.zeros(c["T"], 4, device=DEV)
    for at, kind, v in ((0, c["y_norm"], y), (2, c["r_norm"], r)):
        if kind == "none" or v is None:
            continue
        v = v.double()
        m = v.mean(1) if kind == "layer" else torch.zeros_like(v[:, 0])
        out[:, at] = m
        out[:, at + 1] = ((v - m[:, None]).square().mean(1) + EPS).rsqrt()
    return out


def _prepare_join(c, g):
    T, d = c["T"], c["d"]
    st = BF if c["stream"] == "bf16" else F32
    s = dict(c=c, x=None, y=None, r=None)
    if c["op"] == "join":
        s["x"] = _normal(g, (T, d), 1.0, st)
    else:
        s["r"] = _normal(g, (T, d), 1.0, st)
        s["dr"] = _normal(g, (T, d), 1.0, st)
        s["dh"] = _normal(g, (T, d), 1.0, BF)
    if c["block"]:
        s["y"] = _normal(g, (T, d), 0.5, BF)
        if c["y_norm"] == "layer":
            s["y"] += 0.25
    ones = lambda on, n: 1.0 + _normal(g, (n,), 0.2) if on else None   # noqa: E731
    s["y_weight"] = ones(c["y_norm"] != "none", d)
    s["y_bias"] = _normal(g, (d,), 0.2) if c["y_norm"] == "layer" else None
    s["r_weight"] = ones(c["r_norm"] != "none", d)
    s["r_bias"] = _normal(g, (d,), 0.2) if c["r_norm"] == "layer" else None
    s["gate"], s["token_gate"] = ones(c["gate"], d), ones(c["token_gate"], T)
    s["rng"] = torch.randint(0, 2 ** 62, (2,), dtype=I64, device=DEV, generator=g) if c["drop"] else None
    if c["op"] == "join_grad":
        s["stats"] = _stats(c, s["y"], s["r"])
    return s


def _prepare_few(c, g):
    T, d, E, f, fs = (c[n] for n in ("T", "d", "E", "f", "fs"))
    # Normal values on a grid (X on multiples of 1/16 up to 6, W_r of std
    # 1/sqrt(d) on 8 bits): every partial sum of a logit is then exact in 32
    # bits, so the logits, and with them the chosen experts, do not depend on
    # the order of summation.
    X = (_normal(g, (T, d), 16.0).round_().clamp_(-96, 96) / 16).to(BF)
    unit = 2.0 ** math.floor(math.log2(d ** -0.5 / 24))
    W_r = (_normal(g, (d, E), d ** -0.5 / unit).round_().clamp_(-240, 240) * unit).to(BF)
    s = dict(c=c, X=X, W_r=W_r, bias=_normal(g, (E,), c["bias"]) if c["bias"] else None,
             balance=_normal(g, (E,), c["balance"]) if c["balance"] else None)
    for name, shape in (("g", (E, d, f)), ("u", (E, d, f)), ("d", (E, f, d))):
        s["W" + name] = _normal(g, shape, shape[1] ** -0.5, BF)
    for name, shape in (("gs", (d, fs)), ("us", (d, fs)), ("ds", (fs, d))):
        s["W" + name] = _normal(g, shape, shape[0] ** -0.5, BF) if fs else None
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    return _prepare_few(case, g) if case["op"] == "few" else _prepare_join(case, g)


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------

def _mul_hi_lo(a, b):
    """High and low 32 bits of the product of a constant and 32-bit values held in 64."""
    p = b * (a & 0xffff)
    q = b * (a >> 16) + (p >> 16)
    return q >> 16, (q & 0xffff) << 16 | p & 0xffff


def _bits16(rng, T, d):
    """16 bits per element of a [T, d] array."""
    lo, hi = rng & 0xffffffff, rng >> 32 & 0xffffffff
    k0, k1 = lo[0], hi[0]
    shape = (T, d // 8)
    c0 = torch.arange(d // 8, device=DEV).expand(shape)
    c1 = torch.arange(T, device=DEV)[:, None].expand(shape)
    c2, c3 = lo[1].expand(shape), hi[1].expand(shape)
    for _ in range(10):
        h0, l0 = _mul_hi_lo(0xD2511F53, c0)
        h1, l1 = _mul_hi_lo(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = k0 + 0x9E3779B9 & 0xffffffff, k1 + 0xBB67AE85 & 0xffffffff
    words = torch.stack((c0, c1, c2, c3), 2)
    return torch.stack((words & 0xffff, words >> 16), 3).view(T, d)


def _kept(st, T, d):
    """What an element is multiplied with: 0, or one over the share that is kept."""
    out = math.floor(st["c"]["drop"] * 65536 + 0.5)
    return torch.where(_bits16(st["rng"], T, d) >= out, 65536.0 / (65536 - out), 0.0)


def _unit(kind, v):
    """A row's values without mean (layer) and divided by their deviation, and one over that."""
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    s = 1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * s, s


def _norm(kind, v, w, b):
    if kind == "none":
        return v
    v = _unit(kind, v)[0] * w
    return v if b is None else v + b


def _norm_grad(kind, v, w, dn):
    """Gradient of the norm of v: with respect to v, the weight and the bias."""
    if kind == "none":
        return dn, None, None
    u, s = _unit(kind, v)
    g = dn * w
    dv = g - u * (g * u).mean(1, keepdim=True)
    if kind == "layer":
        dv = dv - g.mean(1, keepdim=True)
    # the sums over the rows are long
    return s * dv, (dn * u).sum(0, dtype=F64).float(), dn.sum(0, dtype=F64).float() if kind == "layer" else None


def _factor(st):
    """scale, gate and token gate, as far as there are any."""
    a = torch.full((1, 1), st["c"]["scale"], device=DEV)
    if st["gate"] is not None:
        a = a * st["gate"]
    return a if st["token_gate"] is None else a * st["token_gate"][:, None]


def _plain_join(st):
    c = st["c"]
    r = st["x"]
    out = {}
    if c["block"]:
        v = _norm(c["y_norm"], st["y"].float(), st["y_weight"], st["y_bias"])
        if c["drop"]:
            v = v * _kept(st, c["T"], c["d"])
        r = out["r"] = (r.float() + _factor(st) * v).to(r.dtype)
    out["h"] = _norm(c["r_norm"], r.float(), st["r_weight"], st["r_bias"]).to(BF)
    if c["train"]:
        s = torch.zeros(c["T"], 4, device=DEV)
        for at, kind, v in ((0, c["y_norm"], st["y"]), (2, c["r_norm"], r)):
            if kind != "none":
                v = v.float()
                s[:, at] = v.mean(1) if kind == "layer" else 0.0
                s[:, at + 1] = _unit(kind, v)[1][:, 0]
        out["stats"] = s
    return out


def _plain_join_grad(st):
    c, dh, r = st["c"], st["dh"].float(), st["r"].float()
    D, dw, db = _norm_grad(c["r_norm"], r, st["r_weight"], dh)
    D = st["dr"].float() + D
    out = dict(dx=D.to(st["r"].dtype), r_weight=dw, r_bias=db)
    if c["block"]:
        y = st["y"].float()
        v = _norm(c["y_norm"], y, st["y_weight"], st["y_bias"])
        dn = _factor(st) * D
        if c["drop"]:
            kept = _kept(st, c["T"], c["d"])
            v, dn = v * kept, dn * kept
        v = c["scale"] * v * D
        if c["gate"]:
            t = v if st["token_gate"] is None else v * st["token_gate"][:, None]
            out["gate"] = t.sum(0, dtype=F64).float()
        if c["token_gate"]:
            out["token_gate"] = (v if st["gate"] is None else v * st["gate"]).sum(1, dtype=F64).float()
        dy, out["y_weight"], out["y_bias"] = _norm_grad(c["y_norm"], y, st["y_weight"], dn)
        out["dy"] = dy.to(BF)
    return {n: v for n, v in out.items() if v is not None}


def _route(c, logits, balance):
    """Chosen experts in ascending id, and their weights."""
    T, E = logits.shape
    G, k = c["groups"], c["k"]
    z = logits.double()
    if c["score"] == "sigmoid":
        s = 1.0 / (1.0 + torch.exp(-z))
    else:
        s = torch.exp(z - z.amax(1, keepdim=True))
        s = s / s.sum(1, keepdim=True)
    v = s if balance is None else s + balance.double()
    kept = torch.ones_like(v, dtype=torch.bool)
    if G > 1:
        best = v.view(T, G, E // G).sort(dim=2, descending=True).values
        gs = best[:, :, 0]
        if c["group_pair"] and E // G > 1:
            gs = gs + best[:, :, 1]
        order = gs.sort(dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        kept = torch.zeros(T, G, dtype=torch.bool, device=DEV).scatter_(1, order, True)
        kept = kept[:, :, None].expand(T, G, E // G).reshape(T, E)
    order = torch.where(kept, v, -math.inf).sort(dim=1, descending=True, stable=True).indices
    idx = order[:, :k].sort(dim=1).values
    w = s.gather(1, idx)
    if c["renormalise"]:
        w = w / w.sum(1, keepdim=True)
    return idx, (c["scale"] * w).float()


def _ffn(x, Wg, Wu, Wd):
    """[n, rows, d] through n experts."""
    a, b = torch.bmm(x, Wg.float()), torch.bmm(x, Wu.float())
    return torch.bmm(a / (1.0 + torch.exp(-a)) * b, Wd.float())


def _plain_few(st):
    c = st["c"]
    T, d, E, k = c["T"], c["d"], c["E"], c["k"]
    X = st["X"].float()
    logits = X @ st["W_r"].float()
    if st["bias"] is not None:
        logits = logits + st["bias"]
    idx, w = _route(c, logits, st["balance"])
    W = [st["Wg"], st["Wu"], st["Wd"]]
    if T * k <= E:       # few routes: each with its expert's weights
        e = idx.reshape(-1)
        x = X[:, None].expand(T, k, d).reshape(T * k, 1, d)
        y = _ffn(x, *(m[e] for m in W)).view(T, k, d)
    else:                # every token through every expert
        y = _ffn(X.expand(E, T, d), *W)[idx, torch.arange(T, device=DEV)[:, None]]
    Y = (w[:, :, None] * y).sum(1)
    if c["fs"]:
        Y = Y + _ffn(X[None], *(st[n][None] for n in ("Wgs", "Wus", "Wds")))[0]
    return dict(logits=logits, topk_idx=idx.to(I32), topk_w=w, Y=Y.to(BF))


# ---------------------------------------------------------------------------
# The framework's calls
# ---------------------------------------------------------------------------

PARAMS = ("y_weight", "y_bias", "gate", "token_gate", "r_weight", "r_bias")


class _Calls:
    """Outputs, workspace and argument structures that a program keeps."""

    def __init__(self, st):
        from paper_2609_36070_amd import binding as B
        self.B, c = B, st["c"]
        T, d = c["T"], c["d"]
        if c["op"] == "few":
            E, k = c["E"], c["k"]
            self.shape = B.make_shape(T, d, E, k, c["f"], c["fs"])
            self.routing = B.routing(c["score"], groups=c["groups"], top_groups=c["top_groups"],
                                     group_score="pair" if c["group_pair"] else "max",
                                     renormalise=c["renormalise"], scale=c["scale"])
            self.weights = B.weights_struct(*(st["W" + n] for n in ("g", "u", "d", "gs", "us", "ds")))
            self.ws = torch.empty(B.moe_few_workspace_bytes(self.shape), dtype=torch.uint8, device=DEV)
            self.logits = torch.empty(T, E, device=DEV)
            self.topk_idx = torch.empty(T, k, dtype=I32, device=DEV)
            self.topk_w = torch.empty(T, k, device=DEV)
            self.Y = torch.empty(T, d, dtype=BF, device=DEV)
            return
        self.join = B.join(T, d, c["stream"], y_norm=c["y_norm"], r_norm=c["r_norm"], y_eps=EPS, r_eps=EPS,
                           scale=c["scale"], drop=c["drop"])
        self.params = B.join_params(**{n: st[n] for n in PARAMS})
        like = st["x"] if c["op"] == "join" else st["r"]
        if c["op"] == "join":
            self.r = torch.empty_like(like) if c["block"] else None
            self.h = torch.empty(T, d, dtype=BF, device=DEV)
            self.stats = torch.empty(T, 4, device=DEV) if c["train"] else None
            return
        self.dx = torch.empty_like(like)
        self.dy = torch.empty(T, d, dtype=BF, device=DEV) if c["block"] else None
        self.d = {n: torch.empty_like(st[n]) for n in PARAMS if st[n] is not None}
        self.grads = B.join_grads(**self.d)
        self.ws = torch.empty(B.moe_join_workspace_bytes(self.join), dtype=torch.uint8, device=DEV)


def _own(st):
    if "calls" not in st:
        st["calls"] = _Calls(st)
    m, c = st["calls"], st["c"]
    if c["op"] == "few":
        m.B.moe_forward_few(m.shape, m.routing, st["X"], st["W_r"], st["bias"], st["balance"], m.weights,
                            m.logits, m.topk_idx, m.topk_w, m.Y, m.ws)
        return dict(logits=m.logits, topk_idx=m.topk_idx, topk_w=m.topk_w, Y=m.Y)
    if c["op"] == "join":
        m.B.moe_join_forward(m.join, st["x"], st["y"], m.params, st["rng"], m.r, m.h, m.stats)
        return {n: v for n, v in (("r", m.r), ("h", m.h), ("stats", m.stats)) if v is not None}
    m.B.moe_join_backward(m.join, st["y"], st["r"], st["stats"], m.params, st["rng"], st["dr"], st["dh"],
                          m.dx, m.dy, m.grads, m.ws)
    return dict(dx=m.dx, **({"dy": m.dy} if c["block"] else {}), **m.d)


def run(state):
    if own:
        return _own(state)
    plain = {"join": _plain_join, "join_grad": _plain_join_grad, "few": _plain_few}
    return plain[state["c"]["op"]](state)


def work(case):
    T, d = case["T"], case["d"]
    if case["op"] == "few":
        E, k = case["E"], case["k"]
        reached = E * (1.0 - (1.0 - k / E) ** T)
        return {"bytes": 6 * d * (reached * case["f"] + case["fs"]) + 2 * d * E + 4 * T * d + 4 * T * E + 8 * T * k,
                "flops": 6.0 * T * (k * case["f"] + case["fs"]) * d + 2.0 * T * d * E}
    s = 2 if case["stream"] == "bf16" else 4
    y = 2 if case["block"] else 0
    if case["op"] == "join":      # x, y in, r, h out
        return {"bytes": T * d * (s + y + (s if case["block"] else 0) + 2), "flops": 20.0 * T * d}
    # r, dr, dh in, dx out, and y, dy
    return {"bytes": T * d * (3 * s + 2 + 2 * y), "flops": 40.0 * T * d}


# ---------------------------------------------------------------------------
# From the definitions, in 64 bits
# ---------------------------------------------------------------------------

def _exact_kept(c, rng):
    """The multipliers of the kept elements, block of rows by block of rows."""
    seed, offset = (int(v) for v in rng.tolist())
    M = 0xffffffff
    T, n = c["T"], c["d"] // 8
    x = [torch.arange(n, device=DEV).repeat(T), torch.arange(T, device=DEV).repeat_interleave(n),
         torch.full((T * n,), offset & M, device=DEV), torch.full((T * n,), offset >> 32, device=DEV)]
    key = [seed & M, seed >> 32]

    def product(m, v):      # by bytes of the constant
        lo, carry = torch.zeros_like(v), torch.zeros_like(v)
        for i in range(4):
            carry = carry + (m >> 8 * i & 255) * v
            lo = lo | (carry & 255) << 8 * i
            carry = carry >> 8
        return carry, lo

    for i in range(10):
        a, b = product(0xD2511F53, x[0]), product(0xCD9E8D57, x[2])
        x = [b[0] ^ x[1] ^ (key[0] + i * 0x9E3779B9 & M), b[1], a[0] ^ x[3] ^ (key[1] + i * 0xBB67AE85 & M), a[1]]
    share = int(c["drop"] * 65536 + 0.5) / 65536
    out = torch.empty(T * n, 8, dtype=F64, device=DEV)
    for i in range(8):
        u = (x[i // 2] >> 16 * (i % 2) & 0xffff).double() / 65536
        out[:, i] = (u >= share).double() / (1.0 - share)
    return out.view(T, 8 * n)


def _exact_norm(kind, v, w, b):
    if kind == "none":
        return v
    if kind == "layer":
        return (v - v.mean(1, keepdim=True)) / (v.var(1, unbiased=False, keepdim=True) + EPS).sqrt() * w + b
    return v / (v.pow(2).mean(1, keepdim=True) + EPS).sqrt() * w


def _exact_join(c, st):
    wide = {n: None if st[n] is None else st[n].double() for n in PARAMS}
    grad = c["op"] == "join_grad"
    for p in wide.values():
        if grad and p is not None:
            p.requires_grad_()
    kept = _exact_kept(c, st["rng"]) if c["drop"] else 1.0
    y = st["y"].double().requires_grad_(grad) if c["block"] else None
    moved = 0.0
    if c["block"]:
        moved = c["scale"] * kept * _exact_norm(c["y_norm"], y, wide["y_weight"], wide["y_bias"])
        if c["gate"]:
            moved = moved * wide["gate"]
        if c["token_gate"]:
            moved = moved * wide["token_gate"][:, None]
    if not grad:
        r = st["x"].double() + moved
        stored = r.to(st["x"].dtype).double()      # h is the norm of the stored r
        out = dict(h=_exact_norm(c["r_norm"], stored, wide["r_weight"], wide["r_bias"]))
        if c["block"]:
            out["r"] = r
        if c["train"]:
            s = torch.zeros(c["T"], 4, dtype=F64, device=DEV)
            for at, kind, v in ((0, c["y_norm"], y), (2, c["r_norm"], stored)):
                if kind == "layer":
                    s[:, at], s[:, at + 1] = v.mean(1), (v.var(1, unbiased=False) + EPS) ** -0.5
                elif kind == "rms":
                    s[:, at + 1] = (v.pow(2).mean(1) + EPS) ** -0.5
            out["stats"] = s
        return out
    r = st["r"].double().requires_grad_()
    h = _exact_norm(c["r_norm"], r, wide["r_weight"], wide["r_bias"])
    (h * st["dh"].double()).sum().backward()
    D = r.grad + st["dr"].double()
    out = dict(dx=D)
    if c["block"]:
        (moved * D).sum().backward()
        out["dy"] = y.grad
    out.update({n: p.grad for n, p in wide.items() if p is not None})
    return out


def exact(case, seed):
    c, st = case, prepare(case, seed)
    T = c["T"]
    if c["op"] != "few":
        return _exact_join(c, st)
    E = c["E"]
    X = st["X"].double()
    z = X @ st["W_r"].double()
    if st["bias"] is not None:   # the logits are 32-bit values
        z = (z.float() + st["bias"]).double()
    logp = -torch.logaddexp(torch.zeros_like(z), -z) if c["score"] == "sigmoid" else \
        z - torch.logsumexp(z, 1, keepdim=True)
    p = logp.exp()
    v = p if st["balance"] is None else p + st["balance"].double()
    G, n = c["groups"], E // c["groups"]
    allowed = torch.ones(T, G, dtype=torch.bool, device=DEV)
    if G > 1:
        gv = v.view(T, G, n)
        first = gv.max(2)
        gs = first.values.clone()
        if c["group_pair"] and n > 1:
            gs += gv.scatter(2, first.indices[..., None], -math.inf).max(2).values
        ids = torch.arange(G, device=DEV)
        better = (gs[:, None, :] > gs[:, :, None]) | \
            ((gs[:, None, :] == gs[:, :, None]) & (ids[None, None, :] < ids[None, :, None]))
        allowed = better.sum(2) < c["top_groups"]
    free = allowed.repeat_interleave(n, dim=1)
    chosen = torch.zeros(T, E, dtype=torch.bool, device=DEV)
    for _ in range(c["k"]):      # the best one left; argmax of a 0/1 row is its first 1
        left = free & ~chosen
        top = torch.where(left, v, -math.inf).max(1, keepdim=True).values
        chosen.scatter_(1, (left & (v == top)).to(torch.int8).argmax(1, keepdim=True), True)
    idx = chosen.nonzero()[:, 1].view(T, c["k"])
    w = p.gather(1, idx)
    if c["renormalise"]:
        w = w / w.sum(1, keepdim=True)
    w = c["scale"] * w

    def expert(x, Wg, Wu, Wd):
        a = x @ Wg.double()
        return (a * torch.sigmoid(a) * (x @ Wu.double())) @ Wd.double()

    Y = torch.zeros(T, c["d"], dtype=F64, device=DEV)
    for e in idx.unique().tolist():
        t, slot = (idx == e).nonzero(as_tuple=True)
        Y[t] += w[t, slot][:, None] * expert(X[t], st["Wg"][e], st["Wu"][e], st["Wd"][e])
    if c["fs"]:
        Y += expert(X, st["Wgs"], st["Wus"], st["Wds"])
    return dict(logits=z, topk_idx=idx.to(I32), topk_w=w, Y=Y)
