"""Performance cases of the pruned layers of a feed-forward path, from one token to a prompt, with the
gradients that fine-tuning the surviving weights takes.

Four kinds of call are covered; W (and W_gate, W_up) are pruned bf16 layers, x holds `tokens` vectors:
  linear           y = act(W x + bias) + residual in one pass (dbspmspv_linear)
  linear_backward  the gradients of x, of the stored weights and of the bias (dbspmspv_linear_backward)
  gated            y = act(W_gate x) * (W_up x), both projections in one pass (dbspmspv_gated)
  gated_backward   the gradients of x and of the stored weights of both layers (dbspmspv_gated_backward)
"""
import math

import torch

DEV = "cuda"
own = False
ACTS = ("none", "relu", "silu", "gelu")


def listed():
    return [
        # a small projection and one token, its sums handed on in 32 bits: the call's latency
        {"name": "linear_1024x1024_t1", "kind": "linear", "m": 1024, "n": 1024, "tokens": 1, "prune": 0.5, "zeros": 0.0,
         "act": "none", "bias": True, "residual": False, "keep": False, "f32": True, "pad": 0},
        # the fused projection of queries, keys and values: one token of thinned-out activations
        {"name": "linear_12288x4096_t1", "kind": "linear", "m": 12288, "n": 4096, "tokens": 1, "prune": 0.5, "zeros": 0.7,
         "act": "none", "bias": False, "residual": False, "keep": False, "f32": False, "pad": 0},
        # the projection back from the hidden width onto the residual stream, eight sequences side by side
        {"name": "linear_4096x11008_t8", "kind": "linear", "m": 4096, "n": 11008, "tokens": 8, "prune": 0.7, "zeros": 0.5,
         "act": "none", "bias": False, "residual": True, "keep": False, "f32": False, "pad": 0},
        # a short prompt through an ungated layer, sizes and strides off every tile; what its gradient needs is kept
        {"name": "linear_4111x1037_t333", "kind": "linear", "m": 4111, "n": 1037, "tokens": 333, "prune": 0.6, "zeros": 0.0,
         "act": "gelu", "bias": True, "residual": True, "keep": True, "f32": False, "pad": 3},
        # a long prompt through the projection back
        {"name": "linear_4096x11008_t2048", "kind": "linear", "m": 4096, "n": 11008, "tokens": 2048, "prune": 0.5, "zeros": 0.0,
         "act": "none", "bias": False, "residual": True, "keep": False, "f32": False, "pad": 0},
        # the gated half of a feed-forward block: one token as the norm in front of it leaves it, without zeros
        {"name": "gated_11008x4096_t1", "kind": "gated", "m": 11008, "n": 4096, "tokens": 1, "prune": 0.5, "zeros": 0.0,
         "act": "silu", "keep": False, "pad": 0},
        # the same for a handful of drafted tokens, weights pruned further
        {"name": "gated_11008x4096_t6", "kind": "gated", "m": 11008, "n": 4096, "tokens": 6, "prune": 0.7, "zeros": 0.0,
         "act": "relu", "keep": False, "pad": 0},
        # the forward half of a training step: both projections are kept for the gradient
        {"name": "gated_11008x4096_t2048", "kind": "gated", "m": 11008, "n": 4096, "tokens": 2048, "prune": 0.5, "zeros": 0.0,
         "act": "silu", "keep": True, "pad": 0},
        # the gradient of an ungated layer with its bias
        {"name": "linear_bwd_4096x4096_t500", "kind": "linear_backward", "m": 4096, "n": 4096, "tokens": 500, "prune": 0.5,
         "zeros": 0.0, "act": "relu", "bias": True, "pad": 0},
        # the gradient of a narrow layer without an activation, few tokens, strides off the tiles
        {"name": "linear_bwd_1037x2751_t77", "kind": "linear_backward", "m": 1037, "n": 2751, "tokens": 77, "prune": 0.7,
         "zeros": 0.3, "act": "none", "bias": False, "pad": 3},
        # the backward half of the training step
        {"name": "gated_bwd_11008x4096_t2048", "kind": "gated_backward", "m": 11008, "n": 4096, "tokens": 2048, "prune": 0.5,
         "zeros": 0.0, "act": "silu", "pad": 0},
        # and of a narrow block on a short ragged batch
        {"name": "gated_bwd_2751x1025_t301", "kind": "gated_backward", "m": 2751, "n": 1025, "tokens": 301, "prune": 0.6,
         "zeros": 0.0, "act": "gelu", "pad": 1},
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(["linear", "linear", "gated", "gated", "linear_backward", "gated_backward"])
    while True:
        m, n = int(_log_uniform(rng, 200, 12288.99)), int(_log_uniform(rng, 200, 12288.99))
        if m * n <= 11008 * 4096:
            break
    backward = kind.endswith("backward")
    tokens = rng.choice([1, int(_log_uniform(rng, 2, 16.99)), int(_log_uniform(rng, 17, 2048.99))])
    case = {"kind": kind, "m": m, "n": n, "tokens": tokens, "prune": rng.choice([0.5, 0.6, 0.7]),
            "zeros": rng.choice([0.0, 0.0, 0.5, 0.9]), "act": rng.choice(ACTS[1:] if kind.startswith("gated") else ACTS),
            "pad": rng.choice([0, 0, 1, 8])}
    if kind.startswith("linear"):
        case["bias"] = rng.random() < 0.5
    if not backward:
        case["keep"] = rng.random() < 0.3
    if kind == "linear":
        case["residual"] = rng.random() < 0.5
        # (sums handed on in 32 bits: what the next norm or a residual stream of that width takes from a single token)
        case["f32"] = tokens == 1 and rng.random() < 0.5
    return case


def _layer(case, gen):
    """A dense bf16 matrix whose smallest magnitudes, exactly the share `prune` of all, are zero: the scale keeps sums near 1."""
    w = torch.randn(case["m"] * case["n"], generator=gen, device=DEV)
    w[torch.argsort(w.abs())[: int(case["prune"] * w.numel())]] = 0.0
    return (w / math.sqrt(case["n"] * (1.0 - case["prune"]))).to(torch.bfloat16).reshape(case["m"], case["n"])


def _rows(case, width, gen, zeros=0.0, scale=1.0):
    """tokens x width in bf16, rows `pad` entries apart"""
    v = torch.randn((case["tokens"], width + case["pad"]), generator=gen, device=DEV) * scale
    if zeros:
        v *= torch.rand(v.shape, generator=gen, device=DEV) >= zeros
    return v.to(torch.bfloat16)[:, :width]


def _inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    m, n = case["m"], case["n"]
    s = {"x": _rows(case, n, gen, zeros=case["zeros"])}
    if case["kind"].startswith("linear"):
        s["w"] = [_layer(case, gen)]
    else:
        s["w"] = [_layer(case, gen), _layer(case, gen)]
    if case["kind"] == "linear":
        s["bias"] = torch.randn(m, generator=gen, device=DEV).to(torch.bfloat16) if case["bias"] else None
        s["residual"] = _rows(case, m, gen) if case["residual"] else None
    if case["kind"].endswith("backward"):
        s["dy"] = _rows(case, m, gen)
        # what the forward call kept: the values in front of the activation, and the other projection
        s["z"] = None if case["act"] == "none" else _rows(case, m, gen, scale=1.5)
        s["u"] = _rows(case, m, gen) if case["kind"].startswith("gated") else None
    return s


class _State:
    """What a user's program has in hand: the inputs, the layers' handles, the buffers it calls with."""

    def __init__(self, case, seed):
        self.case = case
        self.__dict__.update(_inputs(case, seed))
        self.handles = []
        m, n, t, pad = case["m"], case["n"], case["tokens"], case["pad"]
        backward = case["kind"].endswith("backward")
        # places of the stored weights, row by row (the order of a CSR matrix)
        self.at = [torch.nonzero(w.reshape(-1)).reshape(-1) for w in self.w] if backward or own else None
        if not own:
            return
        from paper_2608_16308_b200 import binding as B
        self.B = B
        self.code = {"none": B.ACT_NONE, "relu": B.ACT_RELU, "silu": B.ACT_SILU, "gelu": B.ACT_GELU}[case["act"]]
        opts = B.default_create_opts()
        opts.linear = 1
        for w, at in zip(self.w, self.at):
            ptr = torch.zeros(m + 1, dtype=torch.int64, device=DEV)
            torch.cumsum((w != 0).sum(dim=1), 0, out=ptr[1:])
            self.handles.append(B.dbspmspv_create_csr(m, n, at.numel(), ptr, (at % n).to(torch.int32), w.reshape(-1)[at], B.BF16, 16, opts))
        self.w = None                                  # (the handles hold the weights)

        def rows(width, dtype=torch.bfloat16):
            return torch.empty((t, width + pad), dtype=dtype, device=DEV)[:, :width]

        if backward:
            self.dx = rows(n)
            self.dw = [torch.empty(at.numel(), dtype=torch.bfloat16, device=DEV) for at in self.at]
            self.dbias = torch.empty(m, dtype=torch.float32, device=DEV) if case.get("bias") else None
        else:
            self.y = rows(m, torch.float32 if case.get("f32") else torch.bfloat16)
            self.z = rows(m) if case["keep"] else None
            self.u = rows(m) if case["keep"] and case["kind"] == "gated" else None
        self.at = None
        up = self.handles[1] if len(self.handles) > 1 else None
        self.room = B.dbspmspv_linear_workspace(self.handles[0], up, t, backward)
        self.workspace = torch.empty(self.room, dtype=torch.uint8, device=DEV)

    def __del__(self):
        for h in getattr(self, "handles", ()):
            self.B.dbspmspv_destroy(h)


def prepare(case, seed):
    return _State(case, seed)


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)


def _plain(s):
    c = s.case
    x = s.x.float()
    w = [v.float() for v in s.w]
    half = torch.bfloat16
    if c["kind"] == "linear":
        z = x @ w[0].T
        if s.bias is not None:
            z = z + s.bias.float()
        y = _act(z, c["act"])
        if s.residual is not None:
            y = y + s.residual.float()
        return {"y": y if c["f32"] else y.to(half), "z": z.to(half) if c["keep"] else None}
    if c["kind"] == "gated":
        g, u = x @ w[0].T, x @ w[1].T
        return {"y": (_act(g, c["act"]) * u).to(half), "z": g.to(half) if c["keep"] else None, "u": u.to(half) if c["keep"] else None}
    dy = s.dy.float()
    if c["kind"] == "linear_backward":
        dz = [dy if s.z is None else dy * _act_slope(s.z.float(), c["act"])]
    else:
        z, u = s.z.float(), s.u.float()
        dz = [dy * u * _act_slope(z, c["act"]), dy * _act(z, c["act"])]
    dx = dz[0] @ w[0]
    if len(dz) > 1:
        dx = dx + dz[1] @ w[1]
    dw = [(d.T @ x).reshape(-1)[at].to(half) for d, at in zip(dz, s.at)]
    return {"dx": dx.to(half), "dw": dw, "dbias": dz[0].sum(dim=0) if c.get("bias") else None}


def _calls(s):
    c, B, h, t = s.case, s.B, s.handles, s.case["tokens"]
    ld = lambda v: v.stride(0) if v is not None else 0  # noqa: E731
    if c["kind"] == "linear":
        B.dbspmspv_linear(h[0], s.x, ld(s.x), t, s.bias, s.code, s.residual, ld(s.residual), s.y, ld(s.y), int(c["f32"]), s.z, ld(s.z), s.workspace, s.room)
        return {"y": s.y, "z": s.z}
    if c["kind"] == "gated":
        B.dbspmspv_gated(h[0], h[1], s.x, ld(s.x), t, s.code, s.y, ld(s.y), s.z, s.u, ld(s.z), s.workspace, s.room)
        return {"y": s.y, "z": s.z, "u": s.u}
    if c["kind"] == "linear_backward":
        B.dbspmspv_linear_backward(h[0], s.x, ld(s.x), t, s.code, s.z, ld(s.z), s.dy, ld(s.dy), s.dx, ld(s.dx), s.dw[0], s.dbias, s.workspace, s.room)
    else:
        B.dbspmspv_gated_backward(h[0], h[1], s.x, ld(s.x), t, s.code, s.z, s.u, ld(s.z), s.dy, ld(s.dy), s.dx, ld(s.dx), s.dw[0], s.dw[1], s.workspace, s.room)
    return {"dx": s.dx, "dw": s.dw, "dbias": s.dbias}


def run(state):
    return _calls(state) if own else _plain(state)


def work(case):
    m, n, t = case["m"], case["n"], case["tokens"]
    layers = 2 if case["kind"].startswith("gated") else 1
    # the weights that some token reaches, 2 bytes each; a product and a sum for each weight and entry that is not zero
    reached = 1.0 - case["zeros"] ** t
    stored = layers * m * n * (1.0 - case["prune"])
    product = 2.0 * stored * t * (1.0 - case["zeros"])
    if case["kind"] in ("linear", "gated"):
        rows = n + m * (2 if case.get("f32") else 1) + (m if case.get("residual") else 0) + (layers * m if case["keep"] else 0)
        return {"bytes": 2.0 * (stored * reached + t * rows + (m if case.get("bias") else 0)), "flops": product}
    rows = 2 * n + m + (0 if case["act"] == "none" else layers * m)
    return {"bytes": 2.0 * (2 * stored + t * rows) + (4.0 * m if case.get("bias") else 0), "flops": 2.0 * stored * t + product}


def exact(case, seed):
    """From the definition, a projection at a time, every sum in 64 bits."""
    s = _inputs(case, seed)
    act, kind = case["act"], case["kind"]

    def f(v):
        return {"none": lambda: v, "relu": lambda: torch.relu(v), "silu": lambda: v * torch.sigmoid(v),
                "gelu": lambda: v * torch.special.ndtr(v)}[act]()

    def slope(v):
        if act == "none":
            return torch.ones_like(v)
        if act == "relu":
            return torch.where(v > 0, 1.0, 0.0).double()
        if act == "silu":
            return torch.sigmoid(v) + v * torch.sigmoid(v) * torch.sigmoid(-v)
        return torch.special.ndtr(v) + v * torch.exp(-v.square() / 2) / math.sqrt(math.tau)

    x = s["x"].double()
    project = lambda k: torch.einsum("tn,mn->tm", x, s["w"][k].double())  # noqa: E731
    if kind == "linear":
        z = project(0)
        if s["bias"] is not None:
            z += s["bias"].double()
        y = f(z)
        if s["residual"] is not None:
            y = y + s["residual"].double()
        return {"y": y, "z": z if case["keep"] else None}
    if kind == "gated":
        g, u = project(0), project(1)
        return {"y": f(g) * u, "z": g if case["keep"] else None, "u": u if case["keep"] else None}
    dy = s["dy"].double()
    z = s["z"].double() if s["z"] is not None else torch.ones_like(dy)
    if kind == "linear_backward":
        d = [dy * slope(z)]
    else:
        d = [dy * s["u"].double() * slope(z), dy * f(z)]
    dx = sum(torch.einsum("tm,mn->tn", v, w.double()) for v, w in zip(d, s["w"]))
    dw = [torch.einsum("tm,tn->mn", v, x)[w != 0] for v, w in zip(d, s["w"])]
    return {"dx": dx, "dw": dw, "dbias": d[0].sum(dim=0) if case.get("bias") else None}
