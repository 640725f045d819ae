"""Performance cases of what stands between and behind the pruned layers of a network: the join of a block with the
residual stream (norms before and after it, gate, dropout, residual scale), dropout by itself, and log probabilities,
each with its gradient, from one token to a long batch.

Five kinds of call are covered:
  join              out = r + scale * drop(gate * norm(b)), h = norm(out)            (dbspmspv_join)
  join_backward     the gradients of r, b, the gate and the norms' parameters        (dbspmspv_join_backward)
  dropout           y = drop(x), forwards and backwards alike                        (dbspmspv_dropout)
  logprobs          log probabilities of given tokens, entropy, top alternatives     (dbspmspv_logprobs)
  logprobs_backward the gradient of the logits                                       (dbspmspv_logprobs_backward)

Random numbers are inputs: an entry in column c of row t takes 16 bits of Philox 4x32-10 (Salmon, Moraes, Dror and Shaw, 2011)
at the counter (c / 8, t, offset), key = seed; it is dropped where they are below 65536 p.
"""
import math

import numpy as np
import torch

DEV = "cuda"
own = False
NORMS = ("none", "rms", "layer")
HALF = torch.bfloat16
EPS = 1e-5


def _join(name, tokens, n, **kw):
    c = {"kind": "join", "tokens": tokens, "n": n, "norm_block": "rms", "norm_next": "rms", "bias": False, "gate": "none", "scale": 1.0,
         "drop": 0.0, "stream_f32": False, "block_f32": False, "params_f32": False, "pad": 0}
    return {**({"name": name} if name else {}), **c, **kw}


def _logprobs(name, tokens, vocab, **kw):
    c = {"kind": "logprobs", "tokens": tokens, "vocab": vocab, "f32": True, "temperature": 1.0, "masked": 0.0, "entropy": True, "top": 0, "pad": 0}
    return {**({"name": name} if name else {}), **c, **kw}


def listed():
    return [
        # one token on its way through a network, norms on both sides of the block: the call's latency
        _join("join_4096_t1", 1, 4096),
        # a few sequences side by side, the stream and the layer's sums in 32 bits, a gate per channel
        _join("join_4096_t8", 8, 4096, stream_f32=True, block_f32=True, params_f32=True, gate="shared", scale=0.22),
        # layer norms with biases, a gate for each token (conditioning), sizes and strides off every vector
        _join("join_1037_t333", 333, 1037, norm_block="layer", norm_next="layer", bias=True, gate="token", pad=3),
        # the forward half of a training step on long rows
        _join("join_4096_t4096", 4096, 4096, gate="shared", drop=0.1, keep=True),
        # the backward half of it
        _join("join_bwd_4096_t4096", 4096, 4096, kind="join_backward", gate="shared", drop=0.1),
        # the gradient of a small layer-normed block, a gate for each token, strides off every vector, parameters in 32 bits
        _join("join_bwd_2751_t77", 77, 2751, kind="join_backward", norm_block="layer", norm_next="layer", bias=True, gate="token", params_f32=True, drop=0.2, pad=3),
        # dropout on the hidden activations of a feed-forward block
        {"name": "dropout_11008_t2048", "kind": "dropout", "tokens": 2048, "n": 11008, "f32": False, "drop": 0.1, "pad": 0},
        # a short ragged batch in 32 bits
        {"name": "dropout_1025_t301", "kind": "dropout", "tokens": 301, "n": 1025, "f32": True, "drop": 0.5, "pad": 1},
        # the next token of one sequence: what it was, and twenty it could have been, some of the vocabulary forbidden
        _logprobs("logprobs_32000_t1", 1, 32000, top=20, temperature=0.7, masked=0.3),
        # scoring a batch of answers
        _logprobs("logprobs_32000_t2048", 2048, 32000, f32=False, top=5),
        # the gradient of that batch's loss with a term for the entropy
        _logprobs("logprobs_bwd_32000_t2048", 2048, 32000, kind="logprobs_backward", f32=False),
        # a large vocabulary of odd size in 32 bits, alternatives distilled
        _logprobs("logprobs_bwd_100003_t63", 63, 100003, kind="logprobs_backward", top=8, pad=5),
    ]


def _log_uniform(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.99))))


def draw(rng):
    kind = rng.choice(["join", "join", "join_backward", "join_backward", "dropout", "logprobs", "logprobs", "logprobs_backward"])
    pad = rng.choice([0, 0, 1, 8])
    if kind.startswith("logprobs"):
        vocab = _log_uniform(rng, 1000, 131072)
        if rng.random() < 0.5:
            vocab -= vocab % 8
        tokens = rng.choice([1, _log_uniform(rng, 2, 64), _log_uniform(rng, 2, 4096)])
        tokens = min(tokens, 2048 * 32000 // vocab)
        return _logprobs("", tokens, vocab, kind=kind, f32=rng.random() < 0.5, temperature=rng.choice([1.0, 1.0, 0.6, 1.7]), masked=rng.choice([0.0, 0.0, 0.5]),
                         entropy=rng.random() < 0.6, top=rng.choice([0, 0, 1, 5, 20]), pad=pad)
    n = _log_uniform(rng, 64, 12288)
    if rng.random() < 0.5:
        n -= n % 8
    tokens = min(rng.choice([1, _log_uniform(rng, 2, 64), _log_uniform(rng, 2, 8192)]), 4096 * 4096 // n)
    if kind == "dropout":
        return {"kind": kind, "tokens": tokens, "n": n, "f32": rng.random() < 0.5, "drop": rng.choice([0.1, 0.25, 0.5]), "pad": pad}
    norm_next = rng.choice(NORMS[1:])
    case = _join("", tokens, n, kind=kind, norm_block=rng.choice(["none", "rms", "layer"]), norm_next=norm_next, bias=rng.random() < 0.3, gate=rng.choice(["none", "shared", "token"]),
                 scale=rng.choice([1.0, 0.22]), drop=rng.choice([0.0, 0.1]), stream_f32=rng.random() < 0.4, block_f32=rng.random() < 0.3, params_f32=rng.random() < 0.5, pad=pad)
    if kind == "join":
        case["keep"] = rng.random() < 0.5
    return case


def _type(f32):
    return torch.float32 if f32 else HALF


class _State:
    """What a user's program has in hand: the inputs, and the buffers it calls with."""

    def __init__(self, case, seed):
        self.case = case
        self.gen = torch.Generator(device=DEV).manual_seed(seed)
        {"join": self.join, "dropout": self.dropout, "logprobs": self.logprobs}[case["kind"].split("_")[0]]()
        self.gen = None
        if own and case["kind"].startswith("join"):
            self.options()

    def rows(self, width, f32=False, scale=1.0, mean=0.0, skew=False):
        """tokens x width, rows `pad` entries apart; skew: tokens of different sizes, as a residual stream has them"""
        v = torch.randn((self.case["tokens"], width + self.case["pad"]), generator=self.gen, device=DEV) * scale + mean
        if skew:
            v *= torch.exp(torch.randn((v.shape[0], 1), generator=self.gen, device=DEV) * 0.5)
        return v.to(_type(f32))[:, :width]

    def room(self, width, dtype=HALF):
        return torch.empty((self.case["tokens"], width + self.case["pad"]), dtype=dtype, device=DEV)[:, :width]

    def vector(self, n, mean=0.0):
        return (torch.randn(n, generator=self.gen, device=DEV) * 0.2 + mean).to(_type(self.case["params_f32"]))

    def numbers(self):
        """seed and offset of the random numbers, as the device holds them"""
        return torch.randint(0, 1 << 62, (2,), generator=self.gen, device=DEV, dtype=torch.int64)

    def join(self):
        c, n = self.case, self.case["n"]
        st, bt, pt = _type(c["stream_f32"]), _type(c["block_f32"]), _type(c["params_f32"])
        backward = c["kind"] == "join_backward"
        # (of a step backwards, r is the stream behind the join: what the forward call wrote)
        self.r = self.rows(n, c["stream_f32"], skew=True)
        self.b = self.rows(n, c["block_f32"], mean=0.1)
        self.w_block = self.vector(n, 1.0) if c["norm_block"] != "none" else None
        self.w_next = self.vector(n, 1.0)
        self.c_block = self.vector(n) if c["bias"] and c["norm_block"] != "none" else None
        self.c_next = self.vector(n) if c["bias"] else None
        self.gate = None if c["gate"] == "none" else self.vector(n, 0.5) if c["gate"] == "shared" else self.rows(n, c["params_f32"], 0.2, 0.5)
        self.random = self.numbers() if c["drop"] else None
        if not backward:
            self.out, self.h = self.room(n, st), self.room(n)
            self.stats = torch.empty((c["tokens"], 4), device=DEV) if c.get("keep") else None
            return
        self.stats = torch.cat([_stats(self.b.float(), c["norm_block"]), _stats(self.r.float(), c["norm_next"])], dim=1).contiguous()
        self.dh, self.dout = self.rows(n, scale=0.5), self.rows(n, c["stream_f32"])
        self.dr, self.db = self.room(n, st), self.room(n, bt)
        self.dgate = None if c["gate"] == "none" else torch.empty(n, device=DEV) if c["gate"] == "shared" else self.room(n, pt)
        self.dw_block, self.dc_block, self.dw_next, self.dc_next = (None if p is None else torch.empty(n, device=DEV) for p in (self.w_block, self.c_block, self.w_next, self.c_next))

    def options(self):
        from paper_2608_16308_b200 import binding as B
        c, o = self.case, B.default_join_opts()
        o.norm_block, o.norm_next, o.eps_block, o.eps_next = NORMS.index(c["norm_block"]), NORMS.index(c["norm_next"]), EPS, EPS
        o.scale, o.drop = c["scale"], c["drop"]
        o.stream_f32, o.block_f32, o.params_f32, o.dblock_f32 = (int(c[k]) for k in ("stream_f32", "block_f32", "params_f32", "block_f32"))
        self.opts = o
        if c["kind"] == "join_backward":
            self.bytes = B.dbspmspv_join_workspace(o, c["tokens"], c["n"])
            self.workspace = torch.empty(self.bytes, dtype=torch.uint8, device=DEV)

    def dropout(self):
        c = self.case
        self.x, self.random, self.y = self.rows(c["n"], c["f32"]), self.numbers(), self.room(c["n"], _type(c["f32"]))

    def logprobs(self):
        c, t, v = self.case, self.case["tokens"], self.case["vocab"]
        logits = torch.randn((t, v + c["pad"]), generator=self.gen, device=DEV) * 2.5
        if c["masked"]:
            logits[torch.rand(logits.shape, generator=self.gen, device=DEV) < c["masked"]] = -math.inf
        logits[:, 7] = 1.0                                     # (something is left in every row)
        self.logits = logits.to(_type(c["f32"]))[:, :v]
        # tokens that were likely; one in sixteen is padding
        likely = torch.rand((t, 64), generator=self.gen, device=DEV)
        at = (likely * v).long().clamp(max=v - 1)
        best = self.logits.float().gather(1, at).argmax(dim=1, keepdim=True)
        padding = torch.rand(t, generator=self.gen, device=DEV) < 1 / 16
        padding[0] = False
        self.targets = torch.where(padding, -1, at.gather(1, best)[:, 0]).to(torch.int32)
        k = c["top"]
        if c["kind"] == "logprobs":
            self.logprob, self.stats = torch.empty(t, device=DEV), torch.empty((t, 2), device=DEV)
            self.entropy = torch.empty(t, device=DEV) if c["entropy"] else None
            self.top_ids = torch.empty((t, k), dtype=torch.int32, device=DEV) if k else None
            self.top_logprobs = torch.empty((t, k), device=DEV) if k else None
            return
        # what a forward call kept: the largest logit, and the logarithm of the sum relative to it
        z = self.logits.float()
        most = z.amax(dim=1, keepdim=True)
        z = (z - most) / c["temperature"]
        self.stats = torch.cat([most, torch.logsumexp(z, dim=1, keepdim=True)], dim=1)
        logp = torch.log_softmax(z, dim=1)
        self.entropy = -(logp.exp() * logp.clamp(min=-1e30)).sum(dim=1) if c["entropy"] else None
        self.top_ids = logp.topk(k, dim=1).indices.to(torch.int32) if k else None
        self.dlogprob = -torch.rand(t, generator=self.gen, device=DEV) / t
        self.dentropy = torch.full((t,), -0.01 / t, device=DEV) if c["entropy"] else None
        self.dtop = torch.randn((t, k), generator=self.gen, device=DEV) / t if k else None
        self.dlogits = self.room(v, _type(c["f32"]))


def prepare(case, seed):
    return _State(case, seed)


# ---- the plain forms -----------------------------------------------------------------------------
def _stats(x, norm):
    """mean and 1 / deviation of each row, as a forward call keeps them"""
    if norm == "none":
        return torch.tensor([0.0, 1.0], device=x.device).expand(x.shape[0], 2)
    mean = x.mean(dim=1, keepdim=True) if norm == "layer" else torch.zeros_like(x[:, :1])
    return torch.cat([mean, 1 / torch.sqrt((x - mean).square().mean(dim=1, keepdim=True) + EPS)], dim=1)


def _numbers(random, tokens, n):
    """16 random bits for each entry: Philox 4x32-10, eight columns to a counter"""
    word = 0xFFFFFFFF
    seed, offset = random[0], random[1]
    k0, k1 = seed & word, (seed >> 32) & word
    blocks = (n + 7) // 8
    a = torch.arange(blocks, device=DEV).expand(tokens, blocks)
    b = torch.arange(tokens, device=DEV)[:, None].expand(tokens, blocks)
    c, d = (offset & word).expand(tokens, blocks), ((offset >> 32) & word).expand(tokens, blocks)
    for _ in range(10):
        p, q = a * 0xD2511F53, c * 0xCD9E8D57                  # (64 bits that wrap: both halves are right)
        a, b, c, d = ((q >> 32) & word) ^ b ^ k0, q & word, ((p >> 32) & word) ^ d ^ k1, p & word
        k0, k1 = (k0 + 0x9E3779B9) & word, (k1 + 0xBB67AE85) & word
    words = torch.stack([a, b, c, d], dim=2)
    return torch.stack([words & 0xFFFF, words >> 16], dim=3).reshape(tokens, blocks * 8)[:, :n]


def _keep(random, tokens, n, drop):
    """what each entry is multiplied with: 0, or what makes up for the dropped ones"""
    if not drop:
        return 1.0
    below = int(drop * 65536 + 0.5)
    return (_numbers(random, tokens, n) >= below).float() * (65536.0 / (65536 - below))


def _plain_join(s):
    c = s.case
    b, r = s.b.float(), s.r.float()
    st = _stats(b, c["norm_block"])
    y = (b - st[:, :1]) * st[:, 1:]
    if s.w_block is not None:
        y = y * s.w_block.float()
    if s.c_block is not None:
        y = y + s.c_block.float()
    if s.gate is not None:
        y = y * s.gate.float()
    out = r + c["scale"] * _keep(s.random, c["tokens"], c["n"], c["drop"]) * y
    sn = _stats(out, c["norm_next"])
    h = (out - sn[:, :1]) * sn[:, 1:] * s.w_next.float()
    if s.c_next is not None:
        h = h + s.c_next.float()
    return {"out": out.to(s.r.dtype), "h": h.to(HALF), "stats": torch.cat([st, sn], dim=1) if c.get("keep") else None}


def _slope(u, xhat, rstd, norm):
    """the gradient in front of a norm from that behind its normalised values"""
    if norm == "none":
        return u
    if norm == "layer":
        u = u - u.mean(dim=1, keepdim=True)
    return rstd * (u - xhat * (u * xhat).mean(dim=1, keepdim=True))


def _plain_join_backward(s):
    c, stats = s.case, s.stats
    dh = s.dh.float()
    xhat = (s.r.float() - stats[:, 2:3]) * stats[:, 3:4]
    g = s.dout.float() + _slope(dh * s.w_next.float(), xhat, stats[:, 3:4], c["norm_next"])
    q = c["scale"] * _keep(s.random, c["tokens"], c["n"], c["drop"]) * g
    bhat = (s.b.float() - stats[:, 0:1]) * stats[:, 1:2]
    dp = q if s.gate is None else q * s.gate.float()
    db = _slope(dp if s.w_block is None else dp * s.w_block.float(), bhat, stats[:, 1:2], c["norm_block"])
    dgate = None
    if s.gate is not None:
        p = bhat if s.w_block is None else bhat * s.w_block.float()
        dgate = q * (p if s.c_block is None else p + s.c_block.float())
        dgate = dgate.sum(dim=0) if c["gate"] == "shared" else dgate.to(s.gate.dtype)
    return {"dr": g.to(s.r.dtype), "db": db.to(s.b.dtype), "dgate": dgate,
            "dw_block": None if s.w_block is None else (dp * bhat).sum(dim=0), "dc_block": None if s.c_block is None else dp.sum(dim=0),
            "dw_next": (dh * xhat).sum(dim=0), "dc_next": None if s.c_next is None else dh.sum(dim=0)}


def _plain_dropout(s):
    c = s.case
    return {"y": (s.x.float() * _keep(s.random, c["tokens"], c["n"], c["drop"])).to(s.x.dtype)}


def _plain_logprobs(s):
    c, k = s.case, s.case["top"]
    logits = s.logits.float()
    most = logits.amax(dim=1, keepdim=True)
    z = (logits - most) / c["temperature"]
    total = z.exp().sum(dim=1, keepdim=True).log()
    logp = z - total
    target = s.targets.long()
    logprob = torch.where(target < 0, 0.0, logp.gather(1, target.clamp(min=0)[:, None])[:, 0])
    entropy = -(logp.exp() * torch.where(logp == -math.inf, 0.0, logp)).sum(dim=1) if c["entropy"] else None
    ids = None
    if k:
        # ties go to the lowest index: the value's order above the index's
        bits = (logits + 0.0).view(torch.int32).long()
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * (1 << 32) - torch.arange(c["vocab"], device=DEV)
        ids = order.topk(k, dim=1).indices
    return {"logprob": logprob, "stats": torch.cat([most, total], dim=1), "entropy": entropy, "top_ids": None if ids is None else ids.to(torch.int32), "top_logprobs": None if ids is None else logp.gather(1, ids)}


def _plain_logprobs_backward(s):
    c = s.case
    logp = (s.logits.float() - s.stats[:, :1]) / c["temperature"] - s.stats[:, 1:]
    p = logp.exp()
    target = s.targets.long()
    d = torch.where(target < 0, 0.0, s.dlogprob)
    given = d if s.dtop is None else d + s.dtop.sum(dim=1)
    dz = -p * given[:, None]
    if s.entropy is not None:
        dz = dz - p * s.dentropy[:, None] * (torch.where(logp == -math.inf, 0.0, logp) + s.entropy[:, None])
    dz.scatter_add_(1, target.clamp(min=0)[:, None], d[:, None])
    if s.dtop is not None:
        dz.scatter_add_(1, s.top_ids.long(), s.dtop)
    return {"dlogits": (dz / c["temperature"]).to(s.logits.dtype)}


# ---- the framework's calls -----------------------------------------------------------------------
def _ld(v):
    return 0 if v is None or v.dim() < 2 else v.stride(0)


def _calls(s):
    from paper_2608_16308_b200 import binding as B
    c, t = s.case, s.case["tokens"]
    if c["kind"] == "dropout":
        B.dbspmspv_dropout(s.x, _ld(s.x), int(c["f32"]), t, c["n"], c["drop"], s.random, s.y, _ld(s.y))
        return {"y": s.y}
    if c["kind"] == "logprobs":
        B.dbspmspv_logprobs(s.logits, _ld(s.logits), int(c["f32"]), t, c["vocab"], c["temperature"], s.targets, s.logprob, s.entropy, s.stats, c["top"], s.top_ids, s.top_logprobs)
        return {"logprob": s.logprob, "stats": s.stats, "entropy": s.entropy, "top_ids": s.top_ids, "top_logprobs": s.top_logprobs}
    if c["kind"] == "logprobs_backward":
        B.dbspmspv_logprobs_backward(s.logits, _ld(s.logits), int(c["f32"]), t, c["vocab"], c["temperature"], s.targets, s.stats, s.entropy, c["top"], s.top_ids, s.dlogprob, s.dentropy,
                                     s.dtop, s.dlogits, _ld(s.dlogits), int(c["f32"]))
        return {"dlogits": s.dlogits}
    if c["kind"] == "join":
        B.dbspmspv_join(s.opts, t, c["n"], s.r, _ld(s.r), s.b, _ld(s.b), s.w_block, s.c_block, s.gate, _ld(s.gate), s.w_next, s.c_next, s.random, s.out, _ld(s.out), s.h, _ld(s.h), s.stats)
        return {"out": s.out, "h": s.h, "stats": s.stats}
    B.dbspmspv_join_backward(s.opts, t, c["n"], s.r, _ld(s.r), s.b, _ld(s.b), s.stats, s.w_block, s.c_block, s.gate, _ld(s.gate), s.w_next, s.random, s.dh, _ld(s.dh), s.dout, _ld(s.dout),
                             s.dr, _ld(s.dr), s.db, _ld(s.db), s.dw_block, s.dc_block, s.dgate, _ld(s.dgate), s.dw_next, s.dc_next, s.workspace, s.bytes)
    return {"dr": s.dr, "db": s.db, "dgate": s.dgate, "dw_block": s.dw_block, "dc_block": s.dc_block, "dw_next": s.dw_next, "dc_next": s.dc_next}


PLAIN = {"join": _plain_join, "join_backward": _plain_join_backward, "dropout": _plain_dropout, "logprobs": _plain_logprobs, "logprobs_backward": _plain_logprobs_backward}


def run(state):
    return _calls(state) if own else PLAIN[state.case["kind"]](state)


def work(case):
    t = case["tokens"]
    if case["kind"].startswith("logprobs"):
        size = (4 if case["f32"] else 2) * case["vocab"]
        if case["kind"] == "logprobs":
            return {"bytes": t * (size + 20 + 8.0 * case["top"]), "flops": 6.0 * t * case["vocab"]}
        return {"bytes": t * (2 * size + 24 + 8.0 * case["top"]), "flops": 8.0 * t * case["vocab"]}
    n = case["n"]
    if case["kind"] == "dropout":
        return {"bytes": 2.0 * t * n * (4 if case["f32"] else 2) + 16, "flops": 2.0 * t * n}
    st, bt, pt = (4 if case[k] else 2 for k in ("stream_f32", "block_f32", "params_f32"))
    vectors = 1 + (case["norm_block"] != "none")
    vectors += vectors if case["bias"] else 0
    vectors += case["gate"] == "shared"
    rows = t * n * pt if case["gate"] == "token" else 0.0
    if case["kind"] == "join":
        return {"bytes": float(t * n * (2 * st + bt + 2) + rows + vectors * n * pt + (16 * t if case.get("keep") else 0)), "flops": 16.0 * t * n}
    return {"bytes": float(t * n * (3 * st + 2 * bt + 2) + 2 * rows + vectors * n * (pt + 4) + 16 * t), "flops": 32.0 * t * n}


# ---- in 64 bits, from the definitions ------------------------------------------------------------
def _exact_mask(random, t, n, drop):
    """The same generator in unsigned 64-bit arithmetic on the host, a word at a time."""
    if not drop:
        return torch.ones((t, n), dtype=torch.float64, device=DEV)
    seed, offset = (int(v) for v in random.tolist())
    lo, u = np.uint64(0xFFFFFFFF), np.uint64
    x = np.zeros((4, t, (n + 7) // 8), dtype=np.uint64)
    x[0] += np.arange(x.shape[2], dtype=np.uint64)
    x[1] += np.arange(t, dtype=np.uint64)[:, None]
    x[2], x[3] = offset & 0xFFFFFFFF, offset >> 32
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        first, second = x[0] * u(0xD2511F53), x[2] * u(0xCD9E8D57)
        x = np.stack([(second >> u(32)) ^ x[1] ^ u(key[0]), second & lo, (first >> u(32)) ^ x[3] ^ u(key[1]), first & lo])
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    out = np.empty((t, x.shape[2], 8))
    for j in range(8):
        out[:, :, j] = (x[j // 2] >> u(16 * (j % 2))) & u(0xFFFF)
    threshold = math.floor(drop * 65536 + 0.5)
    keep = (out.reshape(t, -1)[:, :n] >= threshold) / (1 - threshold / 65536)
    return torch.from_numpy(keep).to(DEV)


def _normed(x, norm):
    """normalised rows by the definition, with their mean and 1 / deviation"""
    x = x.double()
    zero = torch.zeros(x.shape[0], 1, dtype=torch.float64, device=x.device)
    if norm == "none":
        return x, zero, zero + 1
    mean = x.sum(dim=1, keepdim=True) / x.shape[1] if norm == "layer" else zero
    inv = (EPS + torch.linalg.vector_norm(x - mean, dim=1, keepdim=True) ** 2 / x.shape[1]) ** -0.5
    return (x - mean) * inv, mean, inv


def _exact_join(s, c):
    one = torch.ones((), dtype=torch.float64, device=DEV)
    f = lambda v, other: other if v is None else v.double()  # noqa: E731
    wb, cb, gate, wn, cn = f(s.w_block, one), f(s.c_block, 0 * one), f(s.gate, one), f(s.w_next, one), f(s.c_next, 0 * one)
    mask = c["scale"] * _exact_mask(s.random, c["tokens"], c["n"], c["drop"])
    if c["kind"] == "join":
        y, m0, i0 = _normed(s.b, c["norm_block"])
        out = torch.addcmul(s.r.double(), mask * gate, y * wb + cb)
        h, m1, i1 = _normed(out, c["norm_next"])
        return {"out": out, "h": h * wn + cn, "stats": torch.cat([m0, i0, m1, i1], dim=1) if c.get("keep") else None}
    m0, i0, m1, i1 = s.stats.double().split(1, dim=1)
    width = c["n"]

    def back(u, xh, inv, norm):
        if norm == "none":
            return u
        along = torch.einsum("tn,tn->t", u, xh)[:, None] / width
        mean = u.sum(dim=1, keepdim=True) / width if norm == "layer" else 0.0
        return inv * (u - mean - along * xh)

    dh, xh, bh = s.dh.double(), (s.r.double() - m1) * i1, (s.b.double() - m0) * i0
    dr = s.dout.double() + back(dh * wn, xh, i1, c["norm_next"])
    dy = mask * dr
    db = back(dy * gate * wb, bh, i0, c["norm_block"])
    dgate = None
    if s.gate is not None:
        dgate = dy * (bh * wb + cb)
        dgate = torch.einsum("tn->n", dgate) if c["gate"] == "shared" else dgate
    return {"dr": dr, "db": db, "dgate": dgate, "dw_block": None if s.w_block is None else torch.einsum("tn,tn->n", dy * gate, bh),
            "dc_block": None if s.c_block is None else torch.einsum("tn->n", dy * gate), "dw_next": torch.einsum("tn,tn->n", dh, xh),
            "dc_next": None if s.c_next is None else torch.einsum("tn->n", dh)}


def exact(case, seed):
    """From the definitions, every sum in 64 bits."""
    s, c = _State(case, seed), case
    if c["kind"].startswith("join"):
        return _exact_join(s, c)
    if c["kind"] == "dropout":
        return {"y": s.x.double() * _exact_mask(s.random, c["tokens"], c["n"], c["drop"])}
    z = s.logits.double() / c["temperature"]
    have, target = s.targets >= 0, s.targets.long().clamp(min=0)[:, None]
    if c["kind"] == "logprobs":
        lse = torch.logsumexp(z, dim=1)
        p = torch.softmax(z, dim=1)
        top = z.sort(dim=1, descending=True).values[:, :c["top"]] - lse[:, None] if c["top"] else None
        return {"logprob": (torch.take_along_dim(z, target, 1)[:, 0] - lse) * have if not c["masked"] else torch.where(have, torch.take_along_dim(z, target, 1)[:, 0] - lse, 0.0),
                "stats": torch.stack([s.logits.double().amax(dim=1), lse - z.amax(dim=1)], dim=1), "entropy": torch.special.entr(p).sum(dim=1) if c["entropy"] else None, "top_ids": None, "top_logprobs": top}
    p = torch.exp((s.logits.double() - s.stats[:, :1].double()) / c["temperature"] - s.stats[:, 1:].double())
    weight = torch.zeros_like(z)
    weight.scatter_add_(1, target, (s.dlogprob * have).double()[:, None])
    if c["top"]:
        weight.scatter_add_(1, s.top_ids.long(), s.dtop.double())
    dz = weight - p * weight.sum(dim=1, keepdim=True)
    if c["entropy"]:
        dz -= s.dentropy.double()[:, None] * (p * s.entropy.double()[:, None] - torch.special.entr(p))
    return {"dlogits": dz / c["temperature"]}
