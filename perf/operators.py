"""Cases of three operators next to the decode step: what follows a block of the decoder whose norms are root-mean-square
norms and whose products run in 8 bits with biases and smooth activations, and what answers by drawing instead of ranking.

Kinds of case (`kind`), each one pass through one entry point of the package:
  norm    grace_rms_norm: the residual stream takes a block's output and is normalised, to bf16 or to e4m3 with a scale per row
  linear  grace_linear_act: a product of bf16 or of scaled e4m3 operands with bias, activation and residual in its epilogue
  sample  grace_sample: tokens drawn from (allowed) logits by temperature, top-k, top-p, min-p and given random numbers

`own` false: the definition in elementary torch operations.  `own` true: the library's entry points.

Definitions.
  norm    s = x + delta, rounded to x's type;  n = s / sqrt(mean(s^2) + eps) * gamma;  output n in bf16, or
          scale = max(max|n|, 2^-100) / 448 per row and n / scale in e4m3
  linear  y = act(x_scale[m] w_scale[n] sum_k x[m,k] w[n,k] + bias[n]) + residual[m,n]
  sample  allowed tokens of a row in the order (logit descending, token ascending); kept is the shortest prefix that any of
          the limits leaves: the first top_k; of these the fewest whose weights e^((x - max) / T) reach top_p of the sum of
          the top_k's; those with a weight of at least min_p (the first is always kept).  A draw takes the first kept
          token, in ascending order, at which the running sum of kept weights exceeds u times the whole.  Score = prefix
          score + (logit - lse); log q = logarithm of the drawn token's share of the kept weights.  Temperature 0 draws
          the first of the order.  A row without an allowed token: token 0, score and log q -inf.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import torch

own = False

DEV = "cuda:0"
E4M3 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": E4M3}
SIZE = {"bf16": 2, "f32": 4, "e4m3": 1}
MOST_FLOPS, MOST_LOGITS, MOST_STREAM = 2.35e11, 65536 * 2048, 65536 * 512


def listed():
    return [
        # The stream of a single beam's row in front of a product in 8 bits: latency.
        dict(name="norm_one_row", kind="norm", R=1, D=512, stream="bf16", delta=True, out="e4m3"),
        # The benchmark's step: 32 requests x beam 2048, width 512, bf16 stream, the block's output added on the way.
        dict(name="norm_batch", kind="norm", R=65536, D=512, stream="bf16", delta=True, out="e4m3"),
        # A wide model's fp32 stream with an odd number of rows, bf16 for a product in 16 bits.
        dict(name="norm_wide_f32", kind="norm", R=8191, D=2048, stream="f32", delta=True, out="bf16"),
        # Feed-forward of the smallest searches: one request with beam 16.
        dict(name="linear_few_rows", kind="linear", M=16, N=2048, K=512, x="bf16", act="gelu", bias=True, residual=False, y="bf16"),
        # The benchmark's feed-forward in 8 bits, up ...
        dict(name="linear_up", kind="linear", M=65536, N=2048, K=512, x="e4m3", act="gelu", bias=True, residual=False, y="bf16"),
        # ... and down into the residual stream.
        dict(name="linear_down", kind="linear", M=65536, N=512, K=2048, x="e4m3", act="none", bias=True, residual=True, y="bf16"),
        # The wide model's down projection into an fp32 stream: rows, columns and depth that fill no tile.
        dict(name="linear_wide_odd", kind="linear", M=7003, N=2036, K=8184, x="bf16", act="silu", bias=True, residual=True, y="f32"),
        # First step of a sampled search: the root row of one request draws the beam.
        dict(name="sample_root", kind="sample", B=1, M=1, V=64, draws=16, logits="f32", allowed=0.3, T=1.0, top_k=0, top_p=0.95, min_p=0.0),
        # A later step of the benchmark's sizes, a twentieth of the codebook being children of the beam's node.
        dict(name="sample_allowed", kind="sample", B=32, M=2048, V=2048, draws=1, logits="f32", allowed=0.05, T=0.8, top_k=0, top_p=0.9, min_p=0.0),
        # The same rows without a catalog in the way (rollouts of a model in training), every limit set.
        dict(name="sample_dense", kind="sample", B=32, M=2048, V=2048, draws=1, logits="f32", allowed=1.0, T=1.0, top_k=200, top_p=0.95, min_p=0.02),
        # An odd codebook, odd beams, temperature and min-p alone.
        dict(name="sample_odd", kind="sample", B=7, M=999, V=1001, draws=1, logits="bf16", allowed=1.0, T=1.3, top_k=0, top_p=1.0, min_p=0.05),
        # The largest codebook of a 16-bit token, one row per request.
        dict(name="sample_wide", kind="sample", B=64, M=1, V=65472, draws=1, logits="f32", allowed=1.0, T=0.7, top_k=0, top_p=0.95, min_p=0.0),
    ]


def _spread(rng, lo, hi):
    """An integer of [lo, hi], even over the logarithm."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(["norm", "linear", "sample"])
    if kind == "norm":
        D = _spread(rng, 32, 8192)
        return dict(kind=kind, R=_spread(rng, 1, max(1, min(65536, MOST_STREAM // D))), D=D, stream=rng.choice(["bf16", "f32"]),
                    delta=rng.random() < 0.7, out=rng.choice(["bf16", "e4m3"]))
    if kind == "linear":
        x = rng.choice(["bf16", "e4m3"])
        N, K = _spread(rng, 16, 8192), 16 * _spread(rng, 4, 512)
        if x == "bf16" and rng.random() < 0.3:
            K -= 8
        M = _spread(rng, 1, max(1, min(65536, int(MOST_FLOPS / (2.0 * N * K)))))
        return dict(kind=kind, M=M, N=N, K=K, x=x, act=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]),
                    bias=rng.random() < 0.7, residual=rng.random() < 0.5, y=rng.choice(["bf16", "f32"]))
    V = _spread(rng, 2, 65536)
    allowed = rng.choice([1.0, 1.0, 0.2, 0.05, 0.005])
    rows = _spread(rng, 1, max(1, min(65536, MOST_LOGITS // V)))
    B = _spread(rng, 1, min(rows, 64))
    M = max(1, rows // B)
    draws = _spread(rng, 1, 2048) if B * M <= 64 and rng.random() < 0.5 else 1
    return dict(kind=kind, B=B, M=M, V=V, draws=draws, logits=rng.choice(["f32", "bf16"]), allowed=allowed,
                T=rng.choice([0.0, 0.5, 0.8, 1.0, 1.5]), top_k=rng.choice([0, 0, _spread(rng, 1, V)]),
                top_p=rng.choice([1.0, 0.9, 0.95, 0.5]), min_p=rng.choice([0.0, 0.0, 0.01, 0.1]))


# ---------------------------------------------------------------------------------------------------------------
def _e4m3_rows(a):
    """(e4m3 values, fp32 scale per row) of fp32 rows: the largest magnitude of a row becomes 448."""
    scale = a.abs().amax(1).clamp_min(2.0 ** -100) / 448.0
    return (a / scale[:, None]).to(E4M3), scale


def prepare(case, seed):
    c = SimpleNamespace(**case)
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    normal = lambda *shape: torch.randn(*shape, device=DEV, generator=g)  # noqa: E731
    s = SimpleNamespace(case=c)
    if c.kind == "norm":
        s.x = (normal(c.R, c.D) * 2.0).to(TYPES[c.stream])
        s.delta = normal(c.R, c.D).to(torch.bfloat16) if c.delta else None
        s.gamma = 1.0 + 0.1 * normal(c.D)
        s.x_out = torch.empty_like(s.x) if c.delta else None
        s.out = torch.empty(c.R, c.D, dtype=TYPES[c.out], device=DEV)
        s.scale = torch.empty(c.R, device=DEV) if c.out == "e4m3" else None
    elif c.kind == "linear":
        x, w = normal(c.M, c.K), normal(c.N, c.K) * c.K ** -0.5
        s.x_scale = s.w_scale = None
        if c.x == "e4m3":
            (s.x, s.x_scale), (s.w, s.w_scale) = _e4m3_rows(x), _e4m3_rows(w)
        else:
            s.x, s.w = x.to(torch.bfloat16), w.to(torch.bfloat16)
        s.bias = normal(c.N) * 0.5 if c.bias else None
        s.residual = normal(c.M, c.N).to(TYPES[c.y]) if c.residual else None
        s.y = torch.empty(c.M, c.N, dtype=TYPES[c.y], device=DEV)
    else:
        R = c.B * c.M
        logits = normal(R, c.V) * 3.0
        s.logits = logits.to(TYPES[c.logits])
        s.row_lse = torch.logsumexp(s.logits.float(), 1)
        s.row_score = -10.0 * torch.rand(R, device=DEV, generator=g)
        s.bits = s.allow = None
        if c.allowed < 1.0:
            words = (c.V + 63) // 64
            s.allow = torch.zeros(R, words * 64, dtype=torch.bool, device=DEV)
            s.allow[:, :c.V] = torch.rand(R, c.V, device=DEV, generator=g) < c.allowed
            s.bits = torch.zeros(R, words, dtype=torch.int64, device=DEV)
            for j in range(64):
                s.bits |= s.allow[:, j::64].to(torch.int64) << j
            s.allow = s.allow[:, :c.V].contiguous()
        full = lambda v, t: torch.full((c.B,), v, dtype=t, device=DEV)  # noqa: E731
        s.temperature, s.top_k = full(c.T, torch.float32), full(c.top_k, torch.int32)
        s.top_p, s.min_p = full(c.top_p, torch.float32), full(c.min_p, torch.float32)
        s.u = torch.rand(R, c.draws, device=DEV, generator=g)
        s.score, s.logq = torch.empty(c.B, c.M * c.draws, device=DEV), torch.empty(c.B, c.M * c.draws, device=DEV)
        s.token = torch.empty(c.B, c.M * c.draws, dtype=torch.int32, device=DEV)
        s.parent = torch.empty_like(s.token)
    return s


# ---------------------------------------------------------------------------------------------------------------
def _norm(s):
    c = s.case
    x = s.x
    if s.delta is not None:
        x = (s.x.float() + s.delta.float()).to(s.x.dtype)
    f = x.float()
    n = f / torch.sqrt((f * f).mean(1, keepdim=True) + 1e-6) * s.gamma
    got = {"x": x} if s.delta is not None else {}
    if c.out == "bf16":
        return got | {"y": n.to(torch.bfloat16)}
    scale = n.abs().amax(1).clamp_min(2.0 ** -100) / 448.0
    return got | {"y": (n / scale[:, None]).to(E4M3), "scale": scale}


def _act(v, act):
    if act == "relu":
        return v.clamp_min(0.0)
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _linear(s):
    x, w = s.x.float(), s.w.float()
    if s.x_scale is not None:
        x, w = x * s.x_scale[:, None], w * s.w_scale[:, None]
    v = x @ w.T
    if s.bias is not None:
        v = v + s.bias
    v = _act(v, s.case.act)
    if s.residual is not None:
        v = v + s.residual.float()
    return {"y": v.to(s.y.dtype)}


def _sample(s):
    # In 64 bits: which token a draw takes turns on sums next to a border.
    c = s.case
    R, V = s.logits.shape
    x = s.logits.double()
    if s.allow is not None:
        x = torch.where(s.allow, x, float("-inf"))
    per_row = lambda v: v.repeat_interleave(c.M)[:, None]  # noqa: E731
    T, k, p, q = per_row(s.temperature).double(), per_row(s.top_k), per_row(s.top_p).double(), per_row(s.min_p).double()
    top = x.amax(1, keepdim=True)
    dead = top == float("-inf")
    z = torch.where(x > float("-inf"), (x - torch.where(dead, 0.0, top)) / torch.where(T > 0, T, 1.0), float("-inf"))
    w = torch.exp(z)
    _, order = torch.sort(x, dim=1, descending=True, stable=True)
    ws = w.gather(1, order)
    place = torch.arange(V, device=x.device)
    keep = (place < torch.where((k > 0) & (T > 0), k, torch.where(T > 0, V, 1))) & (ws > 0)
    mass = torch.cumsum(ws * keep, 1)
    before = torch.cat([torch.zeros_like(mass[:, :1]), mass[:, :-1]], 1)
    keep &= (before < p * mass[:, -1:]) | (p >= 1.0) | (place == 0)
    keep &= (ws >= q) | (place == 0)
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ws, 0.0))
    run = torch.cumsum(kept, 1)
    whole = run[:, -1:]
    token = torch.searchsorted(run, s.u.double() * whole, right=True)
    token = torch.where(dead, 0, token.clamp_max(V - 1))
    at = s.logits.float().gather(1, token)
    score = torch.where(dead, float("-inf"), s.row_score[:, None] + (at - s.row_lse[:, None]))
    logq = torch.where(dead, float("-inf"), torch.log(kept.gather(1, token) / whole)).float()
    parent = torch.arange(c.M, device=x.device, dtype=torch.int32).repeat(c.B).repeat_interleave(c.draws)
    shape = s.token.shape
    return {"score": score.reshape(shape), "logq": logq.reshape(shape), "token": token.to(torch.int32).reshape(shape), "parent": parent.reshape(shape)}


def run(s):
    c = s.case
    if not own:
        return {"norm": _norm, "linear": _linear, "sample": _sample}[c.kind](s)
    from paper_2608_00938_b200 import api
    if c.kind == "norm":
        api.grace_rms_norm(s.x, s.gamma, s.out, 1e-6, delta=s.delta, x_out=s.x_out, scale=s.scale)
        got = {"x": s.x_out} if s.delta is not None else {}
        return got | ({"y": s.out} if s.scale is None else {"y": s.out, "scale": s.scale})
    if c.kind == "linear":
        api.grace_linear_act(s.x, s.w, s.y, bias=s.bias, act=c.act, residual=s.residual, x_scale=s.x_scale, w_scale=s.w_scale)
        return {"y": s.y}
    api.grace_sample(s.logits, s.u, s.score, s.token, c.B, c.M, allow_bits=s.bits, row_score=s.row_score, row_lse=s.row_lse,
                     temperature=s.temperature, top_k=s.top_k, top_p=s.top_p, min_p=s.min_p, out_logq=s.logq, out_parent=s.parent)
    return {"score": s.score, "logq": s.logq, "token": s.token, "parent": s.parent}


def work(case):
    c = SimpleNamespace(**case)
    if c.kind == "norm":
        per = SIZE[c.stream] * (2 if c.delta else 1) + (2 if c.delta else 0) + SIZE[c.out]
        return {"bytes": c.R * c.D * per + 4 * c.D + (4 * c.R if c.out == "e4m3" else 0), "flops": 7 * c.R * c.D}
    if c.kind == "linear":
        by = SIZE[c.x] * (c.M + c.N) * c.K + SIZE[c.y] * c.M * c.N * (2 if c.residual else 1)
        return {"bytes": by + (4 * c.N if c.bias else 0) + (4 * (c.M + c.N) if c.x == "e4m3" else 0), "flops": 2 * c.M * c.N * c.K}
    R, draws = c.B * c.M, c.draws
    by = SIZE[c.logits] * c.allowed * R * c.V + (8 * R * ((c.V + 63) // 64) if c.allowed < 1.0 else 0)
    return {"bytes": by + R * (8 + 20 * draws) + 16 * c.B, "flops": 4 * c.allowed * R * c.V}


# ---------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    """The definitions in 64 bits, row by row of the text above: norms and products on whole arrays, the kept set of a
    sampled row by its smallest value and the number of its ties that stay."""
    s = prepare(case, seed)
    c = s.case
    if c.kind == "norm":
        x = s.x.double()
        got = {}
        if s.delta is not None:
            total = x + s.delta.double()
            got["x"] = total
            # what is normalised is the stream as it is stored
            x = (s.x.float() + s.delta.float()).to(s.x.dtype).double()
        n = x * torch.rsqrt(x.square().sum(1, keepdim=True) / c.D + 1e-6) * s.gamma.double()
        if c.out == "bf16":
            return got | {"y": n}
        scale = n.abs().max(1).values.clamp_min(2.0 ** -100) / 448.0
        return got | {"y": n / scale[:, None], "scale": scale}
    if c.kind == "linear":
        y = torch.empty(c.M, c.N, dtype=torch.float64, device=DEV)
        w = s.w.double()
        for m in range(0, c.M, 8192):
            v = torch.matmul(s.x[m:m + 8192].double(), w.t())
            if s.x_scale is not None:
                v *= s.x_scale[m:m + 8192, None].double() * s.w_scale.double()
            if s.bias is not None:
                v += s.bias.double()
            if c.act == "relu":
                v = torch.where(v > 0, v, 0.0)
            elif c.act == "gelu":
                v = v * torch.special.erfc(-v / math.sqrt(2.0)) / 2.0
            elif c.act == "gelu_tanh":
                v = v * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3))
            elif c.act == "silu":
                v = v * torch.sigmoid(v)
            if s.residual is not None:
                v += s.residual[m:m + 8192].double()
            y[m:m + 8192] = v
        return {"y": y}
    R = c.B * c.M
    score, logq = (torch.empty(R, c.draws, dtype=torch.float64, device=DEV) for _ in range(2))
    block = max(1, (1 << 25) // c.V)
    for r in range(0, R, block):
        raw = s.logits[r:r + block].double()
        x = raw if s.allow is None else raw.masked_fill(~s.allow[r:r + block], float("-inf"))
        live = torch.isfinite(x).any(1, keepdim=True)
        top = torch.where(live, x.max(1, keepdim=True).values, 0.0)
        down = torch.sort(x, 1, descending=True).values
        n = torch.isfinite(down).sum(1, keepdim=True)
        if c.T == 0:
            n = n.clamp_max(1)
        elif c.top_k > 0:
            n = n.clamp_max(c.top_k)
        place = torch.arange(c.V, device=DEV)
        T = float(torch.tensor(c.T)) if c.T else 1.0
        share = torch.softmax(torch.where(place < n, (down - top) / T, float("-inf")), 1) if c.V > 1 else torch.ones_like(down)
        p, q = float(torch.tensor(c.top_p)), float(torch.tensor(c.min_p))
        if p < 1.0:
            n = torch.minimum(n, (share.cumsum(1) < p).sum(1, keepdim=True) + 1)
        n = torch.minimum(n, ((share >= q * share[:, :1]) & (place < n)).sum(1, keepdim=True).clamp_min(1))
        least = down.gather(1, (n - 1).clamp_min(0))
        ties = n - (down > least).sum(1, keepdim=True)
        kept = (x > least) | ((x == least) & ((x == least).cumsum(1) <= ties))
        share = torch.where(kept & live, torch.exp((x - top) / T), 0.0)
        running = share.cumsum(1)
        for i in range(c.draws):
            u = s.u[r:r + block, i:i + 1].double()
            token = (running > u * running[:, -1:]).to(torch.uint8).argmax(1, keepdim=True)
            logq[r:r + block, i:i + 1] = torch.where(live, (x.gather(1, token) - top) / T - torch.log(running[:, -1:]), float("-inf"))
            value = s.row_score[r:r + block, None].double() + (raw.gather(1, token) - s.row_lse[r:r + block, None].double())
            score[r:r + block, i:i + 1] = torch.where(live, value, float("-inf"))
    return {"score": score.reshape(c.B, -1), "logq": logq.reshape(c.B, -1), "token": None, "parent": None}
