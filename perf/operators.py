"""Operators around the stage's blocks: what is measured of them, and their plain form.

Three groups that a training program meets between its token ids and its
gradients: the embedding lookup with scaling and its gradient by sorted tokens;
the RMS norm of each head's queries and keys with the position rotation in the
same pass, and its gradient; activation checkpoints in 8 bits (e4m3 values, one
power-of-two scale for each 32 features of a token), what they restore to, and
the two gradients that are taken straight from them (GeLU's and a linear
layer's weights').

A case is a dict of plain values; ``kind`` names the call and the other keys
are its sizes.  Inputs are drawn on the GPU from the seed alone.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
BLOCK = 32            # features of a token that share one scale
E4M3_MAX = 448.0
MIN_EXP, MAX_EXP = -117, 120   # exponents that a scale can have (stored + 127)
EPS = 1e-6
THETA = 10000.0


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # One token of a decode step or a check: nothing but latency.
        {"name": "embed-fwd-1x1600", "kind": "embed_fwd", "tokens": 1, "hidden": 1600, "rows": 50304, "vocab": 50304,
         "first": 0, "ids": "int64", "pad": 0.0, "dtype": "bf16"},
        # The first stage's input for a whole global batch, 16 sequences of 2048.
        {"name": "embed-fwd-32768x6144", "kind": "embed_fwd", "tokens": 32768, "hidden": 6144, "rows": 50304,
         "vocab": 50304, "first": 0, "ids": "int64", "pad": 0.0, "dtype": "bf16"},
        # A short, partly padded batch on one of eight tensor-parallel ranks'
        # share of the vocabulary, in the fp32 mode a user checks a model with.
        {"name": "embed-bwd-96x1000-fp32", "kind": "embed_bwd", "tokens": 96, "hidden": 1000, "rows": 6288,
         "vocab": 50304, "first": 12576, "ids": "int32", "pad": 0.25, "dtype": "fp32"},
        # The gradient of one of two ranks' share of the vocabulary, 16 sequences
        # of 1024 tokens: a few tokens are most of the text.
        {"name": "embed-bwd-16384x1920", "kind": "embed_bwd", "tokens": 16384, "hidden": 1920, "rows": 25152,
         "vocab": 50304, "first": 25152, "ids": "int64", "pad": 0.0, "dtype": "bf16"},
        # One token far into a sequence, 25 heads of 64.
        {"name": "qk-fwd-1x25x64", "kind": "qk_fwd", "tokens": 1, "q_heads": 25, "kv_heads": 25, "d": 64, "rope": 64,
         "interleaved": False, "table": 131072, "seq": 0, "dtype": "bf16"},
        # The whole micro-batch of a stage, 20 heads of 96.
        {"name": "qk-fwd-32768x20x96", "kind": "qk_fwd", "tokens": 32768, "q_heads": 20, "kv_heads": 20, "d": 96,
         "rope": 96, "interleaved": False, "table": 2048, "seq": 2048, "dtype": "bf16"},
        # Packed documents of any length in the fp32 check mode: four queries
        # to a key head, half of each head rotated, neighbouring pairs.
        {"name": "qk-bwd-1023x24+6x128-fp32", "kind": "qk_bwd", "tokens": 1023, "q_heads": 24, "kv_heads": 6, "d": 128,
         "rope": 64, "interleaved": True, "table": 4096, "seq": 0, "dtype": "fp32"},
        # The backward pass of 16 sequences of 1024 tokens, 25 heads of 64.
        {"name": "qk-bwd-16384x25x64", "kind": "qk_bwd", "tokens": 16384, "q_heads": 25, "kv_heads": 25, "d": 64,
         "rope": 64, "interleaved": False, "table": 1024, "seq": 1024, "dtype": "bf16"},
        # A block's input kept in 8 bits and restored for its recomputation.
        {"name": "act8-keep-16384x6144", "kind": "act8_keep", "rows": 16384, "cols": 6144, "dtype": "bf16"},
        # GeLU's gradient, and its output again, from the 8-bit input: an odd
        # number of tokens by an FFN of 6400.
        {"name": "act8-gelu-8191x6400", "kind": "act8_gelu", "rows": 8191, "cols": 6400, "dtype": "bf16"},
        # Weight gradient of a narrow shard over a short ragged batch.
        {"name": "act8-dw-333x1920x640", "kind": "act8_dw", "tokens": 333, "n_out": 1920, "n_in": 640, "dtype": "bf16"},
        # Weight gradient of the 2.5B-shaped FFN's first layer over 16 sequences.
        {"name": "act8-dw-16384x7680x1920", "kind": "act8_dw", "tokens": 16384, "n_out": 7680, "n_in": 1920,
         "dtype": "bf16"},
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of step in [lo, hi], spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(-(-lo // step) * step, min(hi // step * step, step * round(v / step)))


_KINDS = ("embed_fwd", "embed_bwd", "qk_fwd", "qk_bwd", "act8_keep", "act8_gelu", "act8_dw")


def draw(rng):
    kind = rng.choice(_KINDS)
    most = max((work(c) for c in listed() if c["kind"] == kind), key=lambda w: w["bytes"] + w["flops"])
    while True:
        case = _draw(rng, kind)
        w = work(case)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return case


def _draw(rng, kind):
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if kind in ("embed_fwd", "embed_bwd"):
        vocab = _log(rng, 1000, 60000)
        ranks = rng.choice([1, 1, 2, 4, 8])
        rows = -(-vocab // ranks)
        return {"kind": kind, "tokens": _log(rng, 1, 32768), "hidden": _log(rng, 64, 6144, 8), "rows": rows,
                "vocab": vocab, "first": rows * rng.randrange(ranks), "ids": rng.choice(["int32", "int64"]),
                "pad": rng.choice([0.0, 0.0, 0.25]), "dtype": dtype}
    if kind in ("qk_fwd", "qk_bwd"):
        kv = rng.randint(1, 25)
        d = rng.choice([64, 96, 128, 128, 80, 256])
        seq = rng.choice([0, 1]) and _log(rng, 1, 4096)
        return {"kind": kind, "tokens": _log(rng, 1, 32768), "q_heads": kv * rng.choice([1, 1, 4]), "kv_heads": kv,
                "d": d, "rope": rng.choice([d, d, 16 * (d // 32)]), "interleaved": rng.random() < 0.3,
                "table": seq or rng.choice([4096, 131072]), "seq": seq, "dtype": dtype}
    if kind == "act8_dw":
        return {"kind": kind, "tokens": _log(rng, 1, 32768), "n_out": _log(rng, 64, 8192, 8),
                "n_in": _log(rng, 64, 8192, 32), "dtype": dtype}
    return {"kind": kind, "rows": _log(rng, 1, 32768), "cols": _log(rng, 64, 8192, 32), "dtype": dtype}


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def _zipf(n):
    p = 1.0 / np.arange(1, n + 1)
    return p / p.sum()


def _token_rows(case):
    """Expected (tokens, distinct tokens) that lie in the case's rows of the table."""
    real = case["tokens"] * (1.0 - case["pad"])
    seen = float(np.sum(-np.expm1(real * np.log1p(-np.minimum(_zipf(case["vocab"]), 1 - 1e-12)))))
    share = min(case["rows"], case["vocab"] - case["first"]) / case["vocab"]
    return real * share, seen * share


def work(case):
    k = case["kind"]
    e = 2 if case["dtype"] == "bf16" else 4
    if k in ("embed_fwd", "embed_bwd"):
        T, H = case["tokens"], case["hidden"]
        ids = T * (8 if case["ids"] == "int64" else 4)
        mine, seen = _token_rows(case)
        if k == "embed_fwd":
            return {"bytes": int(ids + seen * H * e + T * H * e), "flops": int(mine * H)}
        return {"bytes": int(ids + mine * H * e + case["rows"] * H * 4), "flops": int(2 * mine * H)}
    if k in ("qk_fwd", "qk_bwd"):
        T, q, kv, d = case["tokens"], case["q_heads"], case["kv_heads"], case["d"]
        # the rows of the table that the positions can name, and the positions
        small = (0 if case["seq"] else T * 4) + min(T, case["table"]) * case["rope"] * 4 + 2 * d * e
        if k == "qk_fwd":
            return {"bytes": T * (q + 2 * kv) * d * e * 2 + small, "flops": T * (q + kv) * d * 7}
        # the raw queries and keys are read, the raw values are not
        return {"bytes": T * ((q + 2 * kv) * 2 + q + kv) * d * e + small + 2 * d * 4, "flops": T * (q + kv) * d * 16}
    if k == "act8_dw":
        T, n, m = case["tokens"], case["n_out"], case["n_in"]
        return {"bytes": T * n * e + T * m + T * m // BLOCK + n * m * 4, "flops": 2 * T * n * m}
    n = case["rows"] * case["cols"]
    if k == "act8_keep":
        return {"bytes": 2 * (n * e + n + n // BLOCK), "flops": 4 * n}
    return {"bytes": 3 * n * e + n + n // BLOCK, "flops": 20 * n}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

class _Draws:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, *shape, std=1.0, mean=0.0, dtype=torch.float32):
        v = torch.randn(*shape, generator=self.g, device=DEV, dtype=torch.float32)
        return v.mul_(std).add_(mean).to(dtype)

    def uniform(self, n):
        return torch.rand(n, generator=self.g, device=DEV, dtype=torch.float64)

    def below(self, n, count):
        return torch.randint(0, n, (count,), generator=self.g, device=DEV)

    def permutation(self, n):
        return torch.argsort(torch.rand(n, generator=self.g, device=DEV))


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _ids(case, d):
    """Tokens of a text: the r-th most frequent one 1/r as often as the first, in any
    order of ids; padding is -1."""
    cdf = torch.from_numpy(np.cumsum(_zipf(case["vocab"]))).to(DEV)
    rank = torch.searchsorted(cdf, d.uniform(case["tokens"])).clamp_(max=case["vocab"] - 1)
    ids = d.permutation(case["vocab"])[rank]
    if case["pad"]:
        ids = torch.where(d.uniform(case["tokens"]) < case["pad"], torch.full_like(ids, -1), ids)
    return ids.to(torch.int32 if case["ids"] == "int32" else torch.int64)


def _activations(rows, cols, d, dtype):
    """Hidden states: most features of order 1, a few channels many times larger."""
    gain = torch.where(d.uniform(cols) < 0.01, 20.0, 1.0).float()
    return (d.normal(rows, cols) * gain).to(dtype)


def _positions(case, d):
    """Packed documents: each token counts from its document's start, some of which
    begin far into the table (a continued document)."""
    T, P = case["tokens"], case["table"]
    t = torch.arange(T, device=DEV)
    start = d.uniform(T) < 1.0 / 300.0
    start[0] = True
    last = torch.cummax(torch.where(start, t, torch.zeros_like(t)), 0)[0]
    return ((t - last + d.below(P, T)[last]) % P).to(torch.int32)


def _table(positions, rope):
    """cos and sin of position * theta^(-2 i / rope), [positions, rope / 2, 2]."""
    i = torch.arange(rope // 2, device=DEV, dtype=torch.float64)
    a = torch.arange(positions, device=DEV, dtype=torch.float64)[:, None] * THETA ** (-2.0 * i / rope)
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def prepare(case, seed):
    d = _Draws(seed)
    dt = _dtype(case)
    k = case["kind"]
    s = {"case": case, "kind": k}
    if k in ("embed_fwd", "embed_bwd"):
        s["ids"] = _ids(case, d)
        s["scale"] = math.sqrt(case["hidden"])
        if k == "embed_fwd":
            s["table"] = d.normal(case["rows"], case["hidden"], std=0.02, dtype=dt)
        else:
            s["dy"] = d.normal(case["tokens"], case["hidden"], dtype=dt)
    elif k in ("qk_fwd", "qk_bwd"):
        T, q, kv, hd = case["tokens"], case["q_heads"], case["kv_heads"], case["d"]
        s["qkv"] = d.normal(T, q + 2 * kv, hd, dtype=dt)
        s["gq"], s["gk"] = d.normal(hd, std=0.1, mean=1.0, dtype=dt), d.normal(hd, std=0.1, mean=1.0, dtype=dt)
        s["table"] = _table(case["table"], case["rope"])
        s["positions"] = None if case["seq"] else _positions(case, d)
        if k == "qk_bwd":
            s["dout"] = d.normal(T, q + 2 * kv, hd, dtype=dt)
    elif k == "act8_dw":
        s["dy"] = d.normal(case["tokens"], case["n_out"], dtype=dt)
        s["q"], s["scales"] = _codes(_activations(case["tokens"], case["n_in"], d, dt))
    else:
        x = _activations(case["rows"], case["cols"], d, dt)
        if k == "act8_keep":
            s["x"] = x
        else:
            s["q"], s["scales"] = _codes(x)
            s["dg"] = d.normal(case["rows"], case["cols"], dtype=dt)
    if own:
        _buffers(s)
    return s


def _buffers(s):
    """The outputs and workspaces that a program keeps from step to step."""
    from paper_2206_04959_amd import binding as B
    case, k, dt = s["case"], s["kind"], _dtype(s["case"])
    new = lambda *shape, dtype=dt: torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
    b = {}
    if k == "embed_fwd":
        b["y"] = new(case["tokens"], case["hidden"])
    elif k == "embed_bwd":
        b["dtable"] = new(case["rows"], case["hidden"], dtype=torch.float32)
        b["scratch"] = new(B.embedding_scratch_bytes(case["tokens"], case["hidden"]), dtype=torch.uint8)
    elif k == "qk_fwd":
        b["out"] = torch.empty_like(s["qkv"])
    elif k == "qk_bwd":
        b["dqkv"] = torch.empty_like(s["qkv"])
        b["dgq"], b["dgk"] = new(case["d"], dtype=torch.float32), new(case["d"], dtype=torch.float32)
        b["scratch"] = new(B.qk_norm_rope_scratch_elems(case["tokens"], case["q_heads"], case["kv_heads"], case["d"]),
                           dtype=torch.float32)
    elif k == "act8_keep":
        b["q"] = new(case["rows"], case["cols"], dtype=torch.uint8)
        b["scales"] = new(case["rows"], case["cols"] // BLOCK, dtype=torch.uint8)
        b["y"] = new(case["rows"], case["cols"])
    elif k == "act8_gelu":
        b["du"], b["g"] = new(case["rows"], case["cols"]), new(case["rows"], case["cols"])
    else:
        b["dw"] = new(case["n_out"], case["n_in"], dtype=torch.float32)
        b["scratch"] = new(B.act8_gemm_dw_scratch_bytes(s["dy"].dtype, case["tokens"], case["n_out"], case["n_in"]),
                           dtype=torch.uint8)
    s["buf"] = b
    return b


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _PLAIN[s["kind"]](s)


def _run_own(s):
    from paper_2206_04959_amd import binding as B
    case, k = s["case"], s["kind"]
    b = s.get("buf") or _buffers(s)
    if k == "embed_fwd":
        B.embedding_fwd(s["ids"], s["table"], b["y"], scale=s["scale"], first_id=case["first"])
        return b["y"]
    if k == "embed_bwd":
        B.embedding_bwd(s["ids"], s["dy"], b["dtable"], b["scratch"], scale=s["scale"], first_id=case["first"])
        return b["dtable"]
    if k in ("qk_fwd", "qk_bwd"):
        shape = dict(q_heads=case["q_heads"], kv_heads=case["kv_heads"], positions=s["positions"],
                     seq_len=case["seq"] or None, interleaved=case["interleaved"], eps=EPS)
        if k == "qk_fwd":
            B.qk_norm_rope_fwd(s["qkv"], s["gq"], s["gk"], s["table"], b["out"], **shape)
            return b["out"]
        B.qk_norm_rope_bwd(s["dout"], s["qkv"], s["gq"], s["gk"], s["table"], b["dqkv"], b["dgq"], b["dgk"],
                           b["scratch"], **shape)
        return {"dqkv": b["dqkv"], "dgq": b["dgq"], "dgk": b["dgk"]}
    if k == "act8_keep":
        B.act8_save(s["x"], b["q"], b["scales"])
        B.act8_restore(b["q"], b["scales"], b["y"])
        return b["y"]
    if k == "act8_gelu":
        B.act8_gelu_bwd(s["dg"], s["q"], s["scales"], b["du"], b["g"])
        return {"du": b["du"], "g": b["g"]}
    B.act8_gemm_dw(s["dy"], s["q"], s["scales"], b["dw"], b["scratch"])
    return b["dw"]


# ---------------------------------------------------------------------------
# The plain form: elementary torch operations in 32 bits
# ---------------------------------------------------------------------------

def _plain_embed_fwd(s):
    c = s["case"]
    row = s["ids"].long() - c["first"]
    here = (row >= 0) & (row < c["rows"])
    y = s["table"][torch.where(here, row, torch.zeros_like(row))].float() * s["scale"]
    return torch.where(here[:, None], y, torch.zeros_like(y)).to(_dtype(c))


def _plain_embed_bwd(s):
    c = s["case"]
    row = s["ids"].long() - c["first"]
    here = (row >= 0) & (row < c["rows"])
    row = torch.where(here, row, torch.full_like(row, c["rows"]))  # one row more, for what is not here
    out = torch.zeros((c["rows"] + 1, c["hidden"]), dtype=torch.float32, device=DEV)
    return out.index_add_(0, row, s["dy"].float() * s["scale"])[:-1]


def _angles(s):
    """cos and sin of each token, [tokens, 1, rope / 2]."""
    c = s["case"]
    pos = s["positions"].long() if s["positions"] is not None else torch.arange(c["tokens"], device=DEV) % c["seq"]
    cs = s["table"][pos][:, None]
    return cs[..., 0], cs[..., 1]


def _halves(x, rope, interleaved):
    """The two members of each rotated pair, and what is not rotated."""
    if interleaved:
        return x[..., 0:rope:2], x[..., 1:rope:2], x[..., rope:]
    return x[..., :rope // 2], x[..., rope // 2:rope], x[..., rope:]


def _whole(a, b, rest, interleaved):
    ab = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([ab, rest], -1)


def _plain_qk_fwd(s):
    c = s["case"]
    q, kv, rope, inter = c["q_heads"], c["kv_heads"], c["rope"], c["interleaved"]
    cos, sin = _angles(s)
    parts = []
    for x, gain in ((s["qkv"][:, :q].float(), s["gq"].float()), (s["qkv"][:, q:q + kv].float(), s["gk"].float())):
        n = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain
        a, b, rest = _halves(n, rope, inter)
        parts.append(_whole(a * cos - b * sin, b * cos + a * sin, rest, inter).to(_dtype(c)))
    return torch.cat(parts + [s["qkv"][:, q + kv:]], 1)


def _plain_qk_bwd(s):
    c = s["case"]
    q, kv, rope, inter = c["q_heads"], c["kv_heads"], c["rope"], c["interleaved"]
    cos, sin = _angles(s)
    parts, gains = [], []
    for lo, hi, gain in ((0, q, s["gq"].float()), (q, q + kv, s["gk"].float())):
        x, dy = s["qkv"][:, lo:hi].float(), s["dout"][:, lo:hi].float()
        rstd = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        xn = x * rstd
        a, b, rest = _halves(dy, rope, inter)
        dn = _whole(a * cos + b * sin, b * cos - a * sin, rest, inter)
        gains.append((dn * xn).sum((0, 1)))
        dn = dn * gain
        parts.append((rstd * (dn - xn * (dn * xn).mean(-1, keepdim=True))).to(_dtype(c)))
    return {"dqkv": torch.cat(parts + [s["dout"][:, q + kv:]], 1), "dgq": gains[0], "dgk": gains[1]}


def _pow2(e):
    """2^e in 32 bits, from the exponent's bits; -126 <= e <= 127."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _split8(x):
    """x [rows, cols] in 8 bits: the values in units of each block's scale, and the
    scales' exponents.  The scale is the smallest power of two that brings the
    block's largest finite magnitude to 448 or less."""
    b = x.float().reshape(x.shape[0], -1, BLOCK)
    finite = torch.isfinite(b)
    m, e = torch.frexp(torch.where(finite, b, torch.zeros_like(b)).abs().amax(-1))   # |x| = m 2^e, 1/2 <= m < 1
    exp = e - 9 + (m > 0.875).int()
    exp = torch.where(m > 0, exp, torch.full_like(exp, MIN_EXP)).clamp(MIN_EXP, MAX_EXP)
    v = b * _pow2(-exp)[..., None]
    # round to nearest, ties to even: steps of 2^-3 of the value's power of two, at least 2^-9
    step = _pow2(torch.clamp(torch.frexp(v)[1] - 1, -6, 8) - 3)
    r = torch.where(finite, torch.round(v / step) * step, torch.full_like(v, float("nan")))
    return r, exp


def _codes(x):
    """What the checkpoint of x holds: e4m3 codes and biased scale exponents."""
    r, exp = _split8(x)
    return r.to(torch.float8_e4m3fn).view(torch.uint8).reshape(x.shape), (exp + 127).to(torch.uint8)


def _values(q, scales):
    v = q.view(torch.float8_e4m3fn).float().reshape(*scales.shape, BLOCK)
    return (v * _pow2(scales.int() - 127)[..., None]).reshape(q.shape)


def _plain_act8_keep(s):
    r, exp = _split8(s["x"])
    return (r * _pow2(exp)[..., None]).reshape(s["x"].shape).to(s["x"].dtype)


_GELU_C, _GELU_A = math.sqrt(2.0 / math.pi), 0.044715


def _plain_act8_gelu(s):
    u = _values(s["q"], s["scales"])
    t = torch.tanh(_GELU_C * (u + _GELU_A * u * u * u))
    slope = 0.5 * (1.0 + t) + 0.5 * u * (1.0 - t * t) * _GELU_C * (1.0 + 3.0 * _GELU_A * u * u)
    dt = s["dg"].dtype
    return {"du": (s["dg"].float() * slope).to(dt), "g": (0.5 * u * (1.0 + t)).to(dt)}


def _plain_act8_dw(s):
    return s["dy"].float().t() @ _values(s["q"], s["scales"])


_PLAIN = {"embed_fwd": _plain_embed_fwd, "embed_bwd": _plain_embed_bwd, "qk_fwd": _plain_qk_fwd,
          "qk_bwd": _plain_qk_bwd, "act8_keep": _plain_act8_keep, "act8_gelu": _plain_act8_gelu,
          "act8_dw": _plain_act8_dw}


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    k = case["kind"]
    if k == "embed_fwd":
        y = torch.zeros((case["tokens"], case["hidden"]), dtype=torch.float64, device=DEV)
        idx = s["ids"].long() - case["first"]
        mine = ((idx >= 0) & (idx < case["rows"])).nonzero()[:, 0]
        y[mine] = s["table"][idx[mine]].double() * s["scale"]
        return y
    if k == "embed_bwd":
        idx = s["ids"].long() - case["first"]
        mine = ((idx >= 0) & (idx < case["rows"])).nonzero()[:, 0]
        out = torch.zeros((case["rows"], case["hidden"]), dtype=torch.float64, device=DEV)
        out.index_put_((idx[mine],), s["dy"][mine].double() * s["scale"], accumulate=True)
        return out
    if k in ("qk_fwd", "qk_bwd"):
        return _exact_qk(case, s)
    if k == "act8_dw":
        return torch.mm(s["dy"].double().t(), _exact_values(s["q"], s["scales"]))
    if k == "act8_keep":
        x = s["x"].double()
        blocks = x.reshape(case["rows"], -1, BLOCK)
        most = blocks.abs().max(-1)[0].clamp_min(1e-300)
        exp = torch.ceil(torch.log2(most / E4M3_MAX) - 1e-12).clamp(MIN_EXP, MAX_EXP)
        scale = ((exp.long() + 1023) << 52).view(torch.float64)[..., None]
        return ((blocks / scale).float().to(torch.float8_e4m3fn).double() * scale).reshape(x.shape)
    u = _exact_values(s["q"], s["scales"])
    cdf = torch.sigmoid(2.0 * _GELU_C * (u + _GELU_A * u ** 3))
    slope = cdf + u * cdf * (1.0 - cdf) * 2.0 * _GELU_C * (1.0 + 3.0 * _GELU_A * u ** 2)
    return {"du": s["dg"].double() * slope, "g": u * cdf}


def _exact_values(q, scales):
    v = q.view(torch.float8_e4m3fn).double()
    return v * ((scales.long() + (1023 - 127)) << 52).view(torch.float64).repeat_interleave(BLOCK, dim=1)


def _exact_qk(case, s):
    """Each rotated pair as one complex number."""
    T, q, kv, rope = case["tokens"], case["q_heads"], case["kv_heads"], case["rope"]
    pos = torch.arange(T, device=DEV).remainder(case["seq"]) if case["seq"] else s["positions"].long()
    turn = torch.view_as_complex(s["table"].double())[pos].unsqueeze(1)
    gain = torch.cat([s["gq"].double().expand(q, -1), s["gk"].double().expand(kv, -1)])
    x = s["qkv"][:, :q + kv].double()

    def rotate(v, by):
        out = v.clone()
        p = v[..., :rope]
        z = (p.reshape(*p.shape[:-1], -1, 2) if case["interleaved"]
             else p.reshape(*p.shape[:-1], 2, -1).transpose(-1, -2))
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * by)
        out[..., :rope] = (z if case["interleaved"] else z.transpose(-1, -2)).reshape(p.shape)
        return out

    norm = torch.sqrt((x * x).sum(-1, keepdim=True) / case["d"] + EPS)
    unit = x / norm
    if case["kind"] == "qk_fwd":
        return torch.cat([rotate(unit * gain, turn), s["qkv"][:, q + kv:].double()], 1)
    back = rotate(s["dout"][:, :q + kv].double(), turn.conj())
    dgain = (back * unit).sum(0)
    back = back * gain
    dx = (back - unit * (back * unit).sum(-1, keepdim=True) / case["d"]) / norm
    return {"dqkv": torch.cat([dx, s["dout"][:, q + kv:].double()], 1), "dgq": dgain[:q].sum(0), "dgk": dgain[q:].sum(0)}
