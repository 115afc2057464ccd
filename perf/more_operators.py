"""Operators at the end of a model: what is measured of them, and their plain form.

Two groups.  The residual's addition with the root-mean-square norm of the sum, whose
output is also kept in 8 bits (e4m3 values, one power-of-two scale for each 32
features of a token) for the weight gradient of the layer behind it, and its
gradient.  The loss of a student that learns from a teacher's largest logits and
from labels, and the gradient of the student's logits, on the whole vocabulary or
on the shares of tensor-parallel ranks.

A case is a dict of plain values; ``kind`` names the call and the other keys
are its sizes.  Inputs are drawn on the GPU from the seed alone.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
BLOCK = 32            # features of a token that share one scale
E4M3_MAX = 448.0
MIN_EXP, MAX_EXP = -117, 120   # exponents that a scale can have (stored + 127)
EPS = 1e-6


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # One token of a check or a decode step: nothing but latency.
        {"name": "norm-fwd-1x1600", "kind": "norm_fwd", "rows": 1, "cols": 1600, "resid": True, "dtype": "bf16"},
        # The norm before a block's FFN, 16 sequences of 2048.
        {"name": "norm-fwd-32768x6144", "kind": "norm_fwd", "rows": 32768, "cols": 6144, "resid": True,
         "dtype": "bf16"},
        # The same kept in 8 bits for the weight gradient, 16 sequences of 1024; restored as a
        # recomputation would.
        {"name": "norm-keep8-16384x1920", "kind": "norm_keep8", "rows": 16384, "cols": 1920, "resid": True,
         "dtype": "bf16"},
        # Packed documents of any length in the fp32 mode a user checks a model with; the first
        # norm of a model, without a residual.
        {"name": "norm-keep8-1001x6400-fp32", "kind": "norm_keep8", "rows": 1001, "cols": 6400, "resid": False,
         "dtype": "fp32"},
        # A short ragged batch in the fp32 mode; the last norm, whose sum has no other reader.
        {"name": "norm-bwd-96x1000-fp32", "kind": "norm_bwd", "rows": 96, "cols": 1000, "resid": False,
         "dtype": "fp32"},
        # An odd number of tokens, a narrow model.
        {"name": "norm-bwd-4097x1600", "kind": "norm_bwd", "rows": 4097, "cols": 1600, "resid": True,
         "dtype": "bf16"},
        # The backward pass of a wide block, 16 sequences of 1024.
        {"name": "norm-bwd-16384x6144", "kind": "norm_bwd", "rows": 16384, "cols": 6144, "resid": True,
         "dtype": "bf16"},
        # One token's loss.
        {"name": "loss-1x50304", "kind": "loss", "tokens": 1, "vocab": 50304, "ld": 50304, "top": 32, "tau": 2.0,
         "alpha": 0.5, "ranks": 1, "ignore": 0.0, "ids": "int64", "teacher": "fp32", "dtype": "bf16"},
        # A validation batch: no gradient.
        {"name": "loss-8192x50304", "kind": "loss", "tokens": 8192, "vocab": 50304, "ld": 50304, "top": 64, "tau": 2.0,
         "alpha": 0.5, "ranks": 1, "ignore": 0.1, "ids": "int32", "teacher": "bf16", "dtype": "bf16"},
        # A ragged batch in the fp32 mode, a vocabulary that its product pads.
        {"name": "step-333x50257-fp32", "kind": "step", "tokens": 333, "vocab": 50257, "ld": 50304, "top": 100,
         "tau": 1.0, "alpha": 0.3, "ranks": 1, "ignore": 0.2, "ids": "int64", "teacher": "fp32", "dtype": "fp32"},
        # The training step's loss and gradient, 8 sequences of 1024.
        {"name": "step-8192x50304", "kind": "step", "tokens": 8192, "vocab": 50304, "ld": 50304, "top": 64, "tau": 2.0,
         "alpha": 0.5, "ranks": 1, "ignore": 0.1, "ids": "int32", "teacher": "bf16", "dtype": "bf16"},
        # Two tensor-parallel ranks' shares of the vocabulary, one after the other.
        {"name": "shards-2047x2x25152", "kind": "shards", "tokens": 2047, "vocab": 50304, "ld": 25152, "top": 64,
         "tau": 2.0, "alpha": 0.5, "ranks": 2, "ignore": 0.1, "ids": "int32", "teacher": "bf16", "dtype": "bf16"},
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of step in [lo, hi], spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(-(-lo // step) * step, min(hi // step * step, step * round(v / step)))


_KINDS = ("norm_fwd", "norm_keep8", "norm_bwd", "loss", "step", "shards")


def draw(rng):
    kind = rng.choice(_KINDS)
    most = max((work(c) for c in listed() if c["kind"] == kind), key=lambda w: w["bytes"])
    while True:
        case = _draw(rng, kind)
        w = work(case)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return case


def _draw(rng, kind):
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if kind.startswith("norm"):
        return {"kind": kind, "rows": _log(rng, 1, 32768), "cols": _log(rng, 64, 8192, 32 if kind == "norm_keep8" else 8),
                "resid": rng.random() < 0.75, "dtype": dtype}
    ranks = rng.choice([2, 4, 8]) if kind == "shards" else 1
    vocab = _log(rng, 1000, 60000)
    per = -(-vocab // ranks)  # columns of a rank; the last one may have fewer
    alpha = rng.choice([0.0, 0.3, 0.5, 0.9, 1.0])
    return {"kind": kind, "tokens": _log(rng, 1, 8192), "vocab": vocab, "ld": -(-per // 64) * 64,
            "top": _log(rng, 1, 256) if alpha > 0 else 0, "tau": rng.choice([1.0, 2.0, 4.0]), "alpha": alpha,
            "ranks": ranks, "ignore": rng.choice([0.0, 0.1, 0.5]), "ids": rng.choice(["int32", "int64"]),
            "teacher": rng.choice(["bf16", "fp32"]), "dtype": dtype}


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    k = case["kind"]
    e = 2 if case["dtype"] == "bf16" else 4
    if k.startswith("norm"):
        n, cols, r = case["rows"] * case["cols"], case["cols"], int(case["resid"])
        if k == "norm_bwd":   # dy, the sum and its gradient; dx and the gain's gradient
            return {"bytes": n * e * (3 + r) + cols * (e + 4), "flops": n * 12}
        b = n * e * (2 + 2 * r) + cols * e
        if k == "norm_keep8":  # the codes and scales are written, read again, and restored
            b += 2 * (n + n // BLOCK) + 2 * n
        return {"bytes": b, "flops": n * 8}
    T, top = case["tokens"], case["top"]
    n = T * case["vocab"]
    t = T * top * ((8 if case["ids"] == "int64" else 4) + (2 if case["teacher"] == "bf16" else 4))
    t += T * ((8 if case["ids"] == "int64" else 4) + 4)
    both = 2 if case["tau"] != 1.0 and 0.0 < case["alpha"] < 1.0 else 1
    if k == "loss":
        return {"bytes": n * e + t, "flops": n * (1 + 3 * both)}
    # the gradient is written over the padding too
    return {"bytes": n * e + T * case["ranks"] * case["ld"] * e + t + 4 * T, "flops": n * (1 + 7 * both)}


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

    def uniform(self, *shape):
        return torch.rand(*shape, generator=self.g, device=DEV, dtype=torch.float32)


def _dtype(case, key="dtype"):
    return torch.bfloat16 if case[key] == "bf16" else torch.float32


def _width(case, rank):
    """Columns of the vocabulary that a rank has."""
    per = -(-case["vocab"] // case["ranks"])
    return max(0, min(per, case["vocab"] - rank * per))


def _norm_inputs(case, d, s):
    dt, rows, cols = _dtype(case), case["rows"], case["cols"]
    # hidden states: most features of order 1, a few channels many times larger
    gain = torch.where(d.uniform(cols) < 0.01, 20.0, 1.0)
    s["gamma"] = d.normal(cols, std=0.1, mean=1.0, dtype=dt)
    if case["kind"] == "norm_bwd":
        s["h"] = (d.normal(rows, cols) * gain).to(dt)
        s["dy"] = d.normal(rows, cols, dtype=dt)
        s["dsum"] = d.normal(rows, cols, dtype=dt) if case["resid"] else None
    else:
        s["x"] = d.normal(rows, cols, dtype=dt)
        s["resid"] = (d.normal(rows, cols) * gain).to(dt) if case["resid"] else None


def _loss_inputs(case, d, s):
    T, V, K = case["tokens"], case["vocab"], case["top"]
    idt = torch.int32 if case["ids"] == "int32" else torch.int64
    z = d.normal(T, V, std=2.0)
    # the right token of each row, which the student has half learnt
    right = (d.uniform(T) * V).long().clamp_(max=V - 1)
    z.scatter_add_(1, right[:, None], torch.full((T, 1), 6.0, device=DEV))
    s["teacher_ids"] = s["teacher_logits"] = None
    if K:
        # K different tokens, one of each K-th of the vocabulary, the likeliest first
        at = ((torch.arange(K, device=DEV) + d.uniform(T, K)).double() * (V / K)).long().clamp_(max=V - 1)
        at = at.gather(1, torch.argsort(d.uniform(T, K), dim=1))
        t = 12.0 - 2.0 * torch.log(torch.arange(K, device=DEV) + 1.0) + d.normal(T, K, std=0.1)
        t = torch.sort(t, dim=1, descending=True)[0]
        z.scatter_add_(1, at, 0.4 * t)
        # a fifth of the rows were kept with fewer entries
        kept = torch.where(d.uniform(T) < 0.2, (1 + d.uniform(T) * (K - 1)).long(), torch.full((T,), K, device=DEV))
        at = torch.where(torch.arange(K, device=DEV) < kept[:, None], at, torch.full_like(at, -1))
        s["teacher_ids"], s["teacher_logits"] = at.to(idt).contiguous(), t.to(_dtype(case, "teacher"))
    ignored = d.uniform(T) < case["ignore"]  # prompts and padding
    s["labels"] = None
    if case["alpha"] < 1.0:
        s["labels"] = torch.where(ignored, torch.full_like(right, -100), right).to(idt)
    s["dloss"] = torch.where(ignored, torch.zeros(T, device=DEV), torch.full((T,), 1.0, device=DEV))
    dt, per = _dtype(case), -(-V // case["ranks"])
    s["logits"] = []
    for r in range(case["ranks"]):
        w = _width(case, r)
        part = torch.zeros(T, case["ld"], device=DEV, dtype=dt)
        part[:, :w] = z[:, r * per:r * per + w].to(dt)
        s["logits"].append(part)


def prepare(case, seed):
    d = _Draws(seed)
    s = {"case": case, "kind": case["kind"]}
    if case["kind"].startswith("norm"):
        _norm_inputs(case, d, s)
    else:
        _loss_inputs(case, d, s)
    if own:
        _buffers(s)
    return s


def _buffers(s):
    """The outputs and workspaces that a program keeps from step to step."""
    from paper_2206_04959_amd import binding as B
    case, k, dt = s["case"], s["kind"], _dtype(s["case"])
    new = lambda *shape, dtype=dt: torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
    b = {}
    if k.startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        if k == "norm_bwd":
            b["dx"], b["dgamma"] = new(rows, cols), new(cols, dtype=torch.float32)
            b["scratch"] = new(B.add_rms_norm_scratch_elems(rows, cols), dtype=torch.float32)
        else:
            b["y"], b["sum"] = new(rows, cols), new(rows, cols) if case["resid"] else None
        if k == "norm_keep8":
            b["q"] = new(rows, cols, dtype=torch.uint8)
            b["scales"] = new(rows, cols // BLOCK, dtype=torch.uint8)
            b["kept"] = new(rows, cols, dtype=torch.bfloat16)
    else:
        T, ranks = case["tokens"], case["ranks"]
        b["loss"] = new(T, dtype=torch.float32)
        if k != "loss":
            b["dlogits"] = [torch.empty_like(z) for z in s["logits"]]
        if k == "shards":
            b["parts"] = new(ranks, T, B.DISTILL_STATS, dtype=torch.float32)
            b["stats"] = new(T, B.DISTILL_STATS, dtype=torch.float32)
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
    if k == "norm_bwd":
        B.add_rms_norm_bwd(s["dy"], s["h"], s["gamma"], b["dx"], b["dgamma"], b["scratch"], dsum=s["dsum"], eps=EPS)
        return {"dx": b["dx"], "dgamma": b["dgamma"]}
    if k == "norm_fwd":
        B.add_rms_norm_fwd(s["x"], s["gamma"], b["y"], resid=s["resid"], sum=b["sum"], eps=EPS)
        return _given(sum=b["sum"], y=b["y"])
    if k == "norm_keep8":
        B.add_rms_norm_fwd(s["x"], s["gamma"], b["y"], resid=s["resid"], sum=b["sum"], q=b["q"], scales=b["scales"],
                           eps=EPS)
        B.act8_restore(b["q"], b["scales"], b["kept"])
        return _given(sum=b["sum"], y=b["y"], kept=b["kept"])
    learn = dict(teacher_ids=s["teacher_ids"], teacher_logits=s["teacher_logits"], labels=s["labels"],
                 alpha=case["alpha"], temperature=case["tau"])
    if k == "loss":
        B.distill_loss_fwd(s["logits"][0], loss=b["loss"], vocab=case["vocab"], **learn)
        return b["loss"]
    if k == "step":
        B.distill_loss_fwd_bwd(s["logits"][0], s["dloss"], b["loss"], b["dlogits"][0], vocab=case["vocab"], **learn)
        return {"loss": b["loss"], "dlogits": b["dlogits"][0]}
    shares = [dict(vocab=_width(case, r), first_id=r * -(-case["vocab"] // case["ranks"]), vocab_total=case["vocab"])
              for r in range(case["ranks"])]
    for z, part, share in zip(s["logits"], b["parts"], shares):
        B.distill_loss_fwd(z, stats=part, **share, **learn)
    B.distill_loss_join(b["parts"], b["stats"], b["loss"], alpha=case["alpha"], temperature=case["tau"])
    for z, dz, share in zip(s["logits"], b["dlogits"], shares):
        B.distill_loss_bwd(z, b["stats"], s["dloss"], dz, **share, **learn)
    return {"loss": b["loss"], "dlogits": b["dlogits"]}


def _given(**outputs):
    return {k: v for k, v in outputs.items() if v is not None}


# ---------------------------------------------------------------------------
# The plain form: elementary torch operations in 32 bits
# ---------------------------------------------------------------------------

def _plain_sum(s):
    """The sum as it is stored, which is what is normed."""
    if s["resid"] is None:
        return s["x"], None
    h = (s["x"].float() + s["resid"].float()).to(s["x"].dtype)
    return h, h


def _plain_norm(h, gamma):
    v = h.float()
    return v * torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS) * gamma.float()


def _plain_norm_fwd(s):
    h, kept = _plain_sum(s)
    return _given(sum=kept, y=_plain_norm(h, s["gamma"]).to(h.dtype))


def _pow2(e):
    """2^e in 32 bits, from the exponent's bits; -126 <= e <= 127."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _eight_bits(y):
    """What the codes and scales of y [rows, cols] stand for: the scale is the smallest power of
    two that brings the block's largest magnitude to 448 or less."""
    b = y.reshape(y.shape[0], -1, BLOCK)
    m, e = torch.frexp(b.abs().amax(-1))   # |y| = m 2^e, 1/2 <= m < 1
    exp = torch.where(m > 0, e - 9 + (m > 0.875).int(), torch.full_like(e, MIN_EXP)).clamp(MIN_EXP, MAX_EXP)
    v = b * _pow2(-exp)[..., None]
    # round to nearest, ties to even: steps of 2^-3 of the value's power of two, at least 2^-9
    step = _pow2(torch.clamp(torch.frexp(v)[1] - 1, -6, 8) - 3)
    return (torch.round(v / step) * step * _pow2(exp)[..., None]).reshape(y.shape).to(torch.bfloat16)


def _plain_norm_keep8(s):
    h, kept = _plain_sum(s)
    y = _plain_norm(h, s["gamma"])
    return _given(sum=kept, y=y.to(h.dtype), kept=_eight_bits(y))


def _plain_norm_bwd(s):
    h, dy, dt = s["h"].float(), s["dy"].float(), s["h"].dtype
    rstd = torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS)
    n = h * rstd
    dgamma = (dy * n).sum(0)
    dn = dy * s["gamma"].float()
    dx = rstd * (dn - n * (dn * n).mean(-1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    return {"dx": dx.to(dt), "dgamma": dgamma}


def _whole(s):
    """The logits of all ranks' columns, in 32 bits."""
    case = s["case"]
    parts = [z[:, :_width(case, r)] for r, z in enumerate(s["logits"])]
    return (parts[0] if len(parts) == 1 else torch.cat(parts, 1)).float()


def _softmax(z):
    """Logarithms of the softmax of each row, and the softmax."""
    d = z - z.amax(1, keepdim=True)
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    return d - torch.log(total), e / total


def _plain_teacher(s, tau):
    """(columns, probabilities and their logarithms) of the teacher's entries; entries that are
    not there have the probability 0."""
    ids, t = s["teacher_ids"].long(), s["teacher_logits"].float() / tau
    there = ids >= 0
    e = torch.where(there, torch.exp(t - t.amax(1, keepdim=True)), torch.zeros_like(t))
    p = e / e.sum(1, keepdim=True)
    return ids.clamp(min=0), p, torch.log(torch.where(there, p, torch.ones_like(p)))


def _plain_loss(s, gradient=False):
    case = s["case"]
    tau, alpha = case["tau"], case["alpha"]
    z = _whole(s)
    loss, dz = torch.zeros(z.shape[0], device=DEV), None
    w = s["dloss"][:, None]
    if s["teacher_ids"] is not None:
        at, p, logp = _plain_teacher(s, tau)
        logq, q = _softmax(z / tau)
        loss = loss + alpha * tau * tau * (p * (logp - logq.gather(1, at))).sum(1)
        if gradient:
            dz = alpha * tau * w * q.scatter_add(1, at, -p)
        del logq, q
    if s["labels"] is not None:
        label = s["labels"].long()
        counts = (label >= 0).float()
        at = label.clamp(min=0)[:, None]
        logq, q = _softmax(z)
        loss = loss - (1.0 - alpha) * counts * logq.gather(1, at)[:, 0]
        if gradient:
            c = (1.0 - alpha) * counts[:, None]
            part = c * w * q.scatter_add(1, at, -torch.ones_like(at, dtype=torch.float32))
            dz = part if dz is None else dz + part
    return (loss, dz) if gradient else loss


def _shares(case, dz, dt):
    """The gradient laid out as the ranks' logits are; zeros behind a rank's columns."""
    per, out = -(-case["vocab"] // case["ranks"]), []
    for r in range(case["ranks"]):
        w = _width(case, r)
        out.append(torch.nn.functional.pad(dz[:, r * per:r * per + w].to(dt), (0, case["ld"] - w)))
    return out


def _plain_step(s):
    loss, dz = _plain_loss(s, gradient=True)
    parts = _shares(s["case"], dz, _dtype(s["case"]))
    return {"loss": loss, "dlogits": parts if s["kind"] == "shards" else parts[0]}


_PLAIN = {"norm_fwd": _plain_norm_fwd, "norm_keep8": _plain_norm_keep8, "norm_bwd": _plain_norm_bwd,
          "loss": _plain_loss, "step": _plain_step, "shards": _plain_step}


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return _exact_norm(case, s) if case["kind"].startswith("norm") else _exact_loss(case, s)


def _exact_norm(case, s):
    g = s["gamma"].double()
    if case["kind"] == "norm_bwd":
        h, dy = s["h"].double(), s["dy"].double()
        length = torch.sqrt((h * h).sum(-1, keepdim=True) / case["cols"] + EPS)
        unit, up = h / length, dy * g
        dx = (up - unit * (up * unit).sum(-1, keepdim=True) / case["cols"]) / length
        if s["dsum"] is not None:
            dx += s["dsum"].double()
        return {"dx": dx, "dgamma": (dy * unit).sum(0)}
    out = {}
    h = s["x"].double()
    if s["resid"] is not None:
        out["sum"] = h + s["resid"].double()
        h = out["sum"].to(_dtype(case)).double()  # the norm is that of the sum as it is stored
    y = h * g / torch.sqrt((h * h).sum(-1, keepdim=True) / case["cols"] + EPS)
    out["y"] = y
    if case["kind"] == "norm_keep8":
        out["kept"] = None  # a y next to the border of two codes goes to either by its last bit: off by a whole code
    return out


def _exact_loss(case, s):
    T, V, tau, alpha = case["tokens"], case["vocab"], case["tau"], case["alpha"]
    z = torch.cat([part[:, :_width(case, r)].double() for r, part in enumerate(s["logits"])], 1)
    want = torch.zeros(T, V, dtype=torch.float64, device=DEV) if case["kind"] != "loss" else None
    loss = torch.zeros(T, dtype=torch.float64, device=DEV)
    row = torch.arange(T, device=DEV)
    if s["teacher_ids"] is not None:
        there = s["teacher_ids"] >= 0
        p = torch.softmax(torch.where(there, s["teacher_logits"].double() / tau, -math.inf), 1)
        lse = torch.logsumexp(z / tau, 1)
        r, k = there.nonzero(as_tuple=True)
        col, pk = s["teacher_ids"][r, k].long(), p[r, k]
        each = pk * (torch.log(pk) - z[r, col] / tau + lse[r])
        loss.index_add_(0, r, alpha * tau ** 2 * each)
        if want is not None:
            want += alpha * tau * torch.exp(z / tau - lse[:, None])
            want.index_put_((r, col), -alpha * tau * pk, accumulate=True)
    if s["labels"] is not None:
        counts = s["labels"] >= 0
        lse = torch.logsumexp(z, 1)
        r, col = row[counts], s["labels"][counts].long()
        loss.index_add_(0, r, (1.0 - alpha) * (lse[r] - z[r, col]))
        if want is not None:
            want[r] += (1.0 - alpha) * torch.exp(z[r] - lse[r, None])
            want.index_put_((r, col), torch.full_like(z[r, col], -(1.0 - alpha)), accumulate=True)
    if want is None:
        return loss
    want *= s["dloss"].double()[:, None]
    per = -(-V // case["ranks"])
    parts = []
    for r in range(case["ranks"]):
        part = torch.zeros(T, case["ld"], dtype=torch.float64, device=DEV)
        part[:, :_width(case, r)] = want[:, r * per:r * per + _width(case, r)]
        parts.append(part)
    return {"loss": loss, "dlogits": parts if case["kind"] == "shards" else parts[0]}
