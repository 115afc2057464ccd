"""Operators around the blocks in fp64: embedding lookup and gradient, query/key norm
with position rotation and gradient, 8-bit activation checkpoints and the
gradients taken from them.  Written out from the definitions; the HIP side shares
nothing with it.
"""
from __future__ import annotations

import numpy as np


# -- embedding ---------------------------------------------------------------

def embedding(ids, table, scale=1.0, first=0):
    """y[t] = scale * table[ids[t] - first], zeros where that is no row."""
    ids = np.asarray(ids).astype(np.int64).ravel()
    y = np.zeros((ids.size, table.shape[1]))
    for t, i in enumerate(ids):
        if first <= i < first + table.shape[0]:
            y[t] = scale * table[i - first]
    return y


def embedding_backward(ids, dy, rows, scale=1.0, first=0):
    """(gradient of the table, sum of the magnitudes that went into it, tokens of each row)."""
    ids = np.asarray(ids).astype(np.int64).ravel()
    g, mag, count = np.zeros((rows, dy.shape[1])), np.zeros((rows, dy.shape[1])), np.zeros(rows, dtype=np.int64)
    for t, i in enumerate(ids):
        if first <= i < first + rows:
            g[i - first] += scale * dy[t]
            mag[i - first] += np.abs(scale * dy[t])
            count[i - first] += 1
    return g, mag, count


# -- query/key norm with rotation --------------------------------------------

def rope_table(positions, rope_dim, theta=10000.0):
    """[positions, rope_dim / 2, 2]: cosine and sine of p * theta^(-2 i / rope_dim)."""
    a = np.arange(positions)[:, None] * theta ** (-2.0 * np.arange(rope_dim // 2) / rope_dim)
    return np.stack([np.cos(a), np.sin(a)], -1)


def _pairs(rope_dim, interleaved):
    i = np.arange(rope_dim // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rope_dim // 2)


def _turn(z, cs, rope_dim, interleaved, sign):
    """Rotate the pairs of z [tokens, heads, d] by cs [tokens, rope_dim / 2, 2]."""
    out = z.copy()
    if rope_dim:
        ia, ib = _pairs(rope_dim, interleaved)
        c, s = cs[:, None, :, 0], sign * cs[:, None, :, 1]
        out[..., ia] = z[..., ia] * c - z[..., ib] * s
        out[..., ib] = z[..., ib] * c + z[..., ia] * s
    return out


def qk_norm_rope(qkv, gq, gk, cs, q_heads, kv_heads, rope_dim, interleaved=False, eps=1e-6):
    """qkv [tokens, q_heads + 2 kv_heads, d]; cs [tokens, rope_dim / 2, 2]: each token's row of
    the table."""
    out = qkv.copy()
    for lo, hi, g in ((0, q_heads, gq), (q_heads, q_heads + kv_heads, gk)):
        x = qkv[:, lo:hi]
        n = x / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps)
        out[:, lo:hi] = _turn(n * g, cs, rope_dim, interleaved, 1.0)
    return out


def qk_norm_rope_backward(dout, qkv, gq, gk, cs, q_heads, kv_heads, rope_dim, interleaved=False, eps=1e-6):
    """(dqkv, dgq, dgk)."""
    dx = dout.copy()
    gains = []
    for lo, hi, g in ((0, q_heads, gq), (q_heads, q_heads + kv_heads, gk)):
        x = qkv[:, lo:hi]
        r = 1.0 / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps)
        n = x * r
        dz = _turn(dout[:, lo:hi], cs, rope_dim, interleaved, -1.0)
        gains.append((dz * n).sum((0, 1)))
        dn = dz * g
        dx[:, lo:hi] = r * (dn - n * np.mean(dn * n, -1, keepdims=True))
    return dx, gains[0], gains[1]


# -- activation checkpoints in 8 bits ----------------------------------------

BLOCK, LARGEST, MIN_EXP = 32, 448.0, -117
CLIP = 240.0 * 2.0 ** 120  # the next value would be 2^128


def e4m3_values():
    """The value of each of the 256 e4m3 codes."""
    v = np.zeros(256)
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        m = (1 + f / 8.0) * 2.0 ** (e - 7) if e else f / 8.0 * 2.0 ** -6
        v[c] = (-1 if c & 128 else 1) * (np.nan if e == 15 and f == 7 else m)
    return v


def act8_save(x):
    """(codes, scale bytes) of x [rows, cols]: each value's nearest code, the even one of two
    as near."""
    rows, cols = x.shape
    b = x.reshape(rows, cols // BLOCK, BLOCK)
    finite = np.isfinite(b)
    most = np.abs(np.where(finite, b, 0.0)).max(-1)
    exp = np.full(most.shape, MIN_EXP)
    for idx in np.ndindex(most.shape):  # the smallest power of two that is enough
        while most[idx] > LARGEST * 2.0 ** exp[idx]:
            exp[idx] += 1
    grid = e4m3_values()[:127]  # non-negative finite codes, ascending
    v = np.minimum(np.abs(np.where(finite, b, 0.0)), CLIP) / 2.0 ** exp[..., None].astype(np.float64)
    hi = np.clip(np.searchsorted(grid, v), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - v, v - grid[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    code = np.where(finite, code, 127) | np.where(np.signbit(b) & finite, 128, 0)
    return code.reshape(rows, cols).astype(np.uint8), (exp + 127).astype(np.uint8)


def act8_restore(q, scales):
    v = e4m3_values()[q].reshape(q.shape[0], -1, BLOCK)
    return (v * 2.0 ** (scales.astype(np.float64)[..., None] - 127.0)).reshape(q.shape)


def gelu_parts(u):
    """(GeLU(u), GeLU'(u)), tanh form, through the logistic function of both signs so that
    neither tail cancels."""
    c, a = np.sqrt(2.0 / np.pi), 0.044715
    z2 = 2.0 * c * (u + a * u ** 3)
    e = np.exp(-np.abs(z2))
    near, far = 1.0 / (1.0 + e), e / (1.0 + e)
    s, t = np.where(z2 >= 0, near, far), np.where(z2 >= 0, far, near)
    return u * s, s + u * s * t * 2.0 * c * (1.0 + 3.0 * a * u * u)


# -- residual addition and root-mean-square norm --------------------------------

def rms_norm(h, gamma, eps=1e-6):
    """gamma * h / sqrt(mean(h^2) + eps) of each row."""
    return gamma * h / np.sqrt((h * h).mean(-1, keepdims=True) + eps)


def rms_norm_backward(dy, h, gamma, dsum=None, eps=1e-6):
    """(gradient of h, of gamma, magnitudes that went into each): dsum is the gradient that
    reaches h from elsewhere."""
    rstd = 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    n, dn = h * rstd, dy * gamma
    ds = np.zeros_like(h) if dsum is None else dsum
    dx = ds + rstd * (dn - n * (dn * n).mean(-1, keepdims=True))
    mag = np.abs(ds) + rstd * (np.abs(dn) + np.abs(n) * np.abs(dn * n).mean(-1, keepdims=True))
    return dx, (dy * n).sum(0), mag, np.abs(dy * n).sum(0)


# -- distillation from a teacher's top logits ---------------------------------

def distill(z, ids=None, t=None, labels=None, alpha=0.5, tau=1.0, total=None):
    """Loss of each token and its gradient by the logits z [tokens, vocab]; ids and t [tokens, top] are
    the teacher's entries (ids outside the vocabulary are none), labels [tokens].  Third comes a
    dict of what the tolerances need: the magnitudes that went into the loss, and the gradient's
    positive and negative parts."""
    z = np.asarray(z, dtype=np.float64)
    tokens, vocab = z.shape
    total = vocab if total is None else total
    loss, grad, size = np.zeros(tokens), np.zeros_like(z), np.zeros(tokens)
    plus, minus = np.zeros_like(z), np.zeros_like(z)

    def log_softmax(v):
        m = v.max()
        with np.errstate(invalid="ignore"):
            d = v - m
        return d - np.log(np.exp(d).sum()), d

    for i in range(tokens):
        if ids is not None and alpha > 0:
            keep = [(int(c), float(x)) for c, x in zip(ids[i], t[i]) if 0 <= c < total and x != -np.inf]
            if keep:
                x = np.array([x for _, x in keep]) / tau
                lp, _ = log_softmax(x)
                lq, d = log_softmax(z[i] / tau)
                p, q = np.exp(lp), np.exp(lq)
                cols = [c for c, _ in keep]
                use = p > 0
                loss[i] += alpha * tau ** 2 * (p[use] * (lp[use] - lq[cols][use])).sum()
                size[i] += alpha * tau ** 2 * (p[use] * (np.abs(lp[use]) + np.abs(d[cols][use]) + 1)).sum()
                plus[i] += alpha * tau * q
                np.add.at(minus[i], cols, alpha * tau * p)
        if labels is not None and alpha < 1 and 0 <= labels[i] < total:
            lq, d = log_softmax(z[i])
            loss[i] -= (1 - alpha) * lq[labels[i]]
            size[i] += (1 - alpha) * (np.abs(d[labels[i]]) + 1)
            plus[i] += (1 - alpha) * np.exp(lq)
            minus[i, labels[i]] += 1 - alpha
    grad = plus - minus
    return loss, grad, {"loss": size, "plus": plus, "minus": minus}
