"""The operators around the blocks on the GPU, through the C ABI, against the fp64 oracle.

Tolerances count roundings.  u = 2^-24 is half a step of fp32, `half` half a step of
the output's type (2^-8 in bf16, u in fp32), relative to the value.  A sum of n fp32
terms in any order is off by at most n u times the sum of the magnitudes (to first
order).  Each test says which roundings its bound holds; a few more are granted for
products and functions that are within a step or two."""
import numpy as np
import pytest

from oracle import operators as O
from paper_2206_04959_amd import binding as B
from paper_2206_04959_amd import synth
from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "fp32": U}
TINY = 1e-37  # results below the normal numbers


def _type(torch, dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _normal(rng, shape, dtype, std=1.0, mean=0.0):
    """(device tensor, the same values in fp64)"""
    v = rng.standard_normal(size=shape, dtype=np.float32) * np.float32(std) + np.float32(mean)
    return _given(v, dtype)


def _given(v, dtype):
    v = np.asarray(v, dtype=np.float32)
    if dtype == "bf16":
        bits = synth.f32_to_bf16_bits(v)
        return B.to_device(bits), synth.bf16_bits_to_f64(bits)
    return B.to_device(v), v.astype(np.float64)


def _guarded(torch, shape, dtype, extra=64, fill=7.0):
    """(tensor of `shape`, check that nothing behind it was written)"""
    n = int(np.prod(shape))
    whole = torch.full((n + extra,), fill, dtype=dtype, device="cuda")
    return whole[:n].view(shape), lambda: bool((whole[n:] == fill).all())


def _f64(t):
    return t.detach().double().cpu().numpy()


def _within(got, ref, tol):
    got = _f64(got)
    worst = np.max((np.abs(got - ref) - tol))
    assert got.shape == ref.shape and np.isfinite(got).all() and worst <= 0, \
        (worst, np.max(np.abs(got - ref)), np.unravel_index(np.argmax(np.abs(got - ref) - tol), got.shape))


# ---------------------------------------------------------------------------
# Embedding
# ---------------------------------------------------------------------------

def _ids(rng, tokens, rows, first, pattern):
    if pattern == "mixed":     # own rows, other ranks' on both sides, padding
        ids = rng.integers(max(0, first - rows), first + 2 * rows, tokens)
        ids[rng.random(tokens) < 0.1] = -1
    elif pattern == "same":
        ids = np.full(tokens, first + rows // 2)
    elif pattern == "none":
        ids = np.full(tokens, first + rows)
    elif pattern == "falling":  # every row once, last row first
        ids = first + rows - 1 - np.arange(tokens) % rows
    else:                      # a few rows most of the time
        ids = first + np.minimum((rows * rng.random(tokens) ** 6).astype(np.int64), rows - 1)
    return ids.astype(np.int64)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tokens,hidden,rows,first,ids_type", [
    (1, 8, 1, 0, "int32"), (1, 1600, 100, 0, "int64"), (63, 72, 11, 40, "int64"), (257, 1000, 300, 600, "int32"),
    (3001, 64, 50, 0, "int64"), (5, 6144, 9, 3, "int32")])
def test_embedding_forward(dtype, tokens, hidden, rows, first, ids_type):
    torch = need_gpu()
    print(f"[embedding fwd] {dtype} {tokens}x{hidden} rows {rows} from {first}", flush=True)
    rng = np.random.default_rng(tokens)
    ids = _ids(rng, tokens, rows, first, "mixed")
    if tokens == 1:
        ids[:] = first
    if ids_type == "int64" and tokens > 3:
        ids[:3] = [2 ** 62, -2 ** 63, 2 ** 63 - 1]
    table, tv = _normal(rng, (rows, hidden), dtype)
    y, clean = _guarded(torch, (tokens, hidden), table.dtype)
    B.embedding_fwd(torch.from_numpy(ids).to(getattr(torch, ids_type)).cuda(), table, y, scale=1.7, first_id=first)
    torch.cuda.synchronize()
    ref = O.embedding(ids, tv, float(np.float32(1.7)), first)
    _within(y, ref, (HALF[dtype] + U) * np.abs(ref))  # one product, one rounding of the result
    assert clean()


EMBED_BWD = [(1, 8, 1, 0), (2, 1600, 5, 0), (63, 72, 40, 7), (64, 520, 33, 100), (65, 64, 40, 7), (200, 1000, 17, 0),
             (255, 24, 90, 5), (256, 520, 7, 0), (257, 8, 200, 0), (2047, 40, 300, 0), (2048, 16, 60, 9), (2049, 16, 3000, 0), (5003, 24, 100, 50), (17000, 8, 90, 0), (33000, 8, 9, 3)]


@pytest.mark.parametrize("pattern", ["mixed", "same", "none", "falling", "few"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tokens,hidden,rows,first", EMBED_BWD)
def test_embedding_backward(dtype, tokens, hidden, rows, first, pattern):
    torch = need_gpu()
    print(f"[embedding bwd] {dtype} {tokens}x{hidden} rows {rows} from {first} {pattern}", flush=True)
    rng = np.random.default_rng(tokens + hidden)
    ids = _ids(rng, tokens, rows, first, pattern)
    dy, dv = _normal(rng, (tokens, hidden), dtype)
    kind = torch.int32 if tokens % 2 else torch.int64
    dev_ids = torch.from_numpy(ids).to(kind).cuda()
    ref, mag, count = O.embedding_backward(ids, dv, rows, 0.5, first)
    # the sum, its scaling and (accumulating) its addition
    tol = (count[:, None] + 3) * U * mag
    n = B.embedding_scratch_bytes(tokens, hidden)
    scratch, kept = _guarded(torch, (n,), torch.uint8) if n else (None, lambda: True)
    dt, clean = _guarded(torch, (rows, hidden), torch.float32)
    runs = []
    for _ in range(2):
        dt.fill_(float("nan"))
        B.embedding_bwd(dev_ids, dy, dt, scratch, scale=0.5, first_id=first)
        torch.cuda.synchronize()
        runs.append(dt.clone())
    _within(dt, ref, tol)
    assert torch.equal(runs[0], runs[1]) and clean() and kept()
    assert not _f64(dt)[count == 0].any()
    base, bv = _normal(rng, (rows, hidden), "fp32")
    dt.copy_(base)
    B.embedding_bwd(dev_ids, dy, dt, scratch, scale=0.5, first_id=first, accumulate=True)
    torch.cuda.synchronize()
    _within(dt, bv + ref, tol + U * np.abs(bv + ref))
    assert np.array_equal(_f64(dt)[count == 0], bv[count == 0])


# ---------------------------------------------------------------------------
# Query/key norm with rotation
# ---------------------------------------------------------------------------

QK = [  # tokens, q heads, kv heads, head_dim, rope_dim, interleaved, positions given
    (1, 25, 25, 64, 64, False, False), (1, 1, 1, 8, 0, False, False), (3, 4, 2, 96, 96, False, True),
    (129, 8, 8, 96, 48, False, False), (130, 6, 6, 128, 128, True, True), (67, 24, 6, 128, 64, False, True),
    (64, 5, 5, 80, 80, False, False), (33, 3, 1, 256, 256, True, False), (50, 2, 2, 136, 128, False, True),
    (257, 1, 3, 72, 64, True, True), (700, 7, 7, 64, 32, False, False), (9, 4, 4, 16, 16, False, True),
    (40, 4, 2, 192, 192, False, True), (31, 3, 3, 96, 96, True, False), (20, 2, 2, 24, 16, False, False)]


def _qk_case(torch, rng, dtype, tokens, q, kv, d, rope, positions, far=3000):
    qkv, xv = _normal(rng, (tokens, q + 2 * kv, d), dtype, std=2.0)
    gq, gqv = _normal(rng, (d,), dtype, std=0.1, mean=1.0)
    gk, gkv = _normal(rng, (d,), dtype, std=0.1, mean=1.0)
    table, kw, cs = None, {}, None
    if rope:
        table = torch.empty((far, rope // 2, 2), dtype=torch.float32, device="cuda")
        B.rope_table(table)
        torch.cuda.synchronize()
        pos = rng.integers(0, far, tokens) if positions else np.arange(tokens) % 50
        kw = (dict(positions=torch.from_numpy(pos.astype(np.int32)).cuda()) if positions else dict(seq_len=50))
        cs = _f64(table)[pos]
    return (qkv, gq, gk, table), (xv, gqv, gkv, cs), dict(q_heads=q, kv_heads=kv, **kw)


def _turned(mag, cs, rope, inter):
    """Magnitudes that the rotation adds up: |a cos| + |b sin| and |b cos| + |a sin|."""
    if not rope:
        return mag
    out = O._turn(mag, np.stack([np.abs(cs[..., 0]), -np.abs(cs[..., 1])], -1), rope, inter, 1.0)
    ib = O._pairs(rope, inter)[1]
    other = O._turn(mag, np.abs(cs), rope, inter, 1.0)
    out[..., ib] = other[..., ib]
    return out


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tokens,q,kv,d,rope,inter,positions", QK)
def test_qk_norm_rope(dtype, tokens, q, kv, d, rope, inter, positions):
    torch = need_gpu()
    print(f"[qk] {dtype} {tokens} tokens {q}+{kv} heads of {d}, rope {rope} inter {inter}", flush=True)
    rng = np.random.default_rng(d + tokens)
    (qkv, gq, gk, table), (xv, gqv, gkv, cs), kw = _qk_case(torch, rng, dtype, tokens, q, kv, d, rope, positions)
    out, clean = _guarded(torch, qkv.shape, qkv.dtype)
    B.qk_norm_rope_fwd(qkv, gq, gk, table, out, interleaved=inter, **kw)
    torch.cuda.synchronize()
    ref = O.qk_norm_rope(xv, gqv, gkv, cs, q, kv, rope, inter)
    # a mean of d squares under a root, its inverse, two products, a rotation; one
    # rounding of the result
    z = O.qk_norm_rope(xv, gqv, gkv, None, q, kv, 0)
    mag = np.abs(z)
    mag[:, :q + kv] = _turned(mag[:, :q + kv], cs, rope, inter)
    _within(out, ref, HALF[dtype] * np.abs(ref) + (d + 16) * U * mag + TINY)
    assert np.array_equal(_f64(out)[:, q + kv:], xv[:, q + kv:]) and clean()
    same = qkv.clone()
    B.qk_norm_rope_fwd(same, gq, gk, table, same, interleaved=inter, **kw)
    assert torch.equal(same, out)

    dout, dv = _normal(rng, qkv.shape, dtype)
    dqkv, clean = _guarded(torch, qkv.shape, qkv.dtype)
    scratch, kept = _guarded(torch, (B.qk_norm_rope_scratch_elems(tokens, q, kv, d),), torch.float32)
    dgq, dgk = (torch.full((d,), float("nan"), dtype=torch.float32, device="cuda") for _ in range(2))
    B.qk_norm_rope_bwd(dout, qkv, gq, gk, table, dqkv, dgq, dgk, scratch, interleaved=inter, **kw)
    torch.cuda.synchronize()
    assert clean() and kept()
    dx, rq, rk = O.qk_norm_rope_backward(dv, xv, gqv, gkv, cs, q, kv, rope, inter)
    tol = HALF[dtype] * np.abs(dx) + TINY
    for lo, hi, g, got, want in ((0, q, gqv, dgq, rq), (q, q + kv, gkv, dgk, rk)):
        x = xv[:, lo:hi]
        r = 1.0 / np.sqrt(np.mean(x * x, -1, keepdims=True) + 1e-6)
        n = np.abs(x) * r
        dz = _turned(np.abs(dv[:, lo:hi]), cs, rope, inter)  # (a bound either way round)
        part = np.abs(g) * dz
        tol[:, lo:hi] += (2 * d + 32) * U * r * (part + n * np.mean(part * n, -1, keepdims=True))
        _within(got, want, (tokens * (hi - lo) + d + 16) * U * (dz * n).sum((0, 1)))
    _within(dqkv, dx, tol)
    assert np.array_equal(_f64(dqkv)[:, q + kv:], dv[:, q + kv:])
    # in place, added to what is there, and the same bits again
    first = (dgq.clone(), dgk.clone())
    inp = dout.clone()
    B.qk_norm_rope_bwd(inp, qkv, gq, gk, table, inp, dgq, dgk, scratch, interleaved=inter, accumulate=True, **kw)
    torch.cuda.synchronize()
    assert torch.equal(inp, dqkv)
    assert all(torch.equal(g, f + f) or torch.allclose(g, 2 * f, rtol=1e-5, atol=1e-5) for g, f in zip((dgq, dgk), first))


def test_rope_table_far_positions():
    torch = need_gpu()
    table = torch.empty((200000, 48, 2), dtype=torch.float32, device="cuda")
    B.rope_table(table, theta=50000.0)
    torch.cuda.synchronize()
    ref = O.rope_table(200000, 96, 50000.0)
    assert np.abs(_f64(table) - ref).max() <= U + 1e-10  # one rounding of a value up to 1


@pytest.mark.parametrize("inter", [False, True])
def test_qk_positions_outside_the_table_give_nan(inter):
    torch = need_gpu()
    rng = np.random.default_rng(5)
    (qkv, gq, gk, table), _, kw = _qk_case(torch, rng, "bf16", 6, 2, 2, 64, 32, True, far=100)
    kw["positions"][1], kw["positions"][4] = -1, 100
    out = torch.empty_like(qkv)
    B.qk_norm_rope_fwd(qkv, gq, gk, table, out, interleaved=inter, **kw)
    torch.cuda.synchronize()
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[1, :4, :32] = bad[4, :4, :32] = True
    assert torch.equal(torch.isnan(out), bad)


def test_qk_non_finite_values_stay_in_their_head():
    torch = need_gpu()
    rng = np.random.default_rng(6)
    (qkv, gq, gk, table), _, kw = _qk_case(torch, rng, "fp32", 20, 3, 3, 96, 96, False)
    clean = torch.empty_like(qkv)
    B.qk_norm_rope_fwd(qkv, gq, gk, table, clean, **kw)
    qkv[7, 4, 5], qkv[11, 0, 90] = float("nan"), float("inf")
    out = torch.empty_like(qkv)
    B.qk_norm_rope_fwd(qkv, gq, gk, table, out, **kw)
    torch.cuda.synchronize()
    keep = torch.ones((20, 9), dtype=torch.bool)
    keep[7, 4] = keep[11, 0] = False
    assert torch.equal(out[keep], clean[keep]) and torch.isnan(out[7, 4]).all()


# ---------------------------------------------------------------------------
# Activation checkpoints in 8 bits
# ---------------------------------------------------------------------------

def _wild(rng, rows, cols):
    """Rows of every size, with zeros, ties of the rounding, extremes and non-finite values."""
    x = rng.standard_normal((rows, cols)).astype(np.float32)
    x *= (10.0 ** rng.integers(-6, 7, size=(rows, 1))).astype(np.float32)
    x[rng.random((rows, cols)) < 0.05] = 0.0
    for r in range(0, rows, 5):
        x[r] = (rng.integers(-255, 256, cols) * 2.0 ** rng.integers(-12, 3)).astype(np.float32)
    if rows > 8:
        x[1] = 0.0
        x[2, :32], x[3, :32] = 448.0, 449.0
        x[4, 3], x[4, 7], x[6, -1] = np.inf, np.nan, -np.inf
        x[7] *= np.float32(1e-36) / np.abs(x[7]).max().clip(1e-30)
        x[8, 0] = np.finfo(np.float32).max
    return x


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols", [(1, 32), (1, 1600), (7, 96), (333, 320), (64, 6400)])
def test_act8_save_and_restore(dtype, rows, cols):
    torch = need_gpu()
    print(f"[act8] {dtype} {rows}x{cols}", flush=True)
    x, xv = _given(_wild(np.random.default_rng(rows), rows, cols), dtype)
    q, clean_q = _guarded(torch, (rows, cols), torch.uint8)
    s, clean_s = _guarded(torch, (rows, cols // 32), torch.uint8)
    y, clean_y = _guarded(torch, (rows, cols), x.dtype)
    B.act8_save(x, q, s)
    B.act8_restore(q, s, y)
    torch.cuda.synchronize()
    want_q, want_s = O.act8_save(xv)
    got_q = q.cpu().numpy()
    nan = ~np.isfinite(xv)
    assert np.array_equal(s.cpu().numpy(), want_s)
    zero = (want_q & 127) == 0  # (a value that rounds to zero may keep either sign)
    assert np.array_equal(got_q[~nan & ~zero], want_q[~nan & ~zero]) and not (got_q[zero] & 127).any()
    assert (got_q[nan] & 127 == 127).all()
    assert np.array_equal(_f64(y), O.act8_restore(want_q, want_s), equal_nan=True)
    assert clean_q() and clean_s() and clean_y()


def test_act8_every_code_restores_to_its_value():
    torch = need_gpu()
    q = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(247 - 10 + 1, 1)
    s = torch.arange(10, 248, dtype=torch.uint8, device="cuda")[:, None].repeat(1, 8)
    want = O.act8_restore(q.cpu().numpy(), s.cpu().numpy())
    fits = np.abs(np.nan_to_num(want)) < 2.0 ** 128
    for dt in (torch.bfloat16, torch.float32):
        y = torch.empty(q.shape, dtype=dt, device="cuda")
        B.act8_restore(q, s, y)
        torch.cuda.synchronize()
        assert np.array_equal(_f64(y)[fits], want[fits], equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols", [(1, 32), (5, 1600), (333, 96), (40, 6400)])
def test_act8_gelu_backward(dtype, rows, cols):
    torch = need_gpu()
    rng = np.random.default_rng(rows + cols)
    u = rng.standard_normal((rows, cols)).astype(np.float32) * 3
    u[0, :4] = [40.0, -40.0, 1e20, -1e20]
    x, _ = _given(u, dtype)
    q = torch.empty((rows, cols), dtype=torch.uint8, device="cuda")
    s = torch.empty((rows, cols // 32), dtype=torch.uint8, device="cuda")
    B.act8_save(x, q, s)
    dg, dv = _normal(rng, (rows, cols), dtype)
    du, clean = _guarded(torch, (rows, cols), x.dtype)
    g, clean_g = _guarded(torch, (rows, cols), x.dtype)
    B.act8_gelu_bwd(dg, q, s, du, g)
    torch.cuda.synchronize()
    uv = O.act8_restore(q.cpu().numpy(), s.cpu().numpy())
    gv, slope = O.gelu_parts(uv)
    # e = exp(-|w|): the argument's rounding, times |w|, and two steps of the function; then
    # about six products and sums, each of the larger of its terms; below 2^-126 nothing
    uc = np.clip(uv, -64, 64)
    w = np.abs(2 * np.sqrt(2 / np.pi) * (uc + 0.044715 * uc ** 3))
    near, far = 1 / (1 + np.exp(-w)), np.exp(-w) / (1 + np.exp(-w))
    rel = (6 * np.minimum(w, 200) + 16) * U
    s_err = np.where(uv >= 0, near * (far + 1) * rel, far * rel)
    third = np.abs(uc) * near * far * 2 * np.sqrt(2 / np.pi) * (1 + 3 * 0.044715 * uc ** 2)
    _within(g, gv, HALF[dtype] * np.abs(gv) + np.abs(uv) * (s_err + TINY) + TINY)
    _within(du, dv * slope, HALF[dtype] * np.abs(dv * slope) + np.abs(dv) * (s_err + 2 * rel * third + 1e-30) + TINY)
    assert clean() and clean_g()
    same = dg.clone()
    B.act8_gelu_bwd(same, q, s, same)
    torch.cuda.synchronize()
    assert torch.equal(same, du)


def test_act8_gelu_backward_of_nan_is_nan():
    torch = need_gpu()
    x = torch.zeros((1, 32), device="cuda")
    x[0, 3] = float("nan")
    q, s = torch.empty((1, 32), dtype=torch.uint8, device="cuda"), torch.empty((1, 1), dtype=torch.uint8, device="cuda")
    B.act8_save(x, q, s)
    du, g = torch.empty_like(x), torch.empty_like(x)
    B.act8_gelu_bwd(torch.ones_like(x), q, s, du, g)
    torch.cuda.synchronize()
    want = torch.zeros((1, 32), dtype=torch.bool)
    want[0, 3] = True
    assert torch.equal(torch.isnan(du).cpu(), want) and torch.equal(torch.isnan(g).cpu(), want)


DW = [(1, 8, 32), (2, 64, 64), (63, 72, 96), (64, 128, 128), (65, 136, 160), (333, 264, 288), (130, 520, 32),
      (1000, 256, 640), (5000, 64, 64), (129, 1000, 1056), (1, 4104, 2592), (700, 3848, 2688),
      (1025, 6000, 2560), (2000, 5000, 640), (6000, 1600, 1600), (5000, 1928, 1056), (3000, 264, 96), (4100, 1288, 1312), (600, 1000, 512)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tokens,n_out,n_in", DW)
def test_act8_weight_gradient(dtype, tokens, n_out, n_in):
    torch = need_gpu()
    print(f"[act8 dw] {dtype} {tokens} tokens, {n_out} x {n_in}", flush=True)
    rng = np.random.default_rng(tokens + n_out)
    x, _ = _normal(rng, (tokens, n_in), dtype)
    q = torch.empty((tokens, n_in), dtype=torch.uint8, device="cuda")
    s = torch.empty((tokens, n_in // 32), dtype=torch.uint8, device="cuda")
    B.act8_save(x, q, s)
    dy, dv = _normal(rng, (tokens, n_out), dtype)
    xv = O.act8_restore(q.cpu().numpy(), s.cpu().numpy())
    ref, mag = dv.T @ xv, np.abs(dv).T @ np.abs(xv)
    n = B.act8_gemm_dw_scratch_bytes(dy.dtype, tokens, n_out, n_in)
    scratch, kept = _guarded(torch, (n,), torch.uint8) if n else (None, lambda: True)
    dw, clean = _guarded(torch, (n_out, n_in), torch.float32)
    dw.fill_(float("nan"))
    B.act8_gemm_dw(dy, q, s, dw, scratch)
    torch.cuda.synchronize()
    tol = (tokens + 4) * U * mag  # fp32 products and sums
    _within(dw, ref, tol)
    assert clean() and kept()
    first = dw.clone()
    B.act8_gemm_dw(dy, q, s, dw, scratch)
    torch.cuda.synchronize()
    assert torch.equal(first, dw)
    B.act8_gemm_dw(dy, q, s, dw, scratch, accumulate=True)
    torch.cuda.synchronize()
    _within(dw, 2 * ref, 2 * tol + 2 * U * np.abs(2 * ref))
