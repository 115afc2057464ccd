"""The residual norm and the distillation loss on the GPU, through the C ABI, against the fp64
oracle.

Tolerances count roundings, as in test_gpu_operators.py: u = 2^-24, `half` half a step of the
output's type relative to the value.  A sum of fp32 terms that each thread adds one after the
other and that then meet in a tree is off by at most (additions on the longest way) u times the
sum of the magnitudes; each test says how long that way is."""
import numpy as np
import pytest

from oracle import operators as O
from paper_2206_04959_amd import binding as B
from paper_2206_04959_amd import synth
from tests.gpu_util import need_gpu
from tests.test_gpu_operators import HALF, TINY, U, _f64, _given, _guarded, _normal, _type

pytestmark = pytest.mark.gpu


def _close(got, ref, tol, what):
    got = _f64(got)
    bad = np.abs(got - ref) - tol
    assert got.shape == ref.shape, what
    assert np.isfinite(got).all() and (bad <= 0).all(), \
        (what, bad.max(), np.unravel_index(np.argmax(bad), bad.shape), np.abs(got - ref).max())


# ---------------------------------------------------------------------------
# Residual addition and norm
# ---------------------------------------------------------------------------

# widths at and around every layout of a row: 64 to 1024 threads of one chunk, 512 and 1024 of two
WIDTHS = [(1, 8), (5, 64), (257, 72), (9, 512), (3, 520), (66, 1024), (7, 1032), (5, 1536), (4, 1600), (6, 2048), (3, 2056),
          (4, 4096), (3, 4104), (2, 6144), (3, 6152), (5, 8192), (3, 8200), (2, 16384), (5, 13000)]
NORM = 48 * U   # 16 squares in a thread, 6 and 4 steps of the tree; halved by the root; division, root, products


def _rows(rng, rows, cols, dtype, spread=True):
    v = rng.standard_normal(size=(rows, cols), dtype=np.float32)
    if spread:  # a few channels many times larger
        v *= np.where(rng.random(cols) < 0.02, 30.0, 1.0).astype(np.float32)
    return _given(v, dtype)


def _sum_as_kept(x, r, dtype):
    """x + r in fp32, rounded to the type."""
    s = x.astype(np.float32) + r.astype(np.float32)
    return synth.bf16_bits_to_f64(synth.f32_to_bf16_bits(s)) if dtype == "bf16" else s.astype(np.float64)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols", WIDTHS)
@pytest.mark.parametrize("form", ["sum", "no sum", "plain", "on x", "on resid"])
def test_norm_forward(dtype, rows, cols, form):
    torch = need_gpu()
    print(f"[norm fwd] {dtype} {rows}x{cols} {form}", flush=True)
    rng = np.random.default_rng(rows + cols)
    dt = _type(torch, dtype)
    x, xv = _rows(rng, rows, cols, dtype)
    r, rv = (None, None) if form == "plain" else _rows(rng, rows, cols, dtype, False)
    g, gv = _normal(rng, (cols,), dtype, 0.1, 1.0)
    y, clean = _guarded(torch, (rows, cols), dt)
    s, sclean = _guarded(torch, (rows, cols), dt)
    eight = cols % 32 == 0
    q = torch.full((rows, cols), 77, dtype=torch.uint8, device="cuda") if eight else None
    sc = torch.full((rows, cols // 32), 77, dtype=torch.uint8, device="cuda") if eight else None
    out = {"sum": s, "no sum": None, "plain": None, "on x": x, "on resid": r}[form]
    h = xv if r is None else _sum_as_kept(xv, rv, dtype)
    B.add_rms_norm_fwd(x, g, y, resid=r, sum=out, q=q, scales=sc, eps=1e-5)
    torch.cuda.synchronize()
    ref = O.rms_norm(h, gv, float(np.float32(1e-5)))
    _close(y, ref, (HALF[dtype] + NORM) * np.abs(ref) + TINY, "y")
    assert clean() and sclean()
    if out is not None:
        assert np.array_equal(_f64(out), h)
    if form == "no sum":
        assert bool((s == 7).all())
    if eight:
        kept = O.act8_restore(q.cpu().numpy(), sc.cpu().numpy())
        most = np.repeat(np.abs(ref.reshape(rows, -1, 32)).max(-1), 32, axis=-1)
        # e4m3's rounding of a y that is itself off by NORM; below 2^-6 of the scale (at most
        # most / 224) a step of 2^-9 of it
        tol = np.maximum(2.0 ** -4 * np.abs(ref), 2.0 ** -10 * most / 224) * (1 + 2 * NORM) + 2 * NORM * np.abs(ref)
        assert (np.abs(kept - ref) <= tol).all()
        if dtype == "fp32":  # the codes of the very y that is stored
            q2, sc2 = torch.empty_like(q), torch.empty_like(sc)
            B.act8_save(y, q2, sc2)
            assert torch.equal(q, q2) and torch.equal(sc, sc2)
        only, onlysc = torch.empty_like(q), torch.empty_like(sc)
        if form in ("sum", "no sum", "plain"):  # y not wanted: the same codes
            B.add_rms_norm_fwd(x, g, resid=r, q=only, scales=onlysc, eps=1e-5)
            assert torch.equal(q, only) and torch.equal(sc, onlysc)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols", WIDTHS + [(16, 64), (17, 64), (1025, 64), (5000, 24), (1030, 1000), (2100, 1040), (1030, 4104), (40, 8200)])
@pytest.mark.parametrize("form", ["both", "no dsum", "on dy", "on dsum", "added"])
def test_norm_backward(dtype, rows, cols, form):
    torch = need_gpu()
    print(f"[norm bwd] {dtype} {rows}x{cols} {form}", flush=True)
    rng = np.random.default_rng(rows * 3 + cols)
    dt = _type(torch, dtype)
    h, hv = _rows(rng, rows, cols, dtype)
    dy, dyv = _normal(rng, (rows, cols), dtype)
    ds, dsv = (None, None) if form == "no dsum" else _normal(rng, (rows, cols), dtype)
    g, gv = _normal(rng, (cols,), dtype, 0.1, 1.0)
    dx, clean = _guarded(torch, (rows, cols), dt)
    dg, gclean = _guarded(torch, (cols,), torch.float32)
    start = rng.standard_normal(cols).astype(np.float32)
    if form == "added":
        dg.copy_(torch.from_numpy(start))
    out = {"on dy": dy, "on dsum": ds}.get(form, dx)
    scratch, sclean = _guarded(torch, (B.add_rms_norm_scratch_elems(rows, cols),), torch.float32)
    B.add_rms_norm_bwd(dy, h, g, out, dg, scratch, dsum=ds, eps=1e-5, accumulate=form == "added")
    torch.cuda.synchronize()
    rx, rg, mag, gmag = O.rms_norm_backward(dyv, hv, gv, dsv, float(np.float32(1e-5)))
    # the two sums over a row as in the forward pass, whole; a few products
    _close(out, rx, HALF[dtype] * np.abs(rx) + 100 * U * mag + TINY, "dx")
    # a thread's rows one after the other (256 to 2048 rows at once, or few rows of one workgroup),
    # then trees and the parts; each term is off by NORM
    way = rows / 256 + 40
    if form == "added":
        rg = rg + start
        gmag = gmag + np.abs(start)
    _close(dg, rg, (way * U + 2 * NORM) * gmag + TINY, "dgamma")
    assert clean() and gclean() and sclean()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cols", [64, 1024, 2048, 8192, 16384])
def test_norm_of_zeros_and_of_nonfinite_rows(dtype, cols):
    """A row of zeros gives zeros; NaN and infinity stay in their row (and in dgamma's columns)."""
    torch = need_gpu()
    print(f"[norm nonfinite] {dtype} {cols}", flush=True)
    rng = np.random.default_rng(cols)
    x, xv = _rows(rng, 6, cols, dtype)
    x[1] = 0
    x[3, 5] = float("nan")
    x[4, 7] = float("inf")
    g, gv = _normal(rng, (cols,), dtype, 0.1, 1.0)
    y, q = torch.empty_like(x), torch.empty(6, cols, dtype=torch.uint8, device="cuda")
    sc = torch.empty(6, cols // 32, dtype=torch.uint8, device="cuda")
    B.add_rms_norm_fwd(x, g, y, q=q, scales=sc)
    assert not y[1].any() and bool(torch.isnan(y[3]).all())
    assert bool(torch.isnan(y[4, 7])) and not y[4, :7].any()  # infinity / infinity, and 1 / infinity
    assert not (q[1] & 0x7f).any() and bool(((q[3] & 0x7f) == 0x7f).all())
    ref = O.rms_norm(xv[[0, 2, 5]], gv)
    _close(y[[0, 2, 5]], ref, (HALF[dtype] + NORM) * np.abs(ref) + TINY, "y")
    dy, dyv = _normal(rng, (6, cols), dtype)
    dx, dg = torch.empty_like(x), torch.empty(cols, device="cuda")
    scratch = torch.empty(B.add_rms_norm_scratch_elems(6, cols), device="cuda")
    B.add_rms_norm_bwd(dy, x, g, dx, dg, scratch)
    good = [0, 2, 5]
    rx, _, mag, _ = O.rms_norm_backward(dyv[good], xv[good], gv)
    _close(dx[good], rx, HALF[dtype] * np.abs(rx) + 100 * U * mag + TINY, "dx")
    assert bool(torch.isfinite(dx[1]).all()) and bool(torch.isnan(dx[3]).all()) and bool(torch.isnan(dg).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cols", [8, 64, 1024, 2048, 4096, 8192, 16384])
def test_norm_of_large_magnitudes(dtype, cols):
    """Rows whose squares leave fp32, alone or only in their sum, beside ordinary ones: magnitudes from below
    2^57 (16384 of them sum to 2^128) to the type's largest, in whole rows and in one feature."""
    torch = need_gpu()
    print(f"[norm large] {dtype} {cols}", flush=True)
    rng = np.random.default_rng(cols)
    powers = [0, 50, 55, 56, 57, 58, 60, 62, 63, 64, 65, 80, 100, 120, 125, 126]
    v = rng.uniform(1.0, 2.0, size=(2 * len(powers), cols)) * rng.choice([-1.0, 1.0], size=(2 * len(powers), cols))
    for i, p in enumerate(powers):
        v[i] *= 2.0 ** p
        v[len(powers) + i, cols // 2] *= 2.0 ** p
    x, xv = _given(v.astype(np.float32), dtype)
    g, gv = _normal(rng, (cols,), dtype, 0.1, 1.0)
    rows, eps = x.shape[0], float(np.float32(1e-6))
    y, eight = torch.empty_like(x), cols % 32 == 0
    q = torch.empty(rows, cols, dtype=torch.uint8, device="cuda") if eight else None
    sc = torch.empty(rows, cols // 32, dtype=torch.uint8, device="cuda") if eight else None
    B.add_rms_norm_fwd(x, g, y, q=q, scales=sc)
    ref = O.rms_norm(xv, gv, eps)
    norm = NORM + 8 * U  # the inverse root has 22 bits at 2^-128
    _close(y, ref, (HALF[dtype] + norm) * np.abs(ref) + TINY, "y")
    if eight and dtype == "fp32":
        q2, sc2 = torch.empty_like(q), torch.empty_like(sc)
        B.act8_save(y, q2, sc2)
        assert torch.equal(q, q2) and torch.equal(sc, sc2)
    dy, dyv = _normal(rng, (rows, cols), dtype)
    dx, dg = torch.empty_like(x), torch.empty(cols, device="cuda")
    for some in (slice(0, rows), slice(4, 8)):  # many workgroups; one
        n = dyv[some].shape[0]
        B.add_rms_norm_bwd(dy[some], x[some], g, dx[some], dg, torch.empty(B.add_rms_norm_scratch_elems(n, cols), device="cuda"))
        rx, rg, mag, gmag = O.rms_norm_backward(dyv[some], xv[some], gv, None, eps)
        _close(dx[some], rx, HALF[dtype] * np.abs(rx) + 110 * U * mag + TINY, "dx")
        _close(dg, rg, (rows / 256 + 40) * U * gmag + 2 * norm * gmag + TINY, "dgamma")


def test_norm_gradient_sums_integers_exactly():
    """h of +-1 and eps far below 1 ulp make n = h exactly; integer gradients then sum exactly in any
    order, so one lost or doubled term shows."""
    torch = need_gpu()
    rng = np.random.default_rng(8)
    for rows, cols in [(1, 64), (3, 64), (4097, 64), (5003, 1024), (1031, 2048), (1025, 4096), (700, 8192), (300, 16384)]:
        print(f"[norm bwd integers] {rows}x{cols}", flush=True)
        h = torch.from_numpy(rng.choice([-1.0, 1.0], size=(rows, cols)).astype(np.float32)).cuda()
        dy = torch.from_numpy(rng.integers(-8, 9, size=(rows, cols)).astype(np.float32)).cuda()
        dx, dg = torch.empty_like(h), torch.empty(cols, device="cuda")
        B.add_rms_norm_bwd(dy, h, torch.ones(cols, device="cuda"), dx, dg,
                           torch.empty(B.add_rms_norm_scratch_elems(rows, cols), device="cuda"), eps=1e-30)
        assert torch.equal(dg, (dy.double() * h.double()).sum(0).float())


# a width of each layout of the gradient, with the rows that it takes at once
@pytest.mark.parametrize("cols,at_once", [(8, 2048), (520, 1024), (1032, 512), (2056, 256), (4104, 256), (8200, 256)])
def test_norm_gradient_of_many_rows(cols, at_once):
    """Equal terms, whose roundings all go one way: h of 1 and an eps far below 1 ulp make n = 1, and a dy of
    1 + half a step of fp32 at half of 2048 (less one step at 1) would lose that half in each of the last 1024 of
    2048 additions in a row.  A column's additions, one behind the other: 256, the runs of 256, the tree."""
    torch = need_gpu()
    n = 4096 if cols == 8 else 2048   # rows a thread
    rows = n * at_once
    print(f"[norm bwd many rows] {rows}x{cols}", flush=True)
    dy = torch.full((rows, cols), 1.0 + n / 2 * 2.0 ** -24 - 2.0 ** -23, device="cuda")
    term = float(dy[0, 0])
    assert term != 1.0 and float(dy[0, 0] + n / 2) == n / 2 + 1.0
    h, dg = torch.ones_like(dy), torch.empty(cols, device="cuda")
    start = torch.full_like(dg, 3.0)
    scratch, clean = _guarded(torch, (B.add_rms_norm_scratch_elems(rows, cols),), torch.float32)
    for accumulate in (False, True):
        dy.fill_(term)
        if accumulate:
            dg.copy_(start)
        B.add_rms_norm_bwd(dy, h, torch.ones(cols, device="cuda"), dy, dg, scratch, eps=1e-30, accumulate=accumulate)
        torch.cuda.synchronize()
        want = np.full(cols, rows * term + (3.0 if accumulate else 0.0))
        _close(dg, want, (256 + n / 256 + 40) * U * want, "dgamma")
    assert clean()


def test_norm_gradient_of_half_a_million_rows():
    """Whole dgamma of 540000 x 8192, and of an odd part of its rows, against 64-bit sums."""
    torch = need_gpu()
    print("[norm bwd half a million rows]", flush=True)
    rows, cols, eps = 540000, 8192, float(np.float32(1e-6))
    h, dy = [torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    for a in range(0, rows, 60000):
        h[a:a + 60000].normal_(generator=gen)
        dy[a:a + 60000].normal_(mean=0.5, generator=gen)
    g = torch.randn(cols, device="cuda", generator=gen).bfloat16()
    dx, dg = torch.empty_like(h), torch.empty(cols, device="cuda")
    for n in (rows, 131073):
        want, size = torch.zeros(cols, dtype=torch.float64, device="cuda"), torch.zeros(cols, dtype=torch.float64, device="cuda")
        for a in range(0, n, 20000):
            v = h[a:min(a + 20000, n)].double()
            v *= torch.rsqrt(v.square().mean(1, keepdim=True) + eps)
            v *= dy[a:min(a + 20000, n)]
            want += v.sum(0)
            size += v.abs().sum(0)
        B.add_rms_norm_bwd(dy[:n], h[:n], g, dx[:n], dg,
                           torch.empty(B.add_rms_norm_scratch_elems(n, cols), device="cuda"))
        torch.cuda.synchronize()
        # each term is off by NORM and a product
        _close(dg, _f64(want), ((256 + rows / 256 / 256 + 40) * U + 2 * NORM) * _f64(size), "dgamma")


# ---------------------------------------------------------------------------
# Distillation loss
# ---------------------------------------------------------------------------

class _Loss:
    """One loss: inputs on the device, the oracle's results and their tolerances."""

    def __init__(self, torch, dtype, tokens, vocab, top, alpha, tau, seed=0, ld=None, ids="int32", teacher="bf16",
                 labels="int64", std=3.0, change=None):
        rng = np.random.default_rng(seed + vocab)
        self.torch, self.dtype, self.vocab = torch, dtype, vocab
        self.ld = ld or -(-vocab // 8) * 8
        z = rng.standard_normal(size=(tokens, self.ld), dtype=np.float32) * np.float32(std)
        self.at = np.stack([rng.choice(vocab, top, replace=top > vocab) for _ in range(tokens)]) if top else None
        t = -np.sort(-rng.standard_normal(size=(tokens, top)), axis=1).astype(np.float32) * 3
        self.lab = rng.integers(0, vocab, tokens)
        w = rng.standard_normal(tokens).astype(np.float32)
        if top and tokens > 3:
            self.at[1, top // 2:] = -1                   # fewer entries
            self.at[2] = [-1, vocab, 2 * vocab, -7][:1] * top  # none
            self.at[3] = self.at[3, 0]                   # one, many times
            self.at[0, 0] = self.lab[0]                  # the label is the first entry
        if tokens > 3:
            self.lab[1] = -100
            self.lab[tokens - 1] = vocab                 # no label
            w[tokens - 2] = 0.0
        if change:
            change(self, z, t, w)
        self.z, zv = _given(z, dtype)
        self.zv = zv[:, :vocab]
        self.t, self.tv = _given(t, teacher) if top else (None, None)
        self.w, self.wv = torch.from_numpy(w).cuda(), w.astype(np.float64)
        self.ids = torch.from_numpy(self.at).to(getattr(torch, ids)).cuda() if top else None
        self.labels = torch.from_numpy(self.lab).to(getattr(torch, labels)).cuda() if labels else None
        self.kw = dict(teacher_ids=self.ids, teacher_logits=self.t, labels=self.labels, alpha=alpha, temperature=tau)
        with np.errstate(all="ignore"):
            a = float(np.float32(alpha))
            self.loss, self.grad, m = O.distill(self.zv, self.at, self.tv, self.lab if labels else None, a, tau)
            # A sum of exponentials: 8 values a thread and chunk, at most 32 chunks (or batches of four, 128
            # values, rescaled once each), trees; an exponent's rounding counts |exponent| steps.
            n = 16 // (2 if dtype == "bf16" else 4)
            way = 300 + vocab / 512 if vocab > 16384 * n else 8 * 32 + 40
            self.loss_tol = U * ((way + 60) * (a * tau ** 2 + 1 - a) + 80 * m["loss"])
            d = np.abs(self.zv - np.max(self.zv, axis=1, keepdims=True))
            self.grad_tol = (HALF[dtype] * np.abs(self.grad)
                             + U * ((way + 100 + 8 * np.minimum(d, 100)) * m["plus"] + (top + 100) * m["minus"])) \
                * np.abs(self.wv)[:, None] + TINY
            self.grad = self.grad * self.wv[:, None]
        self.grad[self.wv == 0] = 0

    def whole(self):
        """(loss, gradient) by the call that gives both."""
        torch = self.torch
        loss, lclean = _guarded(torch, (self.z.shape[0],), torch.float32)
        dz, clean = _guarded(torch, tuple(self.z.shape), self.z.dtype)
        B.distill_loss_fwd_bwd(self.z, self.w, loss, dz, vocab=self.vocab, **self.kw)
        torch.cuda.synchronize()
        assert lclean() and clean()
        return loss, dz

    def apart(self):
        """The same by the forward call and its gradient, over the logits."""
        torch = self.torch
        T = self.z.shape[0]
        loss, stats = torch.empty(T, device="cuda"), torch.empty(T, 8, device="cuda")
        B.distill_loss_fwd(self.z, stats, loss, vocab=self.vocab, **self.kw)
        dz = self.z.clone()
        B.distill_loss_bwd(dz, stats, self.w, dz, vocab=self.vocab, **self.kw)
        torch.cuda.synchronize()
        return loss, dz

    def shares(self, ranks):
        torch = self.torch
        T, per = self.z.shape[0], -(-self.vocab // ranks)
        ld = -(-per // 8) * 8
        parts, dz = torch.empty(ranks, T, 8, device="cuda"), []
        spans = [(r * per, max(0, min(per, self.vocab - r * per))) for r in range(ranks)]
        pieces = []
        for first, n in spans:
            p = torch.full((T, ld), float("nan"), device="cuda", dtype=self.z.dtype)
            p[:, :n] = self.z[:, first:first + n]
            pieces.append(p)
        for p, part, (first, n) in zip(pieces, parts, spans):
            B.distill_loss_fwd(p, part, vocab=n, first_id=first, vocab_total=self.vocab, **self.kw)
        stats, loss = torch.empty(T, 8, device="cuda"), torch.empty(T, device="cuda")
        B.distill_loss_join(parts, stats, loss, alpha=self.kw["alpha"], temperature=self.kw["temperature"])
        for p, (first, n) in zip(pieces, spans):
            d = torch.empty_like(p)
            B.distill_loss_bwd(p, stats, self.w, d, vocab=n, first_id=first, vocab_total=self.vocab, **self.kw)
            assert not d[:, n:].any()
            dz.append(d[:, :n])
        torch.cuda.synchronize()
        return loss, torch.cat(dz, 1)

    def check(self, got, what, rows=slice(None)):
        loss, dz = got
        _close(loss[rows], self.loss[rows], self.loss_tol[rows], what + ": loss")
        _close(dz[rows, :self.vocab], self.grad[rows], self.grad_tol[rows], what + ": gradient")
        assert not dz[rows, self.vocab:].any(), what + ": padding"


MIX = [(0.5, 1.0), (0.5, 2.0), (0.3, 4.0), (0.6, 3.0), (1.0, 2.0), (0.0, 1.0)]
# vocabularies at and behind every row layout (chunks of 8 in bf16, 4 in fp32), and odd ones
VOCABS = [1, 7, 8, 9, 63, 512, 513, 1000, 1024, 1025, 2048, 2049, 3584, 3585, 4097, 6656, 6657, 7168, 7169, 13312, 13313]
WIDE = [26624, 26625, 38913, 50257, 53248, 53249, 65536, 65537, 77825, 102401, 131073, 200003]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("alpha,tau", MIX)
@pytest.mark.parametrize("vocab", VOCABS)
def test_loss_and_gradient(dtype, vocab, alpha, tau):
    torch = need_gpu()
    print(f"[distill] {dtype} vocab {vocab} alpha {alpha} T {tau}", flush=True)
    case = _Loss(torch, dtype, 7, vocab, min(vocab, 37), alpha, tau)
    case.check(case.whole(), "both")
    case.check(case.apart(), "apart")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("vocab", WIDE)
def test_loss_and_gradient_of_wide_rows(dtype, vocab):
    torch = need_gpu()
    for alpha, tau in ((0.5, 2.0), (0.6, 3.0)):
        print(f"[distill] {dtype} vocab {vocab} alpha {alpha} T {tau}", flush=True)
        case = _Loss(torch, dtype, 5, vocab, 64, alpha, tau, ids="int64", teacher="fp32", labels="int32")
        case.check(case.whole(), "both")
        case.check(case.apart(), "apart")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("top", [0, 1, 3, 4, 5, 63, 64, 65, 127, 256, 257, 600, 1023, 1024])
def test_numbers_of_entries(dtype, top):
    torch = need_gpu()
    for vocab in (2000, 30001):
        print(f"[distill entries] {dtype} top {top} vocab {vocab}", flush=True)
        case = _Loss(torch, dtype, 6, vocab, top, 0.5, 2.0)
        case.check(case.whole(), "both")
        case.check(case.apart(), "apart")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("top", [204, 205, 409, 410, 819, 820])
def test_many_entries(dtype, top):
    """Numbers of entries from which a row has more threads, in rows and on calls of each layout."""
    torch = need_gpu()
    for tokens, vocab in ((6, 600), (6, 4097), (6, 8192), (6, 8200), (5, 28672), (5, 28680), (1025, 700), (1025, 3500)):
        print(f"[distill entries] {dtype} top {top} tokens {tokens} vocab {vocab}", flush=True)
        case = _Loss(torch, dtype, tokens, vocab, top, 0.5, 2.0)
        case.check(case.whole(), "both")
        case.check(case.apart(), "apart")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("top", [24, 25, 50, 51, 101, 102, 203, 204, 408, 409, 818, 819, 1024])
@pytest.mark.parametrize("clash", [False, True])
def test_fullest_tables(dtype, top, clash):
    """Most entries that a table of each size has (four fifths of its slots, less one), and one more, which has
    the next size (so have the rules for rows with many entries, at 204, 409 and 819).  With `clash` all columns begin their
    search in the table's last two slots, so that it goes on from its start, past many others."""
    torch = need_gpu()
    slots = 32
    while 4 * slots < 5 * (top + 1):
        slots *= 2
    for tokens, vocab in ((5, 4097), (5, 8192), (5, 28672), (5, 60000), (1025, 3500), (5, 140000)):
        print(f"[distill tables] {dtype} top {top} clash {clash} tokens {tokens} vocab {vocab}", flush=True)

        def change(self, z, t, w):
            if not clash:
                return
            c = np.arange(vocab, dtype=np.uint64)
            home = ((c * 2654435761 & 0xffffffff) >> 8) & (slots - 1)
            c = c[home >= slots - 2]
            rng = np.random.default_rng(top)
            for i in range(tokens):
                if i not in (2, 3):
                    self.at[i] = rng.choice(c, top, replace=len(c) < top)
            self.lab[0] = self.at[0, top // 2]

        case = _Loss(torch, dtype, tokens, vocab, top, 0.5, 2.0, change=change)
        case.check(case.whole(), "both")
        case.check(case.apart(), "apart")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("ranks", [1, 2, 3, 8])
@pytest.mark.parametrize("alpha,tau", [(0.5, 2.0), (0.6, 3.0), (1.0, 1.0), (0.0, 1.0)])
def test_shares_of_the_vocabulary(dtype, ranks, alpha, tau):
    torch = need_gpu()
    for vocab in (37, 5003):
        print(f"[distill shares] {dtype} {ranks} ranks vocab {vocab} alpha {alpha} T {tau}", flush=True)
        case = _Loss(torch, dtype, 9, vocab, 20, alpha, tau)
        case.check(case.shares(ranks), "shares")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tokens", [1, 2, 511, 512, 700, 1024, 1025])
def test_numbers_of_tokens(dtype, tokens):
    """Fewer and more tokens than there are where the row layout and the gradient's pieces change."""
    torch = need_gpu()
    for vocab in (1200, 2500, 3600, 7160, 9000, 14000):
        print(f"[distill tokens] {dtype} {tokens} vocab {vocab}", flush=True)
        case = _Loss(torch, dtype, tokens, vocab, 16, 0.5, 2.0)
        case.check(case.whole(), "both")
        case.check(case.apart(), "apart")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("vocab,top", [(60, 12), (2500, 12), (9000, 300), (27000, 40), (140000, 12), (3000, 1024)])
@pytest.mark.parametrize("tau", [1.0, 2.0, 3.0])
def test_repeated_ids_of_small_probability(dtype, vocab, top, tau):
    """An id that is there twice or more, with logits 30 to 60 T below the teacher's largest, and a student whose
    logit there is as low: the gradient there is that of the sum of its probabilities, in all its digits."""
    torch = need_gpu()
    print(f"[distill repeats] {dtype} vocab {vocab} top {top} T {tau}", flush=True)

    def change(self, z, t, w):
        low = [5, 17, 29, 41, 53]
        z[:, low] = -400.0
        w[:] = 1.0
        for i in range(8):
            self.lab[i] = 3 if i else 17    # (a label there, too)
            t[i] = -tau * np.linspace(0.0, 60.0, top)
            at = 100 + np.arange(top) if vocab > top + 100 else 50 - np.arange(top) % 4 * 2
            n = 5 if top > 20 else 3
            for k, c in enumerate(low[:n]):  # two entries each, or many; far apart or not
                at[top // 2 + k::n] = c
            if i % 2:
                t[i, top // 2 + i % 5::2] -= 20.0 * tau
            order = np.random.default_rng(i).permutation(top)
            self.at[i], t[i] = at[order], t[i][order]

    case = _Loss(torch, dtype, 9, vocab, top, 0.5, tau, teacher="fp32", change=change)
    _, _, m = O.distill(case.zv, case.at, case.tv, case.lab, 0.5, tau)
    # a p is off by two roundings of its exponent, up to 80 (in steps of e)
    case.grad_tol = case.grad_tol + 4 * 80 * U * m["minus"] * np.abs(case.wv)[:, None]
    small = np.abs(case.grad[:8][:, [5, 29]])
    assert (0 < small).all() and small.max() < 2.0 ** -38
    for got, what in ((case.whole(), "both"), (case.apart(), "apart"), (case.shares(2), "shares")):
        case.check(got, what)


@pytest.mark.parametrize("ranks", [1, 255, 256, 257, 2 ** 16])
def test_join_of_many_ranks(ranks):
    """Equal sums, whose roundings all go one way: 1 + half a step of fp32 at 2^15 (less one step at 1) would lose that
    half in each of the last 2^15 of 2^16 additions in a row.  There are 256 in a row, and 256 of those."""
    torch = need_gpu()
    print(f"[distill join] {ranks} ranks", flush=True)
    T, alpha, tau, each = 300, 0.5, 2.0, 1.0 + 2.0 ** -9 - 2.0 ** -23
    parts = torch.zeros(ranks, T, 8, device="cuda")
    parts[:, :, 0] = -3.0
    parts[:, :, 1:3] = each
    parts[ranks // 2, :, 3:6] = torch.tensor([-0.5, 1.0, 1.0], device="cuda")  # the entries' rank and the label's
    parts[:, :, 6:] = torch.tensor([2.5, 1.5], device="cuda")
    stats, loss = torch.empty(T, 8, device="cuda"), torch.empty(T, device="cuda")
    B.distill_loss_join(parts, stats, loss, alpha=alpha, temperature=tau)
    torch.cuda.synchronize()
    want = np.tile([-3.0, ranks * each, ranks * each, -0.5, 1.0, 1.0, 2.5, 1.5], (T, 1))
    way = min(ranks, 256) + ranks / 256
    _close(stats, want, np.array([0, way * U * ranks * 1.01, way * U * ranks * 1.01, 0, 0, 0, 0, 0]), "stats")
    ref = 0.5 + (alpha * tau ** 2 + 1 - alpha) * np.log(ranks * each)
    _close(loss, np.full(T, ref), (way + 8) * U * (alpha * tau ** 2 + 1 - alpha) + 8 * U * abs(ref), "loss")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [30, 1000, 7000, 53300, 140000])
def test_offsets_and_masks(dtype, vocab):
    """A common offset of the logits changes nothing; masked columns (-infinity, or the type's lowest
    value) have no probability; a row of lowest values only is uniform."""
    torch = need_gpu()
    print(f"[distill masks] {dtype} vocab {vocab}", flush=True)
    low = float(torch.finfo(_type(torch, dtype)).min)

    def change(self, z, t, w):
        z[0] += 1024.0
        z[1] -= 5000.0
        z[2, 1::2] = -np.inf
        z[3, 1::2] = low
        z[4] = low
        z[5] = -np.inf
        z[5, vocab // 2] = 1.0
        z[6] *= 2.0 ** 60           # far apart: one token has all the probability
        self.at[:7] = (self.at[:7] // 2 * 2) % vocab // 2 * 2  # entries and labels at even columns
        self.lab[:7] = self.lab[:7] // 2 * 2 % vocab // 2 * 2
        self.at[5], self.lab[5] = vocab // 2, vocab // 2
        t[0, 3:] = -np.inf          # no entries
        w[:7] = [1, 2, -1, 0.5, 1, 1, 1]

    for alpha, tau in ((0.5, 2.0), (0.4, 3.0), (0.5, 1.0), (0.4, 4.0)):
        case = _Loss(torch, dtype, 9, vocab, 8, alpha, tau, teacher="fp32", change=change)
        assert np.isfinite(case.loss).all()
        for got, what in ((case.whole(), "both"), (case.apart(), "apart"), (case.shares(2), "shares")):
            case.check(got, what)
            dz = _f64(got[1])
            assert not dz[2, 1:vocab:2].any() and not dz[3, 1:vocab:2].any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [50, 2000, 60000, 140000])
@pytest.mark.parametrize("tau", [1.0, 2.0, 3.0, 900.0, 2.0 ** -10])
def test_large_offsets(dtype, vocab, tau):
    """Offsets on both sides of 2^16, from which on the base is subtracted first, up to 2^40, at ordinary and extreme
    temperatures; the spread grows with the type's steps out there, so that several logits count."""
    torch = need_gpu()
    print(f"[distill offsets] {dtype} vocab {vocab} T {tau}", flush=True)
    places = [0.0, 2.0 ** 15, -2.0 ** 15, 65000.0, -65000.0, 2.0 ** 17, -2.0 ** 17, 2.0 ** 24, -2.0 ** 30, 2.0 ** 40, -2.0 ** 50]

    def change(self, z, t, w):
        for i, p in enumerate(places):
            z[i] = z[i] * max(1.0, min(tau, 50.0)) + p
        w[:] = 1.0

    case = _Loss(torch, dtype, len(places) + 3, vocab, 8, 0.5, tau, teacher="fp32", change=change)
    assert np.isfinite(case.loss).all()
    # An exponent x is off by up to two steps of itself (at T = 2^-10 by more than grad_tol's 8 |z - max|
    # holds), and exp(-x) x is at most 1/e.
    case.grad_tol = case.grad_tol + 4 * U * (0.5 * tau + 0.5)
    for got, what in ((case.whole(), "both"), (case.apart(), "apart"), (case.shares(3), "shares")):
        case.check(got, what)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [45, 3001, 60001, 140001])
def test_nonfinite_rows_stay_alone(dtype, vocab):
    torch = need_gpu()
    print(f"[distill nonfinite] {dtype} vocab {vocab}", flush=True)

    def change(self, z, t, w):
        z[0, vocab - 1] = np.nan
        z[1, vocab // 3] = np.inf
        z[2] = -np.inf
        t[3, 1] = np.nan
        t[4, 0] = np.inf
        z[5] = np.nan               # no entry and no label
        self.at[5], self.lab[5] = -1, -1
        z[6] = np.nan               # a weight of 0
        w[:] = 1.0
        w[6] = 0.0
        self.at[:5], self.lab[:5] = np.arange(8), 2
        z[7, vocab // 2] = -np.inf  # the label has no probability
        self.lab[7] = vocab // 2

    for alpha, tau in ((0.5, 2.0), (0.4, 3.0), (0.5, 1.0)):
        case = _Loss(torch, dtype, 10, vocab, 8, alpha, tau, teacher="fp32", change=change)
        for got, what in ((case.whole(), "both"), (case.apart(), "apart"), (case.shares(2), "shares")):
            loss, dz = _f64(got[0]), _f64(got[1])
            assert np.isnan(loss[:5]).all() and np.isnan(dz[:5, :vocab]).all(), what
            assert loss[5] == 0 and not dz[5].any() and np.isnan(loss[6]) and not dz[6].any(), what
            assert loss[7] == np.inf and np.isfinite(dz[7]).all(), what
            assert not dz[:, vocab:].any(), what
            case.check(got, what, slice(8, 10))
    one = _Loss(torch, dtype, 10, vocab, 8, 0.0, 1.0, change=change)  # entries are not looked at
    assert np.isfinite(_f64(one.whole()[0])[3:5]).all()


# the layouts of few and of many rows part below 3584 chunks only
PLACES = [(12, v) for v in (30, 1001, 2047, 3500, 4100, 7001, 13300, 26700, 50257, 77000, 102000, 131001, 140001)] + \
    [(1030, v) for v in (30, 1001, 2047, 3500, 4100, 7001, 13300, 26700)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tokens,vocab", PLACES)
def test_gradient_in_the_place_of_the_logits(dtype, tokens, vocab):
    """Both calls that may write the gradient over the logits, in every layout of a row, give the bits that they give
    apart: ordinary rows, rows far from 0, masked ones, NaN, tokens without anything and without weight."""
    torch = need_gpu()
    print(f"[distill in place] {dtype} tokens {tokens} vocab {vocab}", flush=True)
    dt, bits = _type(torch, dtype), torch.int16 if dtype == "bf16" else torch.int32
    gen = torch.Generator(device="cuda")
    gen.manual_seed(vocab)
    ld, top = -(-vocab // 8) * 8 + 8, 20
    z = (3 * torch.randn(tokens, ld, device="cuda", generator=gen)).to(dt)
    z[1] += 2.0 ** 20
    z[2, 1::2] = -float("inf")
    z[3] = torch.finfo(dt).min
    z[4] = float("nan")
    ids = torch.randint(0, vocab, (tokens, top), device="cuda", generator=gen)
    ids[5], ids[6, ::2] = -1, ids[6, 1]
    lab = torch.randint(0, vocab, (tokens,), device="cuda", generator=gen)
    lab[5], w = -100, torch.rand(tokens, device="cuda", generator=gen)
    w[7] = 0.0
    for alpha, tau in ((0.5, 2.0), (0.4, 3.0)):
        kw = dict(teacher_ids=ids, teacher_logits=torch.randn(tokens, top, device="cuda", generator=gen), labels=lab, alpha=alpha,
                  temperature=tau, vocab=vocab)
        loss, loss2, stats = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda"), torch.empty(tokens, 8, device="cuda")
        apart, place = torch.empty_like(z), z.clone()
        B.distill_loss_fwd_bwd(z, w, loss, apart, **kw)
        B.distill_loss_fwd_bwd(place, w, loss2, place, **kw)
        assert torch.equal(loss.view(torch.int32), loss2.view(torch.int32))
        assert torch.equal(apart.view(bits), place.view(bits))
        B.distill_loss_fwd(z, stats, **kw)
        B.distill_loss_bwd(z, stats, w, apart, **kw)
        place.copy_(z)
        B.distill_loss_bwd(place, stats, w, place, **kw)
        torch.cuda.synchronize()
        assert torch.equal(apart.view(bits), place.view(bits))
        assert not apart[:, vocab:].any()


@pytest.mark.parametrize("ranks", [1, 3])
def test_ids_far_outside_the_vocabulary(ranks):
    """Ids and labels at the ends of 64 bits, and around a share's ends, are no entries."""
    torch = need_gpu()
    for vocab in (90, 5000):
        print(f"[distill ids] {ranks} ranks vocab {vocab}", flush=True)
        wild = [-2 ** 63, -2 ** 63 + vocab, -2 ** 62, -1, vocab, 2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63 - 1, -2 ** 32 + 1]

        def change(self, z, t, w):
            for k, i in enumerate(wild):
                self.at[k % 8, 1 + k // 8] = i
                self.lab[k % 8] = i

        case = _Loss(torch, "bf16", 9, vocab, 12, 0.5, 2.0, ids="int64", change=change)
        case.check(case.shares(ranks) if ranks > 1 else case.whole(), "wild ids")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_losses_of_the_two_calls_and_runs_are_the_same_bits(dtype):
    """Nothing depends on timing: the same bits again, with repeated ids and many entries."""
    torch = need_gpu()
    for vocab, top in ((900, 64), (20000, 300), (50304, 1024)):
        print(f"[distill again] {dtype} {vocab} {top}", flush=True)

        def change(self, z, t, w):
            self.at[:] = self.at // 3 % max(1, vocab // 40)

        case = _Loss(torch, dtype, 64, vocab, top, 0.5, 2.0, change=change)
        bits = torch.int16 if dtype == "bf16" else torch.int32
        first, apart = case.whole(), case.apart()
        for _ in range(3):
            for a, b in ((first, case.whole()), (apart, case.apart())):
                assert torch.equal(a[0].view(torch.int32), b[0].view(torch.int32))
                assert torch.equal(a[1].view(bits), b[1].view(bits))


def test_gradient_against_differences():
    """The gradient against differences of the kernel's own loss.  With steps of 2^-6 in fp32 a
    central difference is off by step^2 / 6 times a third derivative below 1 (times 2 T^2 for
    both terms' weights), and by the losses' roundings over the step."""
    torch = need_gpu()
    case = _Loss(torch, "fp32", 8, 300, 10, 0.5, 2.0, std=1.0)
    loss, dz = case.whole()
    step, rng = 2.0 ** -6, np.random.default_rng(5)
    for _ in range(8):
        v = torch.from_numpy(rng.choice([-1.0, 1.0], size=(8, 1)) * (rng.random((8, case.ld)) < 0.02)).float().cuda()
        ends = []
        for sign in (1, -1):
            l = torch.empty(8, device="cuda")
            B.distill_loss_fwd(case.z + sign * step * v, loss=l, vocab=300, **case.kw)
            ends.append(_f64(l))
        slope = (ends[0] - ends[1]) / (2 * step) * case.wv
        want = (_f64(dz) * v.double().cpu().numpy()).sum(1)
        tol = np.abs(case.wv) * (step ** 2 / 6 * 8 + 2 * case.loss_tol / step) + 1e-6
        assert (np.abs(slope - want) <= tol).all(), (slope - want, tol)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("alpha,tau", [(0.0, 1.0), (0.5, 2.0), (0.4, 3.0), (0.5, 900.0)])
def test_sums_of_the_widest_rows(dtype, alpha, tau):
    """Rows of nearly 2^28 columns (2^19 a thread): one logit above equal ones, normal ones, ascending ones and
    one far from 0, against 64-bit sums.  A thread's terms: 32 in a row, 128 such sums with a rescaling, 128 of
    those in bf16 and 256 in fp32, each rescaling a factor that is off by two steps and a product, then the tree; or 1024 and 512
    where the maximum is far."""
    torch = need_gpu()
    print(f"[distill widest] {dtype} alpha {alpha} T {tau}", flush=True)
    V, ld, top, way = 2 ** 28 - 3, 2 ** 28, 4, 1700
    dt, f64 = _type(torch, dtype), torch.float64
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    z = torch.empty(4, ld, dtype=dt, device="cuda")
    z[0], z[0, 12345678] = -0.75, 0.0
    z[1].normal_(std=2.0, generator=gen)
    z[2] = torch.linspace(-8.0, 0.0, ld, device="cuda")
    z[3], z[3, 200000001] = 2.0 ** 17 - 1024.0, 2.0 ** 17
    ids = torch.tensor([[12345678, 5, 2 ** 28 - 4, 7], [1, 2, 3, 4], [2 ** 28 - 4, 2 ** 27, 9, 3], [200000001, 1, 2, 3]], device="cuda")
    lab = torch.tensor([12345678, 77, 2 ** 28 - 4, 200000001], device="cuda")
    t = torch.randn(4, top, device="cuda", generator=gen)
    w = torch.tensor([1.0, 0.5, 2.0, -1.0], device="cuda")
    kw = dict(teacher_ids=ids, teacher_logits=t, labels=lab, alpha=alpha, temperature=tau, vocab=V)
    loss, loss2, stats, dz = torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), torch.empty(4, 8, device="cuda"), \
        torch.empty_like(z)
    B.distill_loss_fwd_bwd(z, w, loss, dz, **kw)
    B.distill_loss_fwd(z, stats, loss2, **kw)
    a, piece = float(np.float32(alpha)), 2 ** 24
    cuts = [slice(c, min(c + piece, V)) for c in range(0, V, piece)]
    for r in range(4):
        m = z[r, :V].max().to(f64)
        s_t, s_1 = [sum(torch.exp((z[r, c].to(f64) - m) / k).sum() for c in cuts) for k in (tau, 1.0)]
        p = torch.softmax(t[r].to(f64) / tau, 0)
        d, dl = z[r, ids[r]].to(f64) - m, z[r, lab[r]].to(f64) - m
        want = a * tau ** 2 * (p * (torch.log(p) - d / tau + torch.log(s_t))).sum() + (1 - a) * (torch.log(s_1) - dl)
        size = a * tau ** 2 * (p * (torch.log(p).abs() + d.abs() / tau + 1)).sum() + (1 - a) * (dl.abs() + 1)
        tol = U * ((way + 60) * (a * tau ** 2 + 1 - a) + 80 * float(size))
        for l in (loss, loss2):
            assert abs(float(l[r]) - float(want)) <= tol, (r, float(l[r]), float(want), tol)
    for turn in range(2):  # the gradient of the call that gives both; the one from the statistics, in the logits' place
        got = dz
        if turn:
            got = z.clone()
            B.distill_loss_bwd(got, stats, w, got, **kw)
        for r in range(4):
            m = z[r, :V].max().to(f64)
            s_t, s_1 = [sum(torch.exp((z[r, c].to(f64) - m) / k).sum() for c in cuts) for k in (tau, 1.0)]
            p = torch.softmax(t[r].to(f64) / tau, 0)
            for c in cuts:
                d = z[r, c].to(f64) - m
                plus = a * tau * torch.exp(d / tau) / s_t + (1 - a) * torch.exp(d) / s_1
                minus = torch.zeros_like(plus)
                for k in range(top):
                    if c.start <= int(ids[r, k]) < c.stop:
                        minus[int(ids[r, k]) - c.start] += a * tau * p[k]
                if c.start <= int(lab[r]) < c.stop:
                    minus[int(lab[r]) - c.start] += 1 - a
                tol = HALF[dtype] * (plus - minus).abs() + U * ((way + 100 + 8 * d.abs().clamp(max=100)) * plus + (top + 100) * minus)
                off = (got[r, c].to(f64) - float(w[r]) * (plus - minus)).abs()
                assert bool((off <= tol * abs(float(w[r])) + TINY).all()), (turn, r, c, float((off - tol).max()))
        assert not got[:, V:].any()


@pytest.mark.parametrize("vocab", [100, 2000])
def test_a_term_without_weight_needs_no_arrays(vocab):
    """At the C entry points, alpha = 0 with `top` entries but no arrays of them is the labels' loss, and
    alpha = 1 with a label type that is none the teacher's."""
    torch = need_gpu()
    print(f"[distill weights] vocab {vocab}", flush=True)
    T, ld, stream = 5, -(-vocab // 8) * 8, torch.cuda.current_stream().cuda_stream
    L, case = B.lib(), _Loss(torch, "bf16", T, vocab, 6, 0.5, 2.0)
    for alpha, top, given in ((0.0, 6, (None, None, case.labels.data_ptr())),
                              (1.0, 6, (case.ids.data_ptr(), case.t.data_ptr(), case.labels.data_ptr()))):
        got, want = [[torch.empty(T, device="cuda"), torch.empty(T, 8, device="cuda"), torch.empty(T, device="cuda"),
                      torch.empty_like(case.z), torch.empty_like(case.z)] for _ in range(2)]
        kinds = (0, 0, 1) if alpha == 0.0 else (0, 0, 9)
        for loss, stats, loss2, dz, dz2 in (got,):
            mix = (top, *kinds, alpha, 2.0, case.z.data_ptr(), *given)
            assert L.merak_distill_loss_fwd_bwd(0, T, vocab, ld, *mix, case.w.data_ptr(), loss.data_ptr(), dz.data_ptr(),
                                                stream) == 0
            assert L.merak_distill_loss_fwd(0, T, vocab, ld, 0, vocab, *mix, stats.data_ptr(), loss2.data_ptr(), stream) == 0
            assert L.merak_distill_loss_bwd(0, T, vocab, ld, 0, vocab, *mix, stats.data_ptr(), case.w.data_ptr(),
                                            dz2.data_ptr(), stream) == 0
        kw = dict(labels=case.labels) if alpha == 0.0 else dict(teacher_ids=case.ids, teacher_logits=case.t)
        kw.update(alpha=alpha, temperature=2.0, vocab=vocab)
        B.distill_loss_fwd_bwd(case.z, case.w, want[0], want[3], **kw)
        B.distill_loss_fwd(case.z, want[1], want[2], **kw)
        B.distill_loss_bwd(case.z, want[1], case.w, want[4], **kw)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))
