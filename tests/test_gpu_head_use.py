"""The residual norm and the distillation loss as a program uses them: the end of a training step
through both and the framework's own kernels, on one rank and on two, captured into graphs, on
side streams, on arrays beyond 2^32 elements and calls of several launches."""
import numpy as np
import pytest

from oracle import operators as O
from paper_2206_04959_amd import binding as B
from tests.gpu_util import need_gpu, rel_err
from tests.test_gpu_operators import _f64, _normal, _type

pytestmark = pytest.mark.gpu


def _step(torch, dtype, ranks, seed=3):
    """Residual and norm (kept in 8 bits), the head's product, loss, its gradient, the head's weight gradient from
    the kept input, and the norm's gradient.  Returns what the GPU made and what fp64 makes of it."""
    rng = np.random.default_rng(seed)
    T, h, V, K, alpha, tau = 128, 192, 640, 12, 0.4, 2.0
    dt, f32 = _type(torch, dtype), torch.float32
    new = lambda *s, dtype=dt: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
    x, xv = _normal(rng, (T, h), dtype)
    r, rv = _normal(rng, (T, h), dtype)
    g, gv = _normal(rng, (h,), dtype, 0.1, 1.0)
    W, Wv = _normal(rng, (V, h), dtype, 0.1)
    ds, dsv = _normal(rng, (T, h), dtype, 0.01)
    at = np.stack([rng.permutation(V)[:K] for _ in range(T)])
    at[rng.random((T, K)) < 0.1] = -1
    t, tv = _normal(rng, (T, K), "fp32", 3.0)
    lab = rng.integers(0, V, T)
    lab[rng.random(T) < 0.2] = -100
    w = np.where(lab >= 0, 1.0 / T, 0.5 / T).astype(np.float32)
    kw = dict(teacher_ids=torch.from_numpy(at).cuda(), teacher_logits=t, labels=torch.from_numpy(lab).cuda(), alpha=alpha,
              temperature=tau)
    wt = torch.from_numpy(w).cuda()

    # forward
    s, y, q, sc = new(T, h), new(T, h), new(T, h, dtype=torch.uint8), new(T, h // 32, dtype=torch.uint8)
    B.add_rms_norm_fwd(x, g, y, resid=r, sum=s, q=q, scales=sc)
    per = V // ranks
    loss = new(T, dtype=f32)
    shares = [W[i * per:(i + 1) * per] for i in range(ranks)]
    logits = [new(T, per) for _ in range(ranks)]
    for z, part in zip(logits, shares):
        B.gemm(y, part, z, T, per, h)
    if ranks == 1:
        B.distill_loss_fwd_bwd(logits[0], wt, loss, logits[0], **kw)  # the gradient in the logits' place
    else:
        parts, stats = new(ranks, T, 8, dtype=f32), new(T, 8, dtype=f32)
        own = [dict(vocab=per, first_id=i * per, vocab_total=V) for i in range(ranks)]
        for z, p, o in zip(logits, parts, own):
            B.distill_loss_fwd(z, p, **o, **kw)
        B.distill_loss_join(parts, stats, loss, alpha=alpha, temperature=tau)
        for z, o in zip(logits, own):
            B.distill_loss_bwd(z, stats, wt, z, **o, **kw)

    # backward
    dW, dy = new(V, h, dtype=f32), torch.zeros(T, h, device="cuda")
    for i, (z, part) in enumerate(zip(logits, shares)):
        d = dW[i * per:(i + 1) * per]
        nb = B.act8_gemm_dw_scratch_bytes(dt, T, per, h)
        B.act8_gemm_dw(z, q, sc, d, new(max(nb, 1), dtype=torch.uint8))
        one = new(T, h, dtype=f32)
        B.gemm(z, part, one, T, h, per, b_trans=1, epilogue=B.EPI_F32, dtype=B.BF16 if dtype == "bf16" else B.FP32)
        dy += one                                      # the ranks' sum
    dy = dy.to(dt)
    dx, dg = ds.clone(), new(h, dtype=f32)
    B.add_rms_norm_bwd(dy, s, g, dx, dg, new(B.add_rms_norm_scratch_elems(T, h), dtype=f32), dsum=dx)
    torch.cuda.synchronize()

    # fp64
    S = xv + rv
    Y = O.rms_norm(S, gv)
    L, D, _ = O.distill(Y @ Wv.T, at, tv, lab, alpha, tau)
    D = D * w[:, None].astype(np.float64)
    kept = O.act8_restore(q.cpu().numpy(), sc.cpu().numpy())
    X, G, _, _ = O.rms_norm_backward(D @ Wv, S, gv, dsv)
    got = dict(sum=s, y=y, loss=loss, dlogits=torch.cat(logits, 1), dW=dW, dx=dx, dg=dg)
    return got, dict(sum=S, y=Y, loss=L, dlogits=D, dW=D.T @ kept, dx=X, dg=G), kept


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("ranks", [1, 2])
def test_end_of_a_training_step(dtype, ranks):
    """Bars: the framework's stated ones, 2e-2 in bf16 and 1e-4 in the fp32 check mode.  The oracle takes the kept
    values as the GPU kept them (a value on the border of two codes may go either way)."""
    torch = need_gpu()
    print(f"[end of step] {dtype} {ranks} ranks", flush=True)
    got, want, kept = _step(torch, dtype, ranks)
    bar = 2e-2 if dtype == "bf16" else 1e-4
    for k in want:
        assert rel_err(_f64(got[k]), want[k]) <= bar, (k, rel_err(_f64(got[k]), want[k]))
    Y = want["y"]
    most = np.repeat(np.abs(Y.reshape(len(Y), -1, 32)).max(-1), 32, axis=-1)
    err = np.abs(kept - Y)
    assert (err <= np.maximum(2.0 ** -4 * np.abs(Y), 2.0 ** -17 * most) + 2e-2 * most * (dtype == "bf16") + 1e-5 * most).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_two_ranks_give_what_one_gives(dtype):
    """The same step on one rank and on two: the losses and gradients differ by roundings only."""
    torch = need_gpu()
    one, _, _ = _step(torch, dtype, 1)
    two, _, _ = _step(torch, dtype, 2)
    for k in one:
        tol = {"sum": 0, "y": 0, "loss": 1e-6}.get(k, 1e-2 if dtype == "bf16" else 1e-5)
        assert rel_err(_f64(two[k]), _f64(one[k])) <= tol, k


def _calls(torch, dtype, seed, rows=700, h=1920, V=5003, ranks=2):
    """A set of inputs, outputs and the calls of every entry point on them."""
    rng = torch.Generator(device="cuda").manual_seed(seed)
    dt = _type(torch, dtype)
    rand = lambda *s: torch.randn(*s, generator=rng, device="cuda").to(dt)  # noqa: E731
    new = lambda *s, dtype=dt: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
    f32, ld = torch.float32, -(-V // 8) * 8
    i = dict(x=rand(rows, h), r=rand(rows, h), g=rand(h), dy=rand(rows, h), ds=rand(rows, h), z=rand(rows, ld),
             t=rand(rows, 20), ids=torch.randint(0, V, (rows, 20), generator=rng, device="cuda"),
             lab=torch.randint(-1, V, (rows,), generator=rng, device="cuda"),
             w=torch.rand(rows, generator=rng, device="cuda"))
    o = dict(sum=new(rows, h), y=new(rows, h), q=new(rows, h, dtype=torch.uint8), sc=new(rows, h // 32, dtype=torch.uint8),
             dx=new(rows, h), dg=new(h, dtype=f32), loss=new(rows, dtype=f32), dz=new(rows, ld), stats=new(rows, 8, dtype=f32),
             loss2=new(rows, dtype=f32), dz2=new(rows, ld), joined=new(rows, 8, dtype=f32), loss3=new(rows, dtype=f32))
    scratch = new(B.add_rms_norm_scratch_elems(rows, h), dtype=f32)
    kw = dict(teacher_ids=i["ids"], teacher_logits=i["t"], labels=i["lab"], alpha=0.5, temperature=2.0)

    def run(stream=None):
        B.add_rms_norm_fwd(i["x"], i["g"], o["y"], resid=i["r"], sum=o["sum"], q=o["q"], scales=o["sc"], stream=stream)
        B.add_rms_norm_bwd(i["dy"], o["sum"], i["g"], o["dx"], o["dg"], scratch, dsum=i["ds"], stream=stream)
        B.distill_loss_fwd_bwd(i["z"], i["w"], o["loss"], o["dz"], vocab=V, stream=stream, **kw)
        B.distill_loss_fwd(i["z"], o["stats"], o["loss2"], vocab=V, stream=stream, **kw)
        B.distill_loss_join(o["stats"][None], o["joined"], o["loss3"], alpha=0.5, temperature=2.0, stream=stream)
        B.distill_loss_bwd(i["z"], o["joined"], i["w"], o["dz2"], vocab=V, stream=stream, **kw)

    return i, o, run


def _bits(o):
    import torch
    return {k: v.clone().view(torch.uint8) if v.dtype is torch.uint8 else v.clone().contiguous().view(torch.int16)
            for k, v in o.items()}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_captured_and_replayed(dtype):
    """Every call in one graph, replayed on new inputs between eager work: the same bits as eager calls.  Two graphs
    share the scratch, one behind the other."""
    torch = need_gpu()
    print(f"[head graph] {dtype}", flush=True)
    i, o, run = _calls(torch, dtype, 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        graphs.append(g)
    for turn in range(4):
        fresh, _, _ = _calls(torch, dtype, 10 + turn)
        for k in i:
            i[k].copy_(fresh[k])
        run()
        torch.cuda.synchronize()
        want = _bits(o)
        for v in o.values():
            v.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        got = _bits(o)
        for k in want:
            assert torch.equal(want[k], got[k]), (turn, k)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_streams_at_the_same_time(dtype):
    """Three sets of calls on three streams at once give what each gives alone."""
    torch = need_gpu()
    print(f"[head streams] {dtype}", flush=True)
    sets = [_calls(torch, dtype, s) for s in (1, 2, 3)]
    want = []
    for _, o, run in sets:
        run()
        torch.cuda.synchronize()
        want.append(_bits(o))
        for v in o.values():
            v.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        for (_, _, run), s in zip(sets, streams):
            run(stream=s)
    torch.cuda.synchronize()
    for (_, o, _), w in zip(sets, want):
        got = _bits(o)
        assert all(torch.equal(got[k], w[k]) for k in w)


def test_logits_beyond_32_bit_offsets():
    """87000 x 50304 logits (4.4e9 elements): the last tokens, and some in between, give the bits that they give in a
    call of their own."""
    torch = need_gpu()
    print("[head large] logits", flush=True)
    T, V, K = 87000, 50304, 16
    z = torch.empty(T, V, dtype=torch.bfloat16, device="cuda")
    for a in range(0, T, 10000):
        z[a:a + 10000].normal_(std=2.0)
    ids = torch.randint(0, V, (T, K), device="cuda", dtype=torch.int32)
    t, lab, w = torch.randn(T, K, device="cuda"), torch.randint(0, V, (T,), device="cuda"), torch.rand(T, device="cuda")
    loss, dz, loss2, stats = torch.empty(T, device="cuda"), torch.empty_like(z), torch.empty(T, device="cuda"), \
        torch.empty(T, 8, device="cuda")
    args = lambda s: dict(teacher_ids=ids[s].clone(), teacher_logits=t[s].clone(), labels=lab[s].clone(), alpha=0.5,
                           temperature=2.0)  # noqa: E731
    every = slice(0, T)
    B.distill_loss_fwd_bwd(z, w, loss, dz, **args(every))
    B.distill_loss_fwd(z, stats, loss2, **args(every))
    spots = [slice(T - 7, T), slice(42684, 42700), slice(85368, 85376), slice(0, 3)]  # 2^31 and 2^32 elements lie in the middle
    for s in spots:
        n = s.stop - s.start
        l, d, l2, st = torch.empty(n, device="cuda"), torch.empty(n, V, dtype=z.dtype, device="cuda"), \
            torch.empty(n, device="cuda"), torch.empty(n, 8, device="cuda")
        B.distill_loss_fwd_bwd(z[s], w[s].clone(), l, d, **args(s))
        assert torch.equal(l, loss[s]) and torch.equal(d, dz[s])
        B.distill_loss_fwd(z[s], st, l2, **args(s))
        assert torch.equal(l2, loss2[s]) and torch.equal(st, stats[s])
    kept = [dz[s].clone() for s in spots]
    B.distill_loss_bwd(z, stats, w, z, **args(every))  # over the logits
    for s, k in zip(spots, kept):
        # one bf16 step and fp32's roundings between the two calls
        assert bool(((z[s].float() - k.float()).abs() <= 2.0 ** -7 * k.float().abs() + 1e-6).all())
    torch.cuda.synchronize()


def test_norm_beyond_32_bit_offsets():
    torch = need_gpu()
    print("[head large] norm", flush=True)
    rows, cols = 540000, 8192
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    for a in range(0, rows, 60000):
        x[a:a + 60000].normal_()
    g = torch.randn(cols, device="cuda").bfloat16()
    s, y = torch.empty_like(x), torch.empty_like(x)
    q, sc = torch.empty(rows, cols, dtype=torch.uint8, device="cuda"), \
        torch.empty(rows, cols // 32, dtype=torch.uint8, device="cuda")
    B.add_rms_norm_fwd(x, g, y, resid=x, sum=s, q=q, scales=sc)
    spots = [slice(rows - 5, rows), slice(262140, 262148), slice(524284, 524292)]
    for p in spots:
        out = [torch.empty_like(v[p]) for v in (s, y, q, sc)]
        B.add_rms_norm_fwd(x[p], g, out[1], resid=x[p], sum=out[0], q=out[2], scales=out[3])
        assert all(torch.equal(a, b[p]) for a, b in zip(out, (s, y, q, sc)))
    dg, scratch = torch.empty(cols, device="cuda"), torch.empty(B.add_rms_norm_scratch_elems(rows, cols), device="cuda")
    B.add_rms_norm_bwd(y, s, g, x, dg, scratch, dsum=y)
    for p in spots:
        n = p.stop - p.start
        dx, d = torch.empty_like(x[p]), torch.empty(cols, device="cuda")
        B.add_rms_norm_bwd(y[p], s[p], g, dx, d, torch.empty(B.add_rms_norm_scratch_elems(n, cols), device="cuda"), dsum=y[p])
        assert torch.equal(dx, x[p])
    torch.cuda.synchronize()


def test_calls_of_several_launches():
    """More tokens and rows than the workgroups of one launch hold."""
    torch = need_gpu()
    print("[head launches]", flush=True)
    T = 2 ** 26 + 5
    z = torch.randn(T, 8, device="cuda").bfloat16()
    lab, w = torch.randint(0, 3, (T,), device="cuda", dtype=torch.int32), torch.ones(T, device="cuda")
    loss, dz = torch.empty(T, device="cuda"), torch.empty_like(z)
    B.distill_loss_fwd_bwd(z, w, loss, dz, labels=lab, alpha=0.0, vocab=3)
    d = z[:, :3].float()
    lse = torch.logsumexp(d, 1)
    want = lse - d.gather(1, lab.long()[:, None])[:, 0]
    assert bool(((loss - want).abs() <= 64 * 2.0 ** -24 * (1 + lse.abs() + d.abs().amax(1))).all())
    p = torch.softmax(d, 1)
    p.scatter_add_(1, lab.long()[:, None], torch.full((T, 1), -1.0, device="cuda"))
    assert bool(((dz[:, :3].float() - p).abs() <= 2.0 ** -8 * p.abs() + 1e-6).all()) and not dz[:, 3:].any()
    stats, loss2 = torch.empty(T, 8, device="cuda"), torch.empty(T, device="cuda")
    B.distill_loss_fwd(z, stats, loss2, labels=lab, alpha=0.0, vocab=3)
    assert bool(((loss2 - want).abs() <= 64 * 2.0 ** -24 * (1 + lse.abs() + d.abs().amax(1))).all())
    dz2 = torch.empty_like(z)
    B.distill_loss_bwd(z, stats, w, dz2, labels=lab, alpha=0.0, vocab=3)
    assert bool(((dz2[:, :3].float() - p).abs() <= 2.0 ** -8 * p.abs() + 1e-6).all()) and not dz2[:, 3:].any()
    g = torch.ones(8, device="cuda").bfloat16()
    y = torch.empty_like(z)
    B.add_rms_norm_fwd(z, g, y, eps=1e-6)
    f = z.float()
    ref = f * torch.rsqrt(f.square().mean(1, keepdim=True) + 1e-6)
    assert bool(((y.float() - ref).abs() <= (2.0 ** -8 + 2.0 ** -18) * ref.abs() + 1e-30).all())
    torch.cuda.synchronize()
