"""Refusals of the residual norm and the distillation loss, before anything is enqueued (no GPU):
the entry points' statuses, the binding's checks, and sizes at and beyond the limits."""
import pytest

from paper_2206_04959_amd import binding as B

torch = pytest.importorskip("torch")

P = [0x10000000 * (i + 1) for i in range(12)]  # addresses far apart; nothing reads them
INVALID, SHAPE, ALIGN, HIP, UNSUPPORTED = -1, -2, -4, -6, -7
NAN, INF = float("nan"), float("inf")


def _status(fn, args, change):
    return getattr(B.lib(), fn)(*{**args, **change}.values())


def _fwd(**c):
    return _status("merak_add_rms_norm_fwd", dict(dtype=0, rows=4, cols=64, eps=1e-6, x=P[0], resid=P[1], gamma=P[2],
                                                  sum=P[3], y=P[4], q=P[5], scales=P[6], stream=None), c)


def _bwd(**c):
    return _status("merak_add_rms_norm_bwd", dict(dtype=0, rows=40, cols=64, eps=1e-6, dy=P[0], dsum=P[1], sum=P[2],
                                                  gamma=P[3], dx=P[4], dgamma=P[5], accumulate=0, scratch=P[6],
                                                  stream=None), c)


_SHAPE = dict(dtype=0, tokens=4, vocab=100, ld=104)
_SHARE = dict(first=0, total=100)
_MIX = dict(top=5, id_type=1, teacher=0, label_type=1, alpha=0.5, tau=2.0)
_IN = dict(logits=P[0], ids=P[1], t=P[2], labels=P[3])


def _loss(**c):
    return _status("merak_distill_loss_fwd", dict(**_SHAPE, **_SHARE, **_MIX, **_IN, stats=P[4], loss=P[5], stream=None), c)


def _grad(**c):
    return _status("merak_distill_loss_bwd", dict(**_SHAPE, **_SHARE, **_MIX, **_IN, stats=P[4], dloss=P[5], dz=P[6],
                                                  stream=None), c)


def _both(**c):
    return _status("merak_distill_loss_fwd_bwd", dict(**_SHAPE, **_MIX, **_IN, dloss=P[4], loss=P[5], dz=P[6],
                                                      stream=None), c)


def _join(**c):
    return _status("merak_distill_loss_join", dict(tokens=4, ranks=2, alpha=0.5, tau=2.0, parts=P[0], stats=P[1],
                                                   loss=P[2], stream=None), c)


@pytest.mark.parametrize("call,change,status", [
    *[(f, c, s) for f in (_fwd, _bwd) for c, s in (
        (dict(dtype=2), INVALID), (dict(rows=0), SHAPE), (dict(rows=-1), SHAPE), (dict(rows=2 ** 30 + 1), SHAPE),
        (dict(cols=0), SHAPE), (dict(cols=60), SHAPE), (dict(cols=16392), UNSUPPORTED), (dict(eps=0.0), SHAPE),
        (dict(eps=NAN), SHAPE), (dict(eps=INF), SHAPE), (dict(gamma=None), INVALID), (dict(gamma=P[3] + 8), ALIGN),
        (dict(sum=P[2] + 4), ALIGN))],
    (_fwd, dict(x=None), INVALID), (_fwd, dict(x=P[0] + 2), ALIGN), (_fwd, dict(resid=P[1] + 8), ALIGN),
    (_fwd, dict(resid=None), INVALID),             # a sum without a residual
    (_fwd, dict(y=None, q=None, scales=None), INVALID), (_fwd, dict(q=None), INVALID), (_fwd, dict(scales=None), INVALID),
    (_fwd, dict(cols=72), SHAPE),                  # whole blocks of 32 for 8 bits
    (_fwd, dict(y=P[0]), INVALID), (_fwd, dict(y=P[1] + 16), INVALID), (_fwd, dict(y=P[3]), INVALID),
    (_fwd, dict(sum=P[0] + 16), INVALID), (_fwd, dict(sum=P[2]), INVALID), (_fwd, dict(q=P[4]), INVALID),
    (_fwd, dict(scales=P[5] + 16), INVALID), (_fwd, dict(y=P[4] + 4), ALIGN), (_fwd, dict(q=P[5] + 8), ALIGN),
    (_bwd, dict(dy=None), INVALID), (_bwd, dict(sum=None), INVALID), (_bwd, dict(dx=None), INVALID),
    (_bwd, dict(dgamma=None), INVALID), (_bwd, dict(accumulate=2), INVALID), (_bwd, dict(scratch=None), INVALID),
    (_bwd, dict(scratch=P[6] + 8), ALIGN), (_bwd, dict(dsum=P[1] + 2), ALIGN), (_bwd, dict(dx=P[2]), INVALID),
    (_bwd, dict(dx=P[0] + 16), INVALID), (_bwd, dict(dx=P[1] + 16), INVALID), (_bwd, dict(dgamma=P[3]), INVALID),
    (_bwd, dict(scratch=P[4]), INVALID), (_bwd, dict(scratch=P[5]), INVALID),
    *[(f, c, s) for f in (_loss, _grad, _both) for c, s in (
        (dict(dtype=-1), INVALID), (dict(tokens=0), SHAPE), (dict(tokens=2 ** 30 + 1), SHAPE), (dict(vocab=0), SHAPE),
        (dict(ld=96), SHAPE), (dict(ld=108), SHAPE), (dict(ld=2 ** 28 + 8), SHAPE), (dict(top=-1), SHAPE),
        (dict(top=1025), SHAPE), (dict(id_type=2), INVALID), (dict(teacher=2), INVALID), (dict(label_type=-1), INVALID),
        (dict(alpha=-0.1), INVALID), (dict(alpha=1.1), INVALID), (dict(alpha=NAN), INVALID), (dict(tau=0.0), INVALID),
        (dict(tau=-1.0), INVALID), (dict(tau=INF), INVALID), (dict(tau=NAN), INVALID), (dict(tau=2.0 ** -11), INVALID),
        (dict(tau=2.0 ** 11), INVALID), (dict(logits=None), INVALID), (dict(logits=P[0] + 2), ALIGN),
        (dict(ids=None), INVALID), (dict(t=None), INVALID), (dict(ids=P[1] + 8), ALIGN), (dict(t=P[2] + 2), ALIGN),
        (dict(labels=P[3] + 4), ALIGN), (dict(top=0, labels=None), INVALID), (dict(alpha=0.0, labels=None), INVALID),
        (dict(top=0, alpha=1.0), INVALID))],
    *[(f, c, s) for f in (_loss, _grad) for c, s in (
        (dict(first=-1), INVALID), (dict(first=1), INVALID), (dict(total=99), INVALID), (dict(stats=P[4] + 8), ALIGN))],
    (_loss, dict(stats=None, loss=None), INVALID), (_loss, dict(total=200), INVALID),   # a share's loss
    (_loss, dict(loss=P[4]), INVALID), (_loss, dict(stats=P[0]), INVALID), (_loss, dict(loss=P[3]), INVALID),
    (_loss, dict(stats=P[1] + 16), INVALID), (_loss, dict(loss=P[5] + 4), ALIGN),
    (_grad, dict(stats=None), INVALID), (_grad, dict(dloss=None), INVALID), (_grad, dict(dz=None), INVALID),
    (_grad, dict(dz=P[0] + 16), INVALID), (_grad, dict(dz=P[4]), INVALID), (_grad, dict(dz=P[2]), INVALID),
    (_grad, dict(dz=P[5]), INVALID), (_grad, dict(dz=P[6] + 4), ALIGN),
    (_both, dict(dloss=None), INVALID), (_both, dict(loss=None), INVALID), (_both, dict(loss=P[4]), INVALID),
    (_both, dict(dz=P[0] + 16), INVALID), (_both, dict(loss=P[6] + 16), INVALID), (_both, dict(dz=None), INVALID),
    *[(_join, c, s) for c, s in (
        (dict(tokens=0), SHAPE), (dict(ranks=0), SHAPE), (dict(ranks=2 ** 16 + 1), SHAPE), (dict(alpha=2.0), INVALID),
        (dict(tau=0.0), INVALID), (dict(parts=None), INVALID), (dict(stats=None), INVALID), (dict(loss=None), INVALID),
        (dict(stats=P[0] + 128), INVALID), (dict(loss=P[1] + 16), INVALID), (dict(parts=P[0] + 4), ALIGN))],
])
def test_entry_points_refuse(call, change, status):
    assert call(**change) == status


def test_scratch_sizes():
    assert B.add_rms_norm_scratch_elems(0, 64) == 0 and B.add_rms_norm_scratch_elems(-3, 64) == 0
    assert B.add_rms_norm_scratch_elems(1, 1600) == 0      # one launch
    sizes = [B.add_rms_norm_scratch_elems(r, 1600) for r in (10, 100, 1000, 10 ** 5, 10 ** 9)]
    assert all(0 < a <= b for a, b in zip(sizes, sizes[1:])) and sizes[-1] == sizes[-2]
    L = B.lib()
    assert L.merak_add_rms_norm_bwd(0, 1, 64, 1e-6, P[0], None, P[1], P[2], P[3] + 4, P[4], 0, None, None) == ALIGN


FAR = [(i + 1) << 44 for i in range(8)]  # addresses that no array of these sizes connects


@pytest.mark.skipif(torch.cuda.is_available(), reason="the allowed sizes would be launched")
def test_largest_sizes_reach_the_launch():
    """The largest rows, widths and entries that the header allows get as far as the launch (which
    fails here, without a GPU)."""
    L = B.lib()
    assert L.merak_add_rms_norm_fwd(0, 2 ** 30, 8, 1e-6, FAR[0], FAR[1], FAR[2], FAR[3], FAR[4], None, None, None) == HIP
    assert L.merak_add_rms_norm_fwd(0, 2 ** 26, 16384, 1e-6, FAR[0], None, FAR[2], None, None, FAR[4], FAR[5], None) == HIP
    assert L.merak_add_rms_norm_bwd(1, 2 ** 26, 16384, 1e-6, FAR[0], FAR[1], FAR[2], FAR[3], FAR[4], FAR[5], 1, FAR[6],
                                    None) == HIP
    for fn, tail in (("fwd", (FAR[4], FAR[5])), ("bwd", (FAR[4], FAR[5], FAR[6]))):
        call = getattr(L, "merak_distill_loss_" + fn)
        assert call(0, 2 ** 30, 1, 8, 0, 1, 1024, 1, 1, 1, 0.5, 2.0, FAR[0], FAR[1], FAR[2], FAR[3], *tail, None) == HIP
        assert call(1, 1000, 2 ** 28, 2 ** 28, 0, 2 ** 28, 1, 1, 1, 1, 0.5, 2.0, FAR[0], FAR[1], FAR[2], FAR[3], *tail,
                    None) == HIP
    # the last columns of the largest vocabulary
    assert L.merak_distill_loss_fwd(0, 1, 8, 8, 2 ** 63 - 9, 2 ** 63 - 1, 1, 1, 1, 1, 0.5, 2.0, FAR[0], FAR[1], FAR[2],
                                    FAR[3], FAR[4], None, None) == HIP
    assert L.merak_distill_loss_fwd(0, 1, 8, 8, 2 ** 63 - 8, 2 ** 63 - 1, 1, 1, 1, 1, 0.5, 2.0, FAR[0], FAR[1], FAR[2],
                                    FAR[3], FAR[4], None, None) == INVALID


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls would be launched")
@pytest.mark.parametrize("call", [_loss, _grad, _both])
def test_arrays_of_a_term_without_weight_are_not_looked_at(call):
    """With alpha = 0 the teacher's arrays and their types, with alpha = 1 the labels, may be anything
    (the calls get as far as the launch, which fails here, without a GPU); `top` keeps its limits."""
    for change in (dict(ids=None, t=None), dict(ids=None), dict(t=None), dict(ids=P[1] + 8, t=P[2] + 2),
                   dict(id_type=7, teacher=7), dict(ids=P[0], t=P[0]), dict(ids=P[6], t=P[5]), dict(top=0)):
        assert call(alpha=0.0, **change) == HIP, change
    for change in (dict(labels=None), dict(labels=P[3] + 4), dict(label_type=7), dict(labels=P[5]), dict(labels=P[0])):
        assert call(alpha=1.0, **change) == HIP, change
    assert call(alpha=0.0, top=1025) == SHAPE and call(alpha=0.0, top=-1) == SHAPE
    assert call(alpha=1.0, ids=None) == INVALID and call(alpha=0.0, label_type=7) == INVALID
    assert call(alpha=2.0 ** -30, ids=None, t=None) == INVALID and call(alpha=1.0 - 2.0 ** -24, label_type=7) == INVALID


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


U8, F32, I32, I64 = torch.uint8, torch.float32, torch.int32, torch.int64
WRAP = 2 ** 32 + 64  # 64 in 32 bits


def _v(*shape, dtype=torch.bfloat16):
    """A tensor of any shape without memory behind it."""
    return torch.empty(shape, dtype=dtype, device="meta")


@pytest.mark.parametrize("call", [
    lambda: B.add_rms_norm_fwd(_t(4, 64), _t(64, dtype=F32), _t(4, 64)),
    lambda: B.add_rms_norm_fwd(_t(4, 64, dtype=torch.float16), _t(64, dtype=torch.float16), _t(4, 64, dtype=torch.float16)),
    lambda: B.add_rms_norm_fwd(_t(4, 64), _t(32), _t(4, 64)),
    lambda: B.add_rms_norm_fwd(_t(4, 64), _t(64), _t(5, 64)),
    lambda: B.add_rms_norm_fwd(_t(4, 64), _t(64), _t(8, 32)),
    lambda: B.add_rms_norm_fwd(_t(4, 64), _t(64), _t(4, 64, dtype=F32)),
    lambda: B.add_rms_norm_fwd(_t(4, 64), _t(64), _t(4, 64), resid=_t(4, 32)),
    lambda: B.add_rms_norm_fwd(_t(4, 64), _t(64), _t(4, 64), sum=_t(4, 64)),
    lambda: B.add_rms_norm_fwd(_t(4, 64), _t(64)),
    lambda: B.add_rms_norm_fwd(_t(4, 64), _t(64), q=_t(4, 64, dtype=U8)),
    lambda: B.add_rms_norm_fwd(_t(4, 64), _t(64), q=_t(5, 64, dtype=U8), scales=_t(5, 2, dtype=U8)),
    lambda: B.add_rms_norm_fwd(_t(4, 40), _t(40), q=_t(4, 40, dtype=U8), scales=_t(4, 1, dtype=U8)),
    lambda: B.add_rms_norm_fwd(_t(64, 4).t(), _t(64), _t(4, 64)),
    lambda: B.add_rms_norm_fwd(_t(4, 64), _t(64), _t(4, 64)),                       # not on a GPU
    lambda: B.add_rms_norm_bwd(_t(4, 64), _t(4, 64), _t(64), _t(4, 64), _t(64)),
    lambda: B.add_rms_norm_bwd(_t(4, 64), _t(4, 64), _t(64), _t(4, 64), _t(32, dtype=F32)),
    lambda: B.add_rms_norm_bwd(_t(5, 64), _t(4, 64), _t(64), _t(4, 64), _t(64, dtype=F32)),
    lambda: B.add_rms_norm_bwd(_t(40, 64), _t(40, 64), _t(64), _t(40, 64), _t(64, dtype=F32)),
    lambda: B.distill_loss_fwd(_t(4, 104), loss=_t(4)),
    lambda: B.distill_loss_fwd(_t(4, 104), loss=_t(5, dtype=F32), labels=_t(4, dtype=I64)),
    lambda: B.distill_loss_fwd(_t(4, 104), stats=_t(4, 6, dtype=F32), labels=_t(4, dtype=I64)),
    lambda: B.distill_loss_fwd(_t(4, 104), stats=_t(8, 4, dtype=F32), labels=_t(4, dtype=I64)),
    lambda: B.distill_loss_fwd(_t(4, 104), labels=_t(4, dtype=I64)),
    lambda: B.distill_loss_fwd(_t(4, 104), loss=_t(4, dtype=F32), labels=_t(4, dtype=I64), vocab=105),
    lambda: B.distill_loss_fwd(_t(4, 104), loss=_t(4, dtype=F32), labels=_t(4, dtype=I64), vocab=50, vocab_total=100),
    lambda: B.distill_loss_fwd(_t(4, 104), loss=_t(4, dtype=F32), labels=_t(5, dtype=I64)),
    lambda: B.distill_loss_fwd(_t(4, 104), loss=_t(4, dtype=F32), labels=_t(4, dtype=torch.int16)),
    lambda: B.distill_loss_fwd(_t(4, 104), loss=_t(4, dtype=F32), teacher_ids=_t(4, 5, dtype=I64)),
    lambda: B.distill_loss_fwd(_t(4, 104), loss=_t(4, dtype=F32), teacher_logits=_t(4, 5)),
    lambda: B.distill_loss_fwd(_t(4, 104), loss=_t(4, dtype=F32), teacher_ids=_t(4, 5, dtype=I64), teacher_logits=_t(4, 6)),
    lambda: B.distill_loss_fwd(_t(4, 104), loss=_t(4, dtype=F32), teacher_ids=_t(4, 5, dtype=I64), teacher_logits=_t(5, 4)),
    lambda: B.distill_loss_fwd(_t(4, 104), loss=_t(4, dtype=F32), teacher_ids=_t(3, 5, dtype=I64), teacher_logits=_t(3, 5)),
    lambda: B.distill_loss_fwd(_t(4, 104), loss=_t(4, dtype=F32), teacher_ids=_t(4, 5, dtype=I64),
                               teacher_logits=_t(4, 5, dtype=torch.float16)),
    lambda: B.distill_loss_join(_t(2, 4, 8, dtype=F32), _t(4, 8, dtype=F32), _t(5, dtype=F32)),
    lambda: B.distill_loss_join(_t(2, 4, 6, dtype=F32), _t(4, 8, dtype=F32), _t(4, dtype=F32)),
    lambda: B.distill_loss_join(_t(2, 4, 8), _t(4, 8, dtype=F32), _t(4, dtype=F32)),
    lambda: B.distill_loss_bwd(_t(4, 104), _t(4, 8, dtype=F32), _t(4, dtype=F32), _t(4, 96), labels=_t(4, dtype=I64)),
    lambda: B.distill_loss_bwd(_t(4, 104), _t(4, 8, dtype=F32), _t(4), _t(4, 104), labels=_t(4, dtype=I64)),
    lambda: B.distill_loss_fwd_bwd(_t(4, 104), _t(4, dtype=F32), _t(4, dtype=F32), _t(4, 104, dtype=F32),
                                   labels=_t(4, dtype=I64)),
    lambda: B.distill_loss_fwd_bwd(_t(4, 104), _t(4, dtype=F32), _t(4, dtype=F32), _t(4, 104), labels=_t(4, dtype=I64)),
])
def test_binding_refuses(call):
    with pytest.raises(ValueError):
        call()


@pytest.mark.parametrize("call", [
    lambda: B.add_rms_norm_fwd(_v(WRAP, 64), _v(64), _v(WRAP, 64)),
    lambda: B.add_rms_norm_fwd(_v(1, WRAP), _v(WRAP), _v(1, WRAP)),
    lambda: B.add_rms_norm_bwd(_v(WRAP, 64), _v(WRAP, 64), _v(64), _v(WRAP, 64), _v(64, dtype=F32)),
    lambda: B.add_rms_norm_scratch_elems(WRAP, 64),
    lambda: B.add_rms_norm_scratch_elems(64, -WRAP),
    lambda: B.distill_loss_fwd(_v(WRAP, 64), loss=_v(WRAP, dtype=F32), labels=_v(WRAP, dtype=I64)),
    lambda: B.distill_loss_fwd(_v(1, WRAP), loss=_v(1, dtype=F32), labels=_v(1, dtype=I64)),
    lambda: B.distill_loss_fwd(_v(1, 64), loss=_v(1, dtype=F32), teacher_ids=_v(1, WRAP, dtype=I64),
                               teacher_logits=_v(1, WRAP)),
    lambda: B.distill_loss_fwd(_v(1, 64), stats=_v(1, 8, dtype=F32), labels=_v(1, dtype=I64), first_id=2 ** 64 + 1,
                               vocab_total=100),
    lambda: B.distill_loss_fwd(_v(1, 64), stats=_v(1, 8, dtype=F32), labels=_v(1, dtype=I64), vocab_total=2 ** 64 + 100),
    lambda: B.distill_loss_join(_v(2, WRAP, 8, dtype=F32), _v(WRAP, 8, dtype=F32), _v(WRAP, dtype=F32)),
    lambda: B.distill_loss_join(_v(WRAP, 1, 8, dtype=F32), _v(1, 8, dtype=F32), _v(1, dtype=F32)),
])
def test_binding_refuses_sizes_that_ctypes_would_cut(call):
    with pytest.raises(ValueError, match="too large"):
        call()
