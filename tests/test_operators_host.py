"""Refusals of the operators around the blocks, before anything is enqueued (no GPU): the
C entry points' statuses and the binding's argument checks."""
import ctypes

import pytest

from paper_2206_04959_amd import binding as B

torch = pytest.importorskip("torch")

P = [0x1000000 * (i + 1) for i in range(12)]  # addresses far apart; nothing reads them
OK = object()


def _status(fn, args, **change):
    return getattr(B.lib(), fn)(*{**args, **change}.values())


def _embed_fwd(**c):
    return _status("merak_embedding_fwd", dict(dtype=0, id_type=1, tokens=10, hidden=64, rows=100, first=0, scale=1.0,
                                               ids=P[0], table=P[1], y=P[2], stream=None), **c)


def _embed_bwd(**c):
    return _status("merak_embedding_bwd", dict(dtype=0, id_type=1, tokens=5000, hidden=64, rows=100, first=0, scale=1.0,
                                               ids=P[0], dy=P[1], dtable=P[2], accumulate=0, scratch=P[3],
                                               stream=None), **c)


_QK = dict(dtype=0, tokens=10, q_heads=4, kv_heads=2, d=64, rope=64, inter=0, eps=1e-6)
_TAIL = dict(table=P[6], table_rows=50, positions=None, seq_len=10)


def _qk_fwd(**c):
    return _status("merak_qk_norm_rope_fwd", dict(**_QK, qkv=P[0], gq=P[1], gk=P[2], **_TAIL, out=P[3], stream=None), **c)


def _qk_bwd(**c):
    return _status("merak_qk_norm_rope_bwd",
                   dict(**_QK, dout=P[4], qkv=P[0], gq=P[1], gk=P[2], **_TAIL, dqkv=P[3], dgq=P[5], dgk=P[7],
                        accumulate=0, scratch=P[8], stream=None), **c)


def _save(**c):
    return _status("merak_act8_save", dict(dtype=0, rows=4, cols=64, x=P[0], q=P[1], scales=P[2], stream=None), **c)


def _restore(**c):
    return _status("merak_act8_restore", dict(dtype=0, rows=4, cols=64, q=P[1], scales=P[2], x=P[0], stream=None), **c)


def _gelu(**c):
    return _status("merak_act8_gelu_bwd", dict(dtype=0, rows=4, cols=64, dg=P[0], q=P[1], scales=P[2], du=P[3],
                                               g=P[4], stream=None), **c)


def _dw(**c):
    return _status("merak_act8_gemm_dw", dict(dtype=0, tokens=4, n_out=64, n_in=64, dy=P[0], q=P[1], scales=P[2],
                                              dw=P[3], accumulate=0, scratch=P[4], stream=None), **c)


INVALID, SHAPE, ALIGN, UNSUPPORTED = -1, -2, -4, -7
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("call,change,status", [
    *[(f, c, s) for f in (_embed_fwd, _embed_bwd) for c, s in (
        (dict(dtype=2), INVALID), (dict(id_type=2), INVALID), (dict(tokens=0), SHAPE), (dict(tokens=-1), SHAPE),
        (dict(tokens=2 ** 30 + 1), SHAPE), (dict(hidden=0), SHAPE), (dict(hidden=12), SHAPE), (dict(rows=0), SHAPE),
        (dict(hidden=2 ** 20 + 8), SHAPE), (dict(first=-1), INVALID), (dict(scale=NAN), INVALID),
        (dict(scale=INF), INVALID), (dict(ids=None), INVALID), (dict(ids=P[0] + 4), ALIGN))],
    (_embed_fwd, dict(table=None), INVALID), (_embed_fwd, dict(y=P[2] + 2), ALIGN),
    (_embed_fwd, dict(y=P[1]), INVALID), (_embed_fwd, dict(y=P[1] + 100 * 128 - 16), INVALID),
    (_embed_bwd, dict(accumulate=2), INVALID), (_embed_bwd, dict(scratch=None), INVALID),
    (_embed_bwd, dict(tokens=2 ** 22 + 1), SHAPE),
    (_embed_bwd, dict(scratch=P[3] + 8), ALIGN), (_embed_bwd, dict(dtable=P[1]), INVALID),
    (_embed_bwd, dict(scratch=P[2] + 16), INVALID),
    *[(f, c, s) for f in (_qk_fwd, _qk_bwd) for c, s in (
        (dict(dtype=-1), INVALID), (dict(tokens=0), SHAPE), (dict(q_heads=0), SHAPE), (dict(kv_heads=0), SHAPE),
        (dict(q_heads=5000), SHAPE), (dict(d=0), SHAPE), (dict(d=60, rope=0), SHAPE), (dict(d=264), UNSUPPORTED),
        (dict(rope=24), SHAPE), (dict(rope=80), SHAPE), (dict(rope=-16), SHAPE), (dict(inter=2), INVALID),
        (dict(eps=0.0), SHAPE), (dict(eps=NAN), SHAPE), (dict(table=None), INVALID), (dict(table_rows=0), SHAPE),
        (dict(seq_len=0), SHAPE), (dict(seq_len=51), SHAPE), (dict(positions=P[9] + 4), ALIGN), (dict(gq=None), INVALID),
        (dict(qkv=None), INVALID), (dict(gk=P[2] + 8), ALIGN))],
    (_qk_fwd, dict(out=P[0] + 64), INVALID), (_qk_fwd, dict(out=P[6]), INVALID),
    (_qk_bwd, dict(dqkv=P[0]), INVALID), (_qk_bwd, dict(dqkv=P[4] + 64), INVALID), (_qk_bwd, dict(dgk=P[5]), INVALID),
    (_qk_bwd, dict(scratch=None), INVALID), (_qk_bwd, dict(accumulate=-1), INVALID),
    (_qk_bwd, dict(scratch=P[4]), INVALID),
    *[(f, c, s) for f in (_save, _restore, _gelu) for c, s in (
        (dict(dtype=3), INVALID), (dict(rows=0), SHAPE), (dict(cols=0), SHAPE), (dict(cols=48), SHAPE),
        (dict(q=None), INVALID), (dict(scales=None), INVALID), (dict(q=P[1] + 8), ALIGN))],
    (_save, dict(x=None), INVALID), (_save, dict(x=P[1]), INVALID), (_restore, dict(x=P[2]), INVALID),
    (_gelu, dict(g=P[3]), INVALID), (_gelu, dict(g=P[0]), INVALID), (_gelu, dict(du=P[0] + 16), INVALID),
    (_gelu, dict(du=None), INVALID),
    *[(_dw, c, s) for c, s in (
        (dict(dtype=2), INVALID), (dict(tokens=0), SHAPE), (dict(n_out=0), SHAPE), (dict(n_out=12), SHAPE),
        (dict(n_in=40), SHAPE), (dict(dw=P[0]), INVALID), (dict(dy=None), INVALID), (dict(accumulate=3), INVALID),
        (dict(dw=P[3] + 4), ALIGN))],
])
def test_entry_points_refuse(call, change, status):
    assert call(**change) == status


@pytest.mark.parametrize("args,status", [
    ((0, 64, 1e4, P[0]), SHAPE), ((10, 24, 1e4, P[0]), SHAPE), ((10, 0, 1e4, P[0]), SHAPE), ((10, 272, 1e4, P[0]), SHAPE),
    ((10, 64, 0.0, P[0]), INVALID), ((10, 64, NAN, P[0]), INVALID), ((10, 64, 1e4, None), INVALID),
    ((10, 64, 1e4, P[0] + 8), ALIGN)])
def test_rope_table_refuses(args, status):
    p, r, theta, t = args
    assert B.lib().merak_rope_table(p, r, ctypes.c_double(theta), t, None) == status


def test_scratch_sizes():
    assert B.embedding_scratch_bytes(1, 1600) == 0 and B.embedding_scratch_bytes(0, 64) == 0
    assert B.embedding_scratch_bytes(-1, 64) == 0
    sizes = [B.embedding_scratch_bytes(t, 64) for t in (100, 1000, 10000, 100000, 10 ** 6)]
    assert all(0 <= a <= b for a, b in zip(sizes, sizes[1:])) and sizes[2] > 0
    assert B.qk_norm_rope_scratch_elems(0, 1, 1, 64) == 0 and B.qk_norm_rope_scratch_elems(10, 4, 2, 64) > 0
    assert B.act8_gemm_dw_scratch_bytes(torch.bfloat16, 0, 64, 64) == 0


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


U8, F32, I32 = torch.uint8, torch.float32, torch.int32


@pytest.mark.parametrize("call", [
    # element types
    lambda: B.embedding_fwd(_t(4, dtype=torch.int64), _t(9, 64), _t(4, 64, dtype=F32)),
    lambda: B.embedding_fwd(_t(4, dtype=torch.int16), _t(9, 64), _t(4, 64)),
    lambda: B.embedding_fwd(_t(4, dtype=torch.int64), _t(9, 64, dtype=torch.float16), _t(4, 64, dtype=torch.float16)),
    lambda: B.embedding_bwd(_t(4, dtype=I32), _t(4, 64), _t(9, 64)),
    lambda: B.act8_save(_t(4, 64), _t(4, 64, dtype=torch.int8), _t(4, 2, dtype=U8)),
    lambda: B.act8_gemm_dw(_t(4, 8), _t(4, 64, dtype=U8), _t(4, 2, dtype=U8), _t(8, 64)),
    lambda: B.rope_table(_t(10, 32, 2)),
    # sizes
    lambda: B.embedding_fwd(_t(4, dtype=I32), _t(9, 64), _t(5, 64)),
    lambda: B.embedding_bwd(_t(4, dtype=I32), _t(4, 32), _t(9, 64, dtype=F32)),
    lambda: B.qk_norm_rope_fwd(_t(4, 5, 64), _t(64), _t(64), None, _t(4, 5, 64), 2, 2),
    lambda: B.qk_norm_rope_fwd(_t(4, 6, 64), _t(64), _t(32), None, _t(4, 6, 64), 2, 2),
    lambda: B.qk_norm_rope_fwd(_t(4, 6, 64), _t(64), _t(64), _t(9, 32, 2, dtype=F32), _t(4, 6, 64), 2, 2),
    lambda: B.qk_norm_rope_fwd(_t(4, 6, 64), _t(64), _t(64), _t(9, 32, 2, dtype=F32), _t(4, 6, 64), 2, 2,
                               positions=_t(3, dtype=I32)),
    lambda: B.qk_norm_rope_fwd(_t(4, 6, 64), _t(64), _t(64), None, _t(4, 4, 64), 2, 2),
    lambda: B.qk_norm_rope_bwd(_t(4, 6, 64), _t(4, 6, 64), _t(64), _t(64), None, _t(4, 6, 64), _t(64, dtype=F32),
                               _t(64, dtype=F32), _t(3, dtype=F32), 2, 2),
    lambda: B.act8_save(_t(4, 48), _t(4, 48, dtype=U8), _t(4, 1, dtype=U8)),
    lambda: B.act8_save(_t(4, 64), _t(4, 64, dtype=U8), _t(4, 1, dtype=U8)),
    lambda: B.act8_restore(_t(4, 64, dtype=U8), _t(2, 4, dtype=U8), _t(4, 64)),
    lambda: B.act8_gelu_bwd(_t(4, 64), _t(4, 64, dtype=U8), _t(4, 2, dtype=U8), _t(4, 64), _t(4, 32)),
    lambda: B.act8_gemm_dw(_t(5, 8), _t(4, 64, dtype=U8), _t(4, 2, dtype=U8), _t(8, 64, dtype=F32)),
    # layout
    lambda: B.embedding_fwd(_t(8, dtype=I32)[::2], _t(9, 64), _t(4, 64)),
    lambda: B.act8_save(_t(64, 4).t(), _t(4, 64, dtype=U8), _t(4, 2, dtype=U8)),
    # not on a GPU
    lambda: B.embedding_fwd(_t(4, dtype=I32), _t(9, 64), _t(4, 64)),
    lambda: B.act8_restore(_t(4, 64, dtype=U8), _t(4, 2, dtype=U8), _t(4, 64)),
])
def test_binding_refuses(call):
    with pytest.raises(ValueError):
        call()
