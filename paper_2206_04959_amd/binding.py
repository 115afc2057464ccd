"""ctypes binding of libmerak_stage.so (argument marshalling only).

Every step of the forward, recompute and backward passes runs in the HIP
library; this module only converts Python arguments to the C ABI of
``include/merak_stage.h``.  PyTorch supplies device memory and streams.
If the library is missing the calls raise: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Dict, List, Optional, Sequence

import numpy as np

from . import synth

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmerak_stage.so")
PARAMS_PER_BLOCK = 12
BF16, FP32 = 0, 1

STATUS = {0: "MERAK_OK", -1: "MERAK_ERR_INVALID_ARG", -2: "MERAK_ERR_SHAPE", -3: "MERAK_ERR_ORDER",
          -4: "MERAK_ERR_ALIGN", -5: "MERAK_ERR_WORKSPACE", -6: "MERAK_ERR_HIP", -7: "MERAK_ERR_UNSUPPORTED"}

EPI_STORE, EPI_BIAS, EPI_BIAS_GELU, EPI_BIAS_RESID, EPI_GELU_BWD, EPI_F32 = range(6)
(KC_NONE, KC_GEMM_FWD, KC_GEMM_DX, KC_GEMM_DW, KC_ATTN_FWD, KC_ATTN_BWD, KC_LN_FWD, KC_LN_BWD,
 KC_REDUCE, KC_GEMM_DW_ATTN) = range(10)


class MerakError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {STATUS.get(status, status)}")
        self.status = status


class StageConfig(ctypes.Structure):
    _fields_ = [("n_blocks", ctypes.c_int32), ("hidden", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("ffn", ctypes.c_int32), ("seq_len", ctypes.c_int32), ("micro_batch", ctypes.c_int32),
                ("tp_degree", ctypes.c_int32), ("n_sub_microbatches", ctypes.c_int32),
                ("recompute_mask", ctypes.c_uint64), ("dtype", ctypes.c_int32), ("ln_eps", ctypes.c_float)]


_lib = None
_P, _I, _SZ, _F = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_float
_L = ctypes.c_int64
_SIGS = {
    "merak_status_str": ([_I], ctypes.c_char_p),
    "merak_stage_validate": ([ctypes.POINTER(StageConfig)], _I),
    "merak_stage_param_layout": ([ctypes.POINTER(StageConfig), ctypes.POINTER(_SZ), _P], _I),
    "merak_stage_workspace_bytes": ([ctypes.POINTER(StageConfig), ctypes.POINTER(_SZ), ctypes.POINTER(_SZ)], _I),
    "merak_stage_create": ([ctypes.POINTER(StageConfig), _P, _SZ, _P, _SZ, ctypes.POINTER(_P)], _I),
    "merak_stage_destroy": ([_P], _I),
    "merak_stage_fwd": ([_P, _P, _P, _P, _P, _P, _P], _I),
    "merak_stage_recompute": ([_P, _P, _P, _P], _I),
    "merak_stage_bwd": ([_P, _P, _P, _P, _P, _I, _P, _P, _P], _I),
    "merak_stage_set_timing": ([_P, _I], _I),
    "merak_stage_read_timing": ([_P, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)], _I),
    "merak_gemm": ([_I, _I, _I, _I, _I, _I, _I, _P, _I, _P, _I, _P, _P, _P, _P, _I, _P], _I),
    "merak_gemm_tile_override": ([_I], _I),
    "merak_plan_recompute": ([_I, ctypes.c_double, _I, _P, _P], _I),
    "merak_schedule_stage": ([_I, _I, _I, _I, _P, _I, ctypes.POINTER(_I)], _I),
    "merak_schedule_simulate": ([_I, _I, _I, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                                 ctypes.POINTER(ctypes.c_double), _P], _I),
    "merak_debug_fail_after": ([_I], _I),
    "merak_schedule_inflight": ([_I, _I, _I, _I, ctypes.POINTER(_I)], _I),
    "merak_schedule_run": ([_I, _I, _I, _I, _P, _I, _P, _P, _P, _P, _P, _P, _I, _P, _P], _I),
    "merak_graph_shard": ([_I, _P, _P, _P, _P, _P, _I, _P, _I, _P, ctypes.POINTER(ctypes.c_int32), _P, _P, _I], _I),
    "merak_plan_alpha1": ([_I, ctypes.c_double, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                           ctypes.POINTER(ctypes.c_double)], _I),
    "merak_layernorm_fwd": ([_I, _I, _I, _F, _P, _P, _P, _P, _P, _P, _P], _I),
    "merak_reduce_scratch_elems": ([_I, _I], _SZ),
    "merak_layernorm_bwd": ([_I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I, _P, _P], _I),
    "merak_layernorm_bwd_noalloc": ([_I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I, _P], _I),
    "merak_noalloc_scratch_elems": ([], _SZ),
    "merak_column_sum": ([_I, _I, _I, _P, _P, _I, _P, _P], _I),
    "merak_count_nonfinite": ([_I, _P, ctypes.c_int64, _P, _P], _I),
    "merak_attention_fwd": ([_I, _I, _I, _I, _I, _P, _P, _P, _P], _I),
    "merak_attention_bwd": ([_I, _I, _I, _I, _I, _P, _P, _P, _P, _P, _P, _P], _I),
    "merak_embedding_fwd": ([_I, _I, _I, _I, _I, _L, _F, _P, _P, _P, _P], _I),
    "merak_embedding_scratch_bytes": ([_I, _I], _SZ),
    "merak_embedding_bwd": ([_I, _I, _I, _I, _I, _L, _F, _P, _P, _P, _I, _P, _P], _I),
    "merak_rope_table": ([_I, _I, ctypes.c_double, _P, _P], _I),
    "merak_qk_norm_rope_fwd": ([_I, _I, _I, _I, _I, _I, _I, _F, _P, _P, _P, _P, _I, _P, _I, _P, _P], _I),
    "merak_qk_norm_rope_scratch_elems": ([_I, _I, _I, _I], _SZ),
    "merak_qk_norm_rope_bwd": ([_I, _I, _I, _I, _I, _I, _I, _F, _P, _P, _P, _P, _P, _I, _P, _I, _P, _P, _P, _I, _P,
                                _P], _I),
    "merak_act8_save": ([_I, _I, _I, _P, _P, _P, _P], _I),
    "merak_act8_restore": ([_I, _I, _I, _P, _P, _P, _P], _I),
    "merak_act8_gelu_bwd": ([_I, _I, _I, _P, _P, _P, _P, _P, _P], _I),
    "merak_act8_gemm_dw_scratch_bytes": ([_I, _I, _I, _I], _SZ),
    "merak_act8_gemm_dw": ([_I, _I, _I, _I, _P, _P, _P, _P, _I, _P, _P], _I),
}


def lib() -> ctypes.CDLL:
    """Load the HIP library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2206_04959_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        for name, (args, res) in _SIGS.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = res
        _lib = L
    return _lib


def _check(status: int, what: str) -> None:
    if status != 0:
        raise MerakError(status, what)


def make_config(shape: synth.StageShape) -> StageConfig:
    return StageConfig(shape.n_blocks, shape.hidden, shape.n_heads, shape.ffn, shape.seq_len, shape.micro_batch,
                       shape.tp_degree, shape.n_sub, shape.recompute_mask,
                       BF16 if shape.dtype == "bf16" else FP32, shape.ln_eps)


def validate(cfg: StageConfig) -> int:
    return lib().merak_stage_validate(ctypes.byref(cfg))


def param_layout(cfg: StageConfig):
    """(total elements, offsets [n_blocks, 12])."""
    total = ctypes.c_size_t()
    offs = np.zeros(cfg.n_blocks * PARAMS_PER_BLOCK, dtype=np.uint64)
    _check(lib().merak_stage_param_layout(ctypes.byref(cfg), ctypes.byref(total),
                                          offs.ctypes.data_as(ctypes.c_void_p)), "param_layout")
    return int(total.value), offs.reshape(cfg.n_blocks, PARAMS_PER_BLOCK).astype(np.int64)


def workspace_bytes(cfg: StageConfig):
    ws, rc = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().merak_stage_workspace_bytes(ctypes.byref(cfg), ctypes.byref(ws), ctypes.byref(rc)),
           "workspace_bytes")
    return int(ws.value), int(rc.value)


def pack_params(cfg: StageConfig, blocks: Sequence[Dict[str, np.ndarray]]) -> np.ndarray:
    """Flat host parameter buffer (uint16 bf16 bits or float32) in the library's
    layout from per-block dicts of device-format arrays."""
    total, offs = param_layout(cfg)
    dt = np.uint16 if cfg.dtype == BF16 else np.float32
    flat = np.zeros(total, dtype=dt)
    for l, blk in enumerate(blocks):
        for i, name in enumerate(synth.PARAM_NAMES):
            a = np.ascontiguousarray(blk[name]).ravel()
            flat[offs[l, i]: offs[l, i] + a.size] = a.astype(dt, copy=False)
    return flat


def unpack(cfg: StageConfig, flat: np.ndarray, shape: synth.StageShape) -> List[Dict[str, np.ndarray]]:
    """Per-block dicts of views into a flat buffer laid out like the parameters."""
    _, offs = param_layout(cfg)
    shapes = shape.local_param_shapes()
    out = []
    for l in range(cfg.n_blocks):
        d = {}
        for i, name in enumerate(synth.PARAM_NAMES):
            n = int(np.prod(shapes[name]))
            d[name] = flat[offs[l, i]: offs[l, i] + n].reshape(shapes[name])
        out.append(d)
    return out


# ---------------------------------------------------------------------------
# torch plumbing (device memory and streams)
# ---------------------------------------------------------------------------

def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(s) -> Optional[int]:
    import torch
    if s is None:
        return torch.cuda.current_stream().cuda_stream
    return s.cuda_stream


def to_device(payload: np.ndarray, device="cuda"):
    """Upload a device-format host array (uint16 bf16 bits or float32)."""
    import torch
    if payload.dtype == np.uint16:
        return torch.from_numpy(np.ascontiguousarray(payload).view(np.int16)).view(torch.bfloat16).to(device)
    return torch.from_numpy(np.ascontiguousarray(payload, dtype=np.float32)).to(device)


def to_host_f64(t) -> np.ndarray:
    import torch
    return t.detach().to(torch.float32).cpu().numpy().astype(np.float64)


class Stage:
    """A handle of the HIP library plus its caller-owned device memory."""

    def __init__(self, shape: synth.StageShape, recompute_area=None, device="cuda"):
        import torch
        self.shape = shape
        self.cfg = make_config(shape)
        ws, rc = workspace_bytes(self.cfg)
        self.workspace_bytes, self.recompute_bytes = ws, rc
        self.workspace = torch.empty(max(ws, 256), dtype=torch.uint8, device=device)
        if rc > 0 and recompute_area is None:
            recompute_area = torch.empty(rc, dtype=torch.uint8, device=device)
        self.recompute_area = recompute_area
        h = ctypes.c_void_p()
        _check(lib().merak_stage_create(ctypes.byref(self.cfg), self.workspace.data_ptr(), ws,
                                        _ptr(recompute_area), rc, ctypes.byref(h)), "merak_stage_create")
        self.handle = h

    def fwd(self, params, x, y, fwd_partials=None, streams=(None, None)) -> None:
        _check(lib().merak_stage_fwd(self.handle, _ptr(params), _ptr(x), _ptr(y), _ptr(fwd_partials),
                                     _stream(streams[0]), _stream(streams[1])), "merak_stage_fwd")

    def recompute(self, params, streams=(None, None)) -> None:
        _check(lib().merak_stage_recompute(self.handle, _ptr(params), _stream(streams[0]), _stream(streams[1])),
               "merak_stage_recompute")

    def bwd(self, params, dy, dx, grads, accumulate=False, bwd_partials=None, streams=(None, None)) -> None:
        _check(lib().merak_stage_bwd(self.handle, _ptr(params), _ptr(dy), _ptr(dx), _ptr(grads), int(accumulate),
                                     _ptr(bwd_partials), _stream(streams[0]), _stream(streams[1])),
               "merak_stage_bwd")

    def set_timing(self, kernel_class: int) -> None:
        _check(lib().merak_stage_set_timing(self.handle, kernel_class), "merak_stage_set_timing")

    def read_timing(self):
        """(total ms, launches) of the timed kernel class since the last read."""
        ms, n = ctypes.c_double(), ctypes.c_int64()
        _check(lib().merak_stage_read_timing(self.handle, ctypes.byref(ms), ctypes.byref(n)),
               "merak_stage_read_timing")
        return float(ms.value), int(n.value)

    def close(self) -> None:
        if getattr(self, "handle", None):
            lib().merak_stage_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------------------
# Per-kernel entry points
# ---------------------------------------------------------------------------

def _dt(t) -> int:
    import torch
    return BF16 if t.dtype == torch.bfloat16 else FP32


def gemm(a, b, c, M, N, K, a_trans=False, b_trans=False, epilogue=EPI_STORE, bias=None, resid=None, aux=None,
         accumulate=False, lda=None, ldb=None, dtype=None, stream=None) -> None:
    dt = _dt(a) if dtype is None else dtype
    lda = lda if lda is not None else (M if a_trans else K)
    ldb = ldb if ldb is not None else (N if b_trans else K)
    _check(lib().merak_gemm(dt, int(a_trans), int(b_trans), epilogue, M, N, K, _ptr(a), lda, _ptr(b), ldb,
                            _ptr(c), _ptr(bias), _ptr(resid), _ptr(aux), int(accumulate), _stream(stream)),
           "merak_gemm")


SCHED_1F1B, SCHED_EARLY_RECOMPUTE, SCHED_SCP = range(3)
OP_FWD, OP_RECOMPUTE, OP_BWD, OP_RECOMPUTE_BWD = range(4)


def schedule_stage(kind: int, n_stages: int, n_micro: int, stage: int):
    """Op list of one stage: [(op type, micro-batch)]."""
    n = ctypes.c_int()
    buf = (ctypes.c_int32 * (3 * n_micro + 4))()
    _check(lib().merak_schedule_stage(kind, n_stages, n_micro, stage, buf, len(buf), ctypes.byref(n)),
           "merak_schedule_stage")
    return [(int(v) >> 24, int(v) & 0xFFFFFF) for v in buf[:n.value]]


def schedule_simulate(kind: int, n_stages: int, n_micro: int, cost_fwd=1.0, cost_rc=1.0, cost_bwd=2.0):
    """(makespan, [busy time per stage]) of the greedy in-order execution."""
    mk = ctypes.c_double()
    busy = (ctypes.c_double * n_stages)()
    _check(lib().merak_schedule_simulate(kind, n_stages, n_micro, cost_fwd, cost_rc, cost_bwd, ctypes.byref(mk), busy),
           "merak_schedule_simulate")
    return float(mk.value), list(busy)


def schedule_inflight(kind: int, n_stages: int, n_micro: int, stage: int) -> int:
    """Handles merak_schedule_run needs for this stage (micro-batches in flight)."""
    n = ctypes.c_int()
    _check(lib().merak_schedule_inflight(kind, n_stages, n_micro, stage, ctypes.byref(n)), "merak_schedule_inflight")
    return int(n.value)


def schedule_run(kind: int, n_stages: int, n_micro: int, stage: int, stages, params, xs, ys, dys, dxs, grads,
                 accumulate=False, streams=(None, None)) -> None:
    """Run one stage's op list through its handles (`stages`: Stage objects)."""
    hs = (ctypes.c_void_p * len(stages))(*[s.handle.value for s in stages])
    arr = lambda ts: (ctypes.c_void_p * len(ts))(*[t.data_ptr() for t in ts])  # noqa: E731
    _check(lib().merak_schedule_run(kind, n_stages, n_micro, stage, hs, len(stages), _ptr(params), arr(xs), arr(ys),
                                    arr(dys), arr(dxs), _ptr(grads), int(accumulate), _stream(streams[0]),
                                    _stream(streams[1])), "merak_schedule_run")


def plan_recompute(n_stages: int, alpha1: float, blocks_per_stage: int):
    """Stage-aware recomputation plan: ([alpha_i], [recompute mask of stage i])."""
    a = (ctypes.c_double * n_stages)()
    m = (ctypes.c_uint64 * n_stages)()
    _check(lib().merak_plan_recompute(n_stages, alpha1, blocks_per_stage, a, m), "merak_plan_recompute")
    return list(a), list(m)


def plan_alpha1(n_stages: int, mem_runtime: float, mem_activation: float, capacity: float, step: float) -> float:
    """Largest feasible alpha_1 on the grid of `step` under the stage memory model."""
    out = ctypes.c_double()
    _check(lib().merak_plan_alpha1(n_stages, mem_runtime, mem_activation, capacity, step, ctypes.byref(out)),
           "merak_plan_alpha1")
    return float(out.value)


def debug_fail_after(launches: int) -> int:
    """Inject a launch failure after `launches` more stage launches (-1: off)."""
    return int(lib().merak_debug_fail_after(int(launches)))


def gemm_tile_override(cfg: int) -> int:
    """Force a bf16 GEMM tile shape (1..10) or restore the built-in choice (0);
    returns the previous setting."""
    prev = int(lib().merak_gemm_tile_override(int(cfg)))
    if prev < 0:
        raise ValueError(f"tile configuration {cfg} out of range")
    return prev


def layernorm_fwd(x, gamma, beta, y, mean, rstd, eps=1e-5, stream=None) -> None:
    rows, h = x.shape[0], x.shape[-1]
    _check(lib().merak_layernorm_fwd(_dt(x), rows, h, eps, _ptr(x), _ptr(gamma), _ptr(beta), _ptr(y), _ptr(mean),
                                     _ptr(rstd), _stream(stream)), "merak_layernorm_fwd")


def reduce_scratch_elems(rows: int, cols: int) -> int:
    return int(lib().merak_reduce_scratch_elems(rows, cols))


def layernorm_bwd(dout, x, mean, rstd, gamma, dres, dx, dgamma, dbeta, scratch, accumulate=False,
                  stream=None) -> None:
    rows, h = x.shape[0], x.shape[-1]
    _check(lib().merak_layernorm_bwd(_dt(x), rows, h, _ptr(dout), _ptr(x), _ptr(mean), _ptr(rstd), _ptr(gamma),
                                     _ptr(dres), _ptr(dx), _ptr(dgamma), _ptr(dbeta), int(accumulate),
                                     _ptr(scratch), _stream(stream)), "merak_layernorm_bwd")


def layernorm_bwd_noalloc(dout, x, mean, rstd, gamma, dres, dx, dgamma, dbeta, accumulate=False,
                          stream=None) -> None:
    rows, h = x.shape[0], x.shape[-1]
    _check(lib().merak_layernorm_bwd_noalloc(_dt(x), rows, h, _ptr(dout), _ptr(x), _ptr(mean), _ptr(rstd),
                                             _ptr(gamma), _ptr(dres), _ptr(dx), _ptr(dgamma), _ptr(dbeta),
                                             int(accumulate), _stream(stream)), "merak_layernorm_bwd_noalloc")


def noalloc_scratch_elems() -> int:
    return int(lib().merak_noalloc_scratch_elems())


def column_sum(x, out, scratch, accumulate=False, stream=None) -> None:
    rows, cols = x.shape
    _check(lib().merak_column_sum(_dt(x), rows, cols, _ptr(x), _ptr(out), int(accumulate), _ptr(scratch),
                                  _stream(stream)), "merak_column_sum")


def count_nonfinite(x, count, stream=None) -> None:
    """Enqueue the count of NaN/Inf elements of tensor x into count (a device int64 tensor of one element)."""
    import torch
    if x.dtype not in (torch.bfloat16, torch.float32) or count.dtype != torch.int64 or count.numel() != 1:
        raise ValueError("count_nonfinite: x bf16 or fp32, count one int64 element")
    _check(lib().merak_count_nonfinite(_dt(x), _ptr(x), x.numel(), _ptr(count), _stream(stream)),
           "merak_count_nonfinite")


def attention_fwd(qkv, o, lse, batch, seq, heads, head_dim, stream=None) -> None:
    _check(lib().merak_attention_fwd(_dt(qkv), batch, seq, heads, head_dim, _ptr(qkv), _ptr(o), _ptr(lse),
                                     _stream(stream)), "merak_attention_fwd")


def attention_bwd(qkv, o, lse, dout, dqkv, delta, batch, seq, heads, head_dim, stream=None) -> None:
    _check(lib().merak_attention_bwd(_dt(qkv), batch, seq, heads, head_dim, _ptr(qkv), _ptr(o), _ptr(lse),
                                     _ptr(dout), _ptr(dqkv), _ptr(delta), _stream(stream)), "merak_attention_bwd")


# ---------------------------------------------------------------------------
# Operators around the blocks
# ---------------------------------------------------------------------------

I32, I64 = 0, 1
_INT = 0x7fffffff  # the largest size that fits the entry points' integers: ctypes cuts others to 32 bits
_torch = None


def _load_torch():
    """torch, imported by the first call that needs it (an import statement in every function
    costs a short call a tenth of its time)."""
    global _torch
    import torch
    _torch = torch
    return torch


def _call(what: str, fn: str, args, stream, names: str, *tensors) -> None:
    """Call the entry point fn(*args, stream) after checking that the tensors (None: not given)
    are dense and on one GPU.  The call goes to that GPU: its current stream unless `stream`
    names another one of its streams.  (A short call's time is mostly the host's, so the checks
    are kept to a tenth of a microsecond or two each.)"""
    torch = _torch or _load_torch()
    index = tensors[0].get_device()
    for t in tensors:
        if t is not None and (t.get_device() != index or not t.is_contiguous()):
            index = -1
    if index < 0:
        for name, t in zip(names.split(), tensors):
            if t is not None and not t.is_contiguous():
                raise ValueError(f"{what}: {name} is not contiguous")
        where = ", ".join(f"{name}: {t.device}" for name, t in zip(names.split(), tensors) if t is not None)
        raise ValueError(f"{what}: tensors are not on one GPU ({where})")
    if stream is None:
        handle = torch._C._cuda_getCurrentRawStream(index)  # a fifteenth of torch.cuda.current_stream's time
    elif stream.device.index != index:
        raise ValueError(f"{what}: the stream is on {stream.device}, the tensors on cuda:{index}")
    else:
        handle = stream.cuda_stream
    entry = getattr(_lib or lib(), fn)
    if torch._C._cuda_getDevice() == index:
        status = entry(*args, handle)
    else:
        with torch.cuda.device(index):
            status = entry(*args, handle)
    if status:
        raise MerakError(status, fn)


def _element(what: str, *tensors) -> int:
    """BF16 or FP32 of tensors that share that type."""
    torch = _torch or _load_torch()
    dt = tensors[0].dtype
    for t in tensors:
        if t.dtype is not dt:
            raise ValueError(f"{what}: element types differ")
    if dt is torch.bfloat16:
        return BF16
    if dt is torch.float32:
        return FP32
    raise ValueError(f"{what}: element type {dt}: bf16 or fp32")


def _too_large(what: str, **sizes) -> None:
    raise ValueError(f"{what}: too large: " + ", ".join(f"{name} {value}" for name, value in sizes.items()))


def _count(what: str, ids, rows: int, hidden: int, first_id: int) -> int:
    """How many ids there are; all sizes fit the entry point's integers."""
    n = ids.numel()
    if (n | rows | hidden) > _INT or not -1 << 63 <= first_id < 1 << 63:
        _too_large(what, ids=n, rows=rows, hidden=hidden, first_id=first_id)
    return n


def _scratch(what: str, scratch, nbytes: int):
    """Pointer of a scratch tensor of at least nbytes (None if it needs none)."""
    if nbytes == 0:
        return None
    if scratch is None or scratch.numel() * scratch.element_size() < nbytes:
        raise ValueError(f"{what}: scratch of {nbytes} bytes needed")
    return scratch.data_ptr()


def _id_type(what: str, ids) -> int:
    torch = _torch or _load_torch()
    if ids.dtype is torch.int64:
        return I64
    if ids.dtype is torch.int32:
        return I32
    raise ValueError(f"{what}: ids of type {ids.dtype}: int32 or int64")


def embedding_fwd(ids, table, y, scale=1.0, first_id=0, stream=None) -> None:
    """y[t] = scale * table[ids[t] - first_id]; zeros for ids outside the table's rows.
    ids int32 or int64 of any shape, table [rows, hidden], y ids.shape + [hidden]."""
    what = "embedding_fwd"
    dt, it = _element(what, table, y), _id_type(what, ids)
    if table.dim() != 2:
        raise ValueError(f"{what}: table is [rows, hidden]")
    rows, hidden = table.shape
    tokens = _count(what, ids, rows, hidden, first_id)
    if y.numel() != tokens * hidden or y.shape[-1] != hidden:
        raise ValueError(f"{what}: y is one row for each id")
    _call(what, "merak_embedding_fwd", (dt, it, tokens, hidden, rows, first_id, scale, ids.data_ptr(),
                                        table.data_ptr(), y.data_ptr()), stream, "ids table y", ids, table, y)


@functools.lru_cache(maxsize=256)
def embedding_scratch_bytes(tokens: int, hidden: int) -> int:
    if max(abs(tokens), abs(hidden)) > _INT:
        _too_large("embedding_scratch_bytes", tokens=tokens, hidden=hidden)
    return int(lib().merak_embedding_scratch_bytes(tokens, hidden))


def embedding_bwd(ids, dy, dtable, scratch=None, scale=1.0, first_id=0, accumulate=False, stream=None) -> None:
    """dtable[v] (= or +=) scale * sum of dy[t] over the tokens t with ids[t] - first_id = v;
    dtable fp32 [rows, hidden], scratch of embedding_scratch_bytes(tokens, hidden) bytes."""
    torch = _torch or _load_torch()
    what = "embedding_bwd"
    dt, it = _element(what, dy), _id_type(what, ids)
    if dtable.dim() != 2 or dtable.dtype is not torch.float32:
        raise ValueError(f"{what}: dtable is fp32 [rows, hidden]")
    rows, hidden = dtable.shape
    tokens = _count(what, ids, rows, hidden, first_id)
    if dy.numel() != tokens * hidden or dy.shape[-1] != hidden:
        raise ValueError(f"{what}: dy is one row for each id")
    sp = _scratch(what, scratch, embedding_scratch_bytes(tokens, hidden))
    _call(what, "merak_embedding_bwd", (dt, it, tokens, hidden, rows, first_id, scale, ids.data_ptr(), dy.data_ptr(),
                                        dtable.data_ptr(), int(accumulate), sp), stream,
          "ids dy dtable scratch", ids, dy, dtable, scratch)


def rope_table(table, theta=10000.0, stream=None) -> None:
    """Fill table fp32 [positions, rope_dim / 2, 2] with the cosines and sines of
    position * theta^(-2 i / rope_dim)."""
    positions, rope = _table("rope_table", table)
    _call("rope_table", "merak_rope_table", (positions, rope, theta, table.data_ptr()), stream, "table", table)


def _table(what: str, table):
    """(positions, rotated features) of a rotation table."""
    torch = _torch or _load_torch()
    if table.dim() != 3 or table.shape[2] != 2 or table.dtype is not torch.float32:
        raise ValueError(f"{what}: table is fp32 [positions, rope_dim / 2, 2]")
    positions, rope = table.shape[0], 2 * table.shape[1]
    if (positions | rope) > _INT:
        _too_large(what, positions=positions, rope_dim=rope)
    return positions, rope


def _qk_args(what, qkv, q_gamma, k_gamma, table, positions, q_heads, kv_heads, seq_len, interleaved, eps):
    """(leading arguments, table and position arguments) of the query/key norm calls."""
    torch = _torch or _load_torch()
    dt = _element(what, qkv, q_gamma, k_gamma)
    d = q_gamma.numel()
    if k_gamma.numel() != d:
        raise ValueError(f"{what}: q_gamma and k_gamma hold one head's features")
    row, n = (q_heads + 2 * kv_heads) * d, qkv.numel()
    if q_heads <= 0 or kv_heads <= 0 or row <= 0 or n % row != 0:
        raise ValueError(f"{what}: qkv is [tokens, q_heads + 2 * kv_heads, head_dim]")
    tokens = n // row
    if (tokens | q_heads | kv_heads | d) > _INT:
        _too_large(what, tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, head_dim=d)
    if table is None:
        return (dt, tokens, q_heads, kv_heads, d, 0, int(interleaved), eps), (None, 0, None, 0)
    rows, rope = _table(what, table)
    if positions is not None:
        if positions.dtype is not torch.int32 or positions.numel() != tokens:
            raise ValueError(f"{what}: positions is int32, one for each token")
        place = positions.data_ptr()
    else:
        if seq_len is None:
            raise ValueError(f"{what}: positions or seq_len needed")
        if not -_INT <= seq_len <= _INT:
            _too_large(what, seq_len=seq_len)
        place = None
    return ((dt, tokens, q_heads, kv_heads, d, rope, int(interleaved), eps),
            (table.data_ptr(), rows, place, seq_len or 0))


def qk_norm_rope_fwd(qkv, q_gamma, k_gamma, table, out, q_heads, kv_heads, positions=None, seq_len=None,
                     interleaved=False, eps=1e-6, stream=None) -> None:
    """RMS norm of each query and key head of qkv [.., q_heads + 2 * kv_heads, head_dim] and
    rotation by the token's position, into out (qkv itself or another tensor).  Without a
    table the heads are only normalised; without positions token t is at t % seq_len."""
    what = "qk_norm_rope_fwd"
    head, tail = _qk_args(what, qkv, q_gamma, k_gamma, table, positions, q_heads, kv_heads, seq_len, interleaved, eps)
    if out.dtype is not qkv.dtype or out.numel() != qkv.numel():
        raise ValueError(f"{what}: out has qkv's type and size")
    _call(what, "merak_qk_norm_rope_fwd", (*head, qkv.data_ptr(), q_gamma.data_ptr(), k_gamma.data_ptr(), *tail,
                                           out.data_ptr()), stream,
          "qkv q_gamma k_gamma table positions out", qkv, q_gamma, k_gamma, table, positions, out)


@functools.lru_cache(maxsize=256)
def qk_norm_rope_scratch_elems(tokens: int, q_heads: int, kv_heads: int, head_dim: int) -> int:
    if max(map(abs, (tokens, q_heads, kv_heads, head_dim))) > _INT:
        _too_large("qk_norm_rope_scratch_elems", tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim)
    return int(lib().merak_qk_norm_rope_scratch_elems(tokens, q_heads, kv_heads, head_dim))


def qk_norm_rope_bwd(dout, qkv, q_gamma, k_gamma, table, dqkv, dq_gamma, dk_gamma, scratch, q_heads, kv_heads,
                     positions=None, seq_len=None, interleaved=False, eps=1e-6, accumulate=False,
                     stream=None) -> None:
    """Gradient of qk_norm_rope_fwd from the raw qkv: dqkv (dout itself or another tensor) and
    the gains' fp32 gradients, written or added."""
    torch = _torch or _load_torch()
    what = "qk_norm_rope_bwd"
    head, tail = _qk_args(what, qkv, q_gamma, k_gamma, table, positions, q_heads, kv_heads, seq_len, interleaved, eps)
    n = qkv.numel()
    if dout.dtype is not qkv.dtype or dqkv.dtype is not qkv.dtype or dout.numel() != n or dqkv.numel() != n:
        raise ValueError(f"{what}: dout and dqkv have qkv's type and size")
    d = q_gamma.numel()
    for g in (dq_gamma, dk_gamma):
        if g.dtype is not torch.float32 or g.numel() != d:
            raise ValueError(f"{what}: dq_gamma and dk_gamma are fp32 [head_dim]")
    sp = _scratch(what, scratch, 4 * qk_norm_rope_scratch_elems(head[1], q_heads, kv_heads, d))
    _call(what, "merak_qk_norm_rope_bwd", (*head, dout.data_ptr(), qkv.data_ptr(), q_gamma.data_ptr(),
                                           k_gamma.data_ptr(), *tail, dqkv.data_ptr(), dq_gamma.data_ptr(),
                                           dk_gamma.data_ptr(), int(accumulate), sp), stream,
          "dout qkv q_gamma k_gamma table positions dqkv dq_gamma dk_gamma scratch",
          dout, qkv, q_gamma, k_gamma, table, positions, dqkv, dq_gamma, dk_gamma, scratch)


def _act8(what, q, scales):
    """(rows, cols) of a checkpoint."""
    torch = _torch or _load_torch()
    if q.dtype is not torch.uint8 or scales.dtype is not torch.uint8:
        raise ValueError(f"{what}: q and scales are uint8")
    cols, n = q.shape[-1], q.numel()
    if cols <= 0 or cols % 32 or scales.shape[-1] * 32 != cols or scales.numel() * 32 != n:
        raise ValueError(f"{what}: q is [rows, cols] and scales [rows, cols / 32], cols a multiple of 32")
    rows = n // cols
    if (rows | cols) > _INT:
        _too_large(what, rows=rows, cols=cols)
    return rows, cols


def _like(what, q, names, *tensors) -> None:
    for t in tensors:
        if t.numel() != q.numel() or t.shape[-1] != q.shape[-1]:
            raise ValueError(f"{what}: {names} q's shape")


def act8_save(x, q, scales, stream=None) -> None:
    """Keep x [.., cols] as e4m3 codes q uint8 [.., cols] and scales uint8 [.., cols / 32]."""
    what = "act8_save"
    dt = _element(what, x)
    rows, cols = _act8(what, q, scales)
    _like(what, q, "x has", x)
    _call(what, "merak_act8_save", (dt, rows, cols, x.data_ptr(), q.data_ptr(), scales.data_ptr()), stream,
          "x q scales", x, q, scales)


def act8_restore(q, scales, x, stream=None) -> None:
    """x from its checkpoint."""
    what = "act8_restore"
    dt = _element(what, x)
    rows, cols = _act8(what, q, scales)
    _like(what, q, "x has", x)
    _call(what, "merak_act8_restore", (dt, rows, cols, q.data_ptr(), scales.data_ptr(), x.data_ptr()), stream,
          "q scales x", q, scales, x)


def act8_gelu_bwd(dg, q, scales, du, g=None, stream=None) -> None:
    """du = dg * GeLU'(u) and, if given, g = GeLU(u), with u from its checkpoint; du may be dg."""
    what = "act8_gelu_bwd"
    given = (dg, du) if g is None else (dg, du, g)
    dt = _element(what, *given)
    rows, cols = _act8(what, q, scales)
    _like(what, q, "dg, du and g have", *given)
    _call(what, "merak_act8_gelu_bwd", (dt, rows, cols, dg.data_ptr(), q.data_ptr(), scales.data_ptr(), du.data_ptr(),
                                        _ptr(g)), stream, "dg q scales du g", dg, q, scales, du, g)


@functools.lru_cache(maxsize=256)
def act8_gemm_dw_scratch_bytes(dtype, tokens: int, n_out: int, n_in: int) -> int:
    """dtype: the torch type of dy."""
    torch = _torch or _load_torch()
    if max(abs(tokens), abs(n_out), abs(n_in)) > _INT:
        _too_large("act8_gemm_dw_scratch_bytes", tokens=tokens, n_out=n_out, n_in=n_in)
    dt = BF16 if dtype == torch.bfloat16 else FP32
    return int(lib().merak_act8_gemm_dw_scratch_bytes(dt, tokens, n_out, n_in))


def act8_gemm_dw(dy, q, scales, dw, scratch=None, accumulate=False, stream=None) -> None:
    """dw [n_out, n_in] fp32 (= or +=) dy^T X, with dy [.., n_out] and X [.., n_in] from its
    checkpoint; scratch of act8_gemm_dw_scratch_bytes(dy.dtype, tokens, n_out, n_in) bytes."""
    torch = _torch or _load_torch()
    what = "act8_gemm_dw"
    dt = _element(what, dy)
    tokens, n_in = _act8(what, q, scales)
    if dw.dim() != 2 or dw.dtype is not torch.float32 or dw.shape[1] != n_in:
        raise ValueError(f"{what}: dw is fp32 [n_out, n_in]")
    n_out = dw.shape[0]
    if dy.numel() != tokens * n_out or dy.shape[-1] != n_out:
        raise ValueError(f"{what}: dy is [tokens, n_out]")
    sp = _scratch(what, scratch, act8_gemm_dw_scratch_bytes(dy.dtype, tokens, n_out, n_in))
    _call(what, "merak_act8_gemm_dw", (dt, tokens, n_out, n_in, dy.data_ptr(), q.data_ptr(), scales.data_ptr(),
                                       dw.data_ptr(), int(accumulate), sp), stream,
          "dy q scales dw scratch", dy, q, scales, dw, scratch)
