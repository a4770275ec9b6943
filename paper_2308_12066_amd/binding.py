"""Thin ctypes binding of libpgmoe.so: argument marshalling only.

Every step of the path runs inside the library's HIP kernels; torch is used by callers for
device memory and streams.  The functions mirror include/pgmoe.h one to one.  Importing this
module loads the library and raises if it is missing: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, Structure, byref, c_char_p, c_float, c_int, c_int32, c_int64, c_size_t, c_uint32, c_void_p

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libpgmoe.so")

OK, EINVAL, ENOTPINNED, ENOSLOT, EBADINDEX, EHIP, ENODEVICE, ESTATE = 0, -1, -2, -3, -4, -5, -6, -7
F32, BF16, F16, E4M3, E5M2 = 0, 1, 2, 3, 4
SCORE_SOFTMAX, SCORE_SIGMOID = 0, 1
MAX_GROUPS = 16
FP8_BLOCK = 128
STREAMS_COMPUTE_COPY, STREAMS_COMPUTE_OWN, STREAMS_COPY_OWN = 1, 2, 4
FLAG_HOST_ONLY = 1
FLAG_FETCH_MEMCPY = 2
FLAG_FETCH_AUTO = 4
AUTO_COPY_ENGINE_BYTES = 256 << 20
SCHED_PREGATED, SCHED_ON_DEMAND, SCHED_PREFETCH_ALL = 0, 1, 2
CACHE_LRU, CACHE_LFU, CACHE_LIFO = 0, 1, 2
MAX_CACHE_SLOTS = 64
MAX_PREGATE_DISTANCE = 3
MAX_EXPERTS = 256
STATIC_SCRATCH_BYTES = 32 << 20

EXPORTS = [
    "pgmoe_create", "pgmoe_destroy", "pgmoe_last_error", "pgmoe_expert_bytes", "pgmoe_workspace_bytes",
    "pgmoe_pack_expert", "pgmoe_unpack_expert", "pgmoe_pregate_topk", "pgmoe_register_host_experts",
    "pgmoe_register_resident_experts", "pgmoe_fetch_experts", "pgmoe_get_fetch_stats", "pgmoe_unique_experts",
    "pgmoe_permute", "pgmoe_expert_ffn", "pgmoe_combine", "pgmoe_stack_step", "pgmoe_device_flags",
    "pgmoe_ffn_timing_begin", "pgmoe_ffn_timing_end", "pgmoe_slot_address", "pgmoe_fetch_timing", "pgmoe_trace", "pgmoe_get_block_trace", "pgmoe_fetch_all_experts", "pgmoe_set_schedule",
    "pgmoe_ffn_kernel_name", "pgmoe_set_nonmoe_standin", "pgmoe_check_streams", "pgmoe_expert_ffn_static", "pgmoe_migration_engine", "pgmoe_fetch_experts_as_turn",
    "pgmoe_route", "pgmoe_route_backward", "pgmoe_group_rows", "pgmoe_quantize_rows", "pgmoe_quantize_weights", "pgmoe_expert_matmul", "pgmoe_expert_matmul_kernel_name",
]


class Config(Structure):
    _fields_ = [("d_model", c_int32), ("d_ff", c_int32), ("n_experts", c_int32), ("top_k", c_int32),
                ("n_blocks", c_int32), ("max_tokens", c_int32), ("dtype", c_int32), ("slots_per_gen", c_int32),
                ("flags", c_uint32), ("cache_slots", c_int32), ("cache_policy", c_int32),
                ("pregate_distance", c_int32)]


class FetchStats(Structure):
    _fields_ = [("n_unique", c_int32), ("n_copied", c_int32), ("bytes_copied", c_int64),
                ("resident_slots", c_int32), ("cache_hits", c_int32), ("fetch_ms", c_float), ("wait_ms", c_float)]


class BlockTrace(Structure):
    _fields_ = [("fetch_ms", c_float), ("stall_ms", c_float), ("compute_ms", c_float), ("fetch_start_ms", c_float),
                ("fetch_end_ms", c_float), ("block_start_ms", c_float), ("block_end_ms", c_float), ("copy_ms", c_float)]


class StepBuffers(Structure):
    _fields_ = [("gate_w", POINTER(c_void_p)), ("gate_b", POINTER(c_void_p)), ("x_states", c_void_p),
                ("y_blocks", c_void_p), ("topk_idx", c_void_p), ("topk_prob", c_void_p), ("row_of", c_void_p),
                ("expert_offsets", c_void_p), ("x_perm", c_void_p), ("y_perm", c_void_p), ("workspace", c_void_p)]


class RouterConfig(Structure):
    _fields_ = [("n_experts", c_int32), ("top_k", c_int32), ("n_groups", c_int32), ("topk_groups", c_int32), ("score", c_int32),
                ("renormalize", c_int32), ("scale", c_float), ("logits_dtype", c_int32)]


class FP8Rows(Structure):
    _fields_ = [("q", c_void_p), ("q_stride", c_int64), ("scale", c_void_p), ("scale_stride", c_int64), ("rows", c_int32), ("cols", c_int32),
                ("dtype", c_int32)]


class FP8Weights(Structure):
    _fields_ = [("q", c_void_p), ("scale", c_void_p), ("n_experts", c_int32), ("n_in", c_int32), ("n_out", c_int32)]


class PgmoeError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"pgmoe error {code}: {text}")
        self.code = code


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2308_12066_amd.build`")
    # One HIP runtime per process: torch ships its own libamdhip64 and looks it up under a
    # different file name than the system one, so if this library came first the process would
    # hold two runtimes and the second to start would see no device.  Loading torch first makes
    # libpgmoe bind to the runtime torch already brought in (same soname).
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    L = ctypes.CDLL(LIB_PATH)
    vp, i = c_void_p, c_int
    L.pgmoe_create.argtypes = [POINTER(vp), POINTER(Config)]
    L.pgmoe_destroy.argtypes = [vp]
    L.pgmoe_last_error.argtypes = [vp]
    L.pgmoe_last_error.restype = c_char_p
    L.pgmoe_expert_bytes.argtypes = [POINTER(Config)]
    L.pgmoe_expert_bytes.restype = c_size_t
    L.pgmoe_workspace_bytes.argtypes = [vp]
    L.pgmoe_workspace_bytes.restype = c_size_t
    L.pgmoe_pack_expert.argtypes = [POINTER(Config), vp, vp, vp]
    L.pgmoe_unpack_expert.argtypes = [POINTER(Config), vp, vp, vp]
    L.pgmoe_pregate_topk.argtypes = [vp, vp, vp, vp, i, vp, vp, vp, vp]
    L.pgmoe_register_host_experts.argtypes = [vp, vp, c_size_t, c_size_t]
    L.pgmoe_register_resident_experts.argtypes = [vp, vp, c_size_t, c_size_t]
    L.pgmoe_fetch_experts.argtypes = [vp, i, vp, i, vp, vp, POINTER(c_int)]
    L.pgmoe_fetch_experts_as_turn.argtypes = [vp, i, vp, i, vp, i, c_float]
    L.pgmoe_get_fetch_stats.argtypes = [vp, i, POINTER(FetchStats)]
    L.pgmoe_migration_engine.argtypes = [vp]
    L.pgmoe_unique_experts.argtypes = [vp, i, i, vp]
    L.pgmoe_permute.argtypes = [vp, vp, vp, i, vp, vp, vp, vp]
    L.pgmoe_expert_ffn.argtypes = [vp, i, vp, vp, i, vp, vp, vp]
    L.pgmoe_expert_ffn_static.argtypes = [vp, i, vp, vp, i, vp, vp]
    L.pgmoe_combine.argtypes = [vp, vp, vp, vp, i, vp, vp, vp, vp]
    L.pgmoe_stack_step.argtypes = [vp, POINTER(StepBuffers), i, vp, vp]
    L.pgmoe_device_flags.argtypes = [vp, POINTER(c_uint32)]
    L.pgmoe_ffn_timing_begin.argtypes = [vp, i]
    L.pgmoe_ffn_kernel_name.argtypes = [vp, i]
    L.pgmoe_ffn_kernel_name.restype = c_char_p
    L.pgmoe_fetch_timing.argtypes = [vp, i]
    L.pgmoe_trace.argtypes = [vp, i]
    L.pgmoe_fetch_all_experts.argtypes = [vp, i, vp, vp]
    L.pgmoe_set_schedule.argtypes = [vp, i]
    L.pgmoe_set_nonmoe_standin.argtypes = [vp, c_float]
    L.pgmoe_check_streams.argtypes = [vp, vp, vp, POINTER(c_int)]
    L.pgmoe_get_block_trace.argtypes = [vp, i, POINTER(BlockTrace)]
    L.pgmoe_slot_address.argtypes = [vp, i, i, POINTER(vp)]
    L.pgmoe_route.argtypes = [POINTER(RouterConfig), vp, c_int64, vp, i, vp, vp, vp, vp]
    L.pgmoe_route_backward.argtypes = [POINTER(RouterConfig), vp, c_int64, vp, vp, vp, i, vp, c_int64, vp]
    L.pgmoe_group_rows.argtypes = [vp, vp, i, vp, vp, vp]
    L.pgmoe_quantize_rows.argtypes = [vp, c_int64, i, i, vp, i, POINTER(FP8Rows), vp]
    L.pgmoe_quantize_weights.argtypes = [vp, i, POINTER(FP8Weights), POINTER(FP8Weights), vp]
    L.pgmoe_expert_matmul.argtypes = [POINTER(FP8Rows), POINTER(FP8Weights), vp, i, vp, c_int64, i, POINTER(FP8Rows), vp]
    L.pgmoe_expert_matmul_kernel_name.argtypes = [POINTER(FP8Rows), POINTER(FP8Weights), i]
    L.pgmoe_expert_matmul_kernel_name.restype = c_char_p
    L.pgmoe_ffn_timing_end.argtypes = [vp, POINTER(c_int), POINTER(c_float), POINTER(c_float)]
    for name in EXPORTS:
        if name not in ("pgmoe_last_error", "pgmoe_expert_bytes", "pgmoe_workspace_bytes", "pgmoe_ffn_kernel_name", "pgmoe_expert_matmul_kernel_name"):
            getattr(L, name).restype = c_int
    return L


lib = _load()


def _ptr(a):
    """Address of a torch tensor / numpy array / int / None as a void*."""
    if a is None:
        return None
    if isinstance(a, int):
        return c_void_p(a)
    if hasattr(a, "data_ptr"):
        return c_void_p(a.data_ptr())
    if hasattr(a, "ctypes"):
        return c_void_p(a.ctypes.data)
    raise TypeError(f"cannot take the address of {type(a)}")


def _stream(s):
    if s is None:
        return None
    if isinstance(s, int):
        return c_void_p(s)
    return c_void_p(s.cuda_stream)   # torch.cuda.Stream on ROCm carries the hipStream_t here


def last_error(ctx=None) -> str:
    return lib.pgmoe_last_error(ctx).decode()


def make_config(d_model, d_ff, n_experts, top_k, n_blocks, max_tokens, dtype, slots_per_gen=0, flags=0,
                cache_slots=0, cache_policy=0, pregate_distance=0) -> Config:
    return Config(d_model, d_ff, n_experts, top_k, n_blocks, max_tokens, dtype, slots_per_gen, flags, cache_slots,
                  cache_policy, pregate_distance)


def expert_bytes(cfg: Config) -> int:
    return int(lib.pgmoe_expert_bytes(byref(cfg)))


def pack_expert(cfg: Config, w1, w2, blob) -> None:
    rc = lib.pgmoe_pack_expert(byref(cfg), _ptr(w1), _ptr(w2), _ptr(blob))
    if rc:
        raise PgmoeError(rc, last_error())


def unpack_expert(cfg: Config, blob, w1, w2) -> None:
    rc = lib.pgmoe_unpack_expert(byref(cfg), _ptr(blob), _ptr(w1), _ptr(w2))
    if rc:
        raise PgmoeError(rc, last_error())


def unique_experts(idx, n_experts: int):
    import numpy as np
    idx = np.ascontiguousarray(idx, dtype=np.int32).ravel()
    out = np.zeros(max(1, min(n_experts, idx.size)), dtype=np.int32)
    rc = lib.pgmoe_unique_experts(_ptr(idx), idx.size, n_experts, _ptr(out))
    if rc < 0:
        raise PgmoeError(rc, last_error())
    return out[:rc].copy()


# ---- routing and 8-bit experts: no context; tensors carry their sizes, types and strides, and lie on the current GPU.  A call
# takes a few microseconds on the GPU, so what is checked here is checked on the tensors' own attributes.  Without a stream a call
# goes to torch's current one; stream=0 is the null stream.
try:
    import torch as _torch
    _DTYPES = {_torch.float32: F32, _torch.bfloat16: BF16, _torch.float16: F16, _torch.float8_e4m3fn: E4M3, _torch.float8_e5m2: E5M2}
    _f32, _i32 = _torch.float32, _torch.int32
    # address of torch's current stream on a GPU: without a Stream object made for each call, 0.3 us of a call instead of 3
    _current_stream = getattr(_torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: _torch.cuda.current_stream(device).cuda_stream)
except ImportError:  # the calls below take torch tensors
    _DTYPES, _f32, _i32 = {}, None, None


def _dtype(t, name) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} has dtype {t.dtype}: no operator of the library takes it")
    return code


def _expect(t, name, shape, dtype):
    """The checks only the tensor allows: the library sees addresses.  -> its address"""
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, not {dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} is not contiguous")
    return t.data_ptr()


def _stream_for(stream, *tensors):
    """The stream of a call: the given one, or torch's current one, on which the caller's torch operations run.  The library
    launches on the current GPU and sees addresses: all tensors (None: not given) have to be that GPU's."""
    device = tensors[0].get_device()      # -1: not on a GPU
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError(f"tensors on {tensors[0].device} and on {t.device}")
    if device < 0:
        raise ValueError(f"tensors on {tensors[0].device}: the operators take tensors on the GPU")
    if device != _torch.cuda.current_device():
        raise ValueError(f"tensors on {tensors[0].device}, the current GPU is cuda:{_torch.cuda.current_device()}")
    return c_void_p(_current_stream(device)) if stream is None else _stream(stream)


def _row_stride(t, name) -> int:
    """Elements from one row of a matrix to the next; within a row they lie side by side."""
    shape = t.shape
    if len(shape) != 2:
        raise ValueError(f"{name} has {len(shape)} dimensions, not 2")
    row, col = t.stride()
    if col != 1 and shape[1] > 1:
        raise ValueError(f"the elements of a row of {name} do not lie side by side")
    return row if shape[0] > 1 else max(row, shape[1])


def fp8_blocks(n: int) -> int:
    return (n + FP8_BLOCK - 1) // FP8_BLOCK


def _fp8_rows(q, scale, cols, name) -> FP8Rows:
    """q [rows, >= 128 * blocks] codes, scale [blocks, >= rows] float32."""
    code = _DTYPES.get(q.dtype)
    if code != E4M3 and code != E5M2:
        raise TypeError(f"{name} has dtype {q.dtype}, not an 8-bit one")
    stride, (rows, width), blocks = _row_stride(q, name), q.shape, (cols + FP8_BLOCK - 1) // FP8_BLOCK
    if width < FP8_BLOCK * blocks:
        raise ValueError(f"{name} has {width} columns, fewer than the {FP8_BLOCK * blocks} of whole blocks")
    if scale.shape != (blocks, rows) or scale.dtype != _f32:
        raise ValueError(f"{name}'s scale is {scale.dtype} {tuple(scale.shape)}, not float32 {(blocks, rows)}")
    return FP8Rows(q.data_ptr(), stride, scale.data_ptr(), _row_stride(scale, "a scale"), rows, cols, code)


def fp8_weight_shapes(n_experts: int, n_in: int, n_out: int):
    """Shapes of the codes and the scales of n_experts matrices [n_in, n_out]."""
    return ((n_experts, 8 * fp8_blocks(n_out), fp8_blocks(n_in), 2, 4, 16, 16), (n_experts, fp8_blocks(n_out), fp8_blocks(n_in)))


def _fp8_weights(q, scale, n_in, n_out, name) -> FP8Weights:
    n = q.shape[0]
    shape, scale_shape = fp8_weight_shapes(n, n_in, n_out)
    if _DTYPES.get(q.dtype) != E4M3:
        raise TypeError(f"{name} has dtype {q.dtype}, not torch.float8_e4m3fn")
    return FP8Weights(_expect(q, name, shape, q.dtype), _expect(scale, "a scale", scale_shape, _f32), n, n_in, n_out)


class Router:
    """A pgmoe_router: how experts are selected and weighed from logits.  Threads may share one: a call changes nothing in it."""

    def __init__(self, n_experts, top_k, score=SCORE_SOFTMAX, n_groups=1, topk_groups=0, renormalize=False, scale=1.0):
        self._fields = n_experts, top_k, n_groups, topk_groups, score, 1 if renormalize else 0, scale
        self._cfgs = {F32: RouterConfig(*self._fields, F32)}      # by the logits' type, as they come
        self._shape = n_experts, top_k

    def _outer(self, logits):
        stride, (T, E) = _row_stride(logits, "logits"), logits.shape
        if E != self._shape[0]:
            raise ValueError(f"logits of {E} experts, the router has {self._shape[0]}")
        code = _DTYPES.get(logits.dtype)
        cfg = self._cfgs.get(code)
        if cfg is None:
            if code not in (BF16, F16):
                raise TypeError(f"logits have dtype {logits.dtype}, neither float32 nor bfloat16 nor float16")
            cfg = self._cfgs[code] = RouterConfig(*self._fields, code)
        return byref(cfg), T, E, self._shape[1], stride

    def route(self, logits, bias, topk_idx, topk_weight, scores_out=None, stream=None):
        cfg, T, E, k, stride = self._outer(logits)
        args = (cfg, logits.data_ptr(), stride, None if bias is None else _expect(bias, "bias", (E,), _f32), T,
                _expect(topk_idx, "topk_idx", (T, k), _i32), _expect(topk_weight, "topk_weight", (T, k), _f32),
                None if scores_out is None else _expect(scores_out, "scores_out", (T, E), _f32))
        rc = lib.pgmoe_route(*args, _stream_for(stream, logits, bias, topk_idx, topk_weight, scores_out))
        if rc:
            raise PgmoeError(rc, last_error())

    def route_backward(self, logits, topk_idx, d_weight, d_scores, d_logits, stream=None):
        cfg, T, E, k, stride = self._outer(logits)
        if d_logits.shape != (T, E) or d_logits.dtype != logits.dtype:
            raise ValueError(f"d_logits is {d_logits.dtype} {tuple(d_logits.shape)}, logits are {logits.dtype} {(T, E)}")
        args = (cfg, logits.data_ptr(), stride, _expect(topk_idx, "topk_idx", (T, k), _i32), _expect(d_weight, "d_weight", (T, k), _f32),
                None if d_scores is None else _expect(d_scores, "d_scores", (T, E), _f32), T, d_logits.data_ptr(), _row_stride(d_logits, "d_logits"))
        rc = lib.pgmoe_route_backward(*args, _stream_for(stream, logits, topk_idx, d_weight, d_scores, d_logits))
        if rc:
            raise PgmoeError(rc, last_error())


def quantize_rows(x, q, scale, row_of=None, copies=1, stream=None) -> None:
    """x [T, cols] -> codes q [rows, 128 * blocks] and scales [blocks, rows]; row_of [T * copies] deals the rows out."""
    stride, (T, cols) = _row_stride(x, "x"), x.shape
    out = _fp8_rows(q, scale, cols, "q")
    args = (x.data_ptr(), stride, _dtype(x, "x"), T, None if row_of is None else _expect(row_of, "row_of", (T * copies,), _i32), copies, byref(out))
    rc = lib.pgmoe_quantize_rows(*args, _stream_for(stream, x, q, scale, row_of))
    if rc:
        raise PgmoeError(rc, last_error())


def quantize_weights(w, forward_q, forward_scale, backward_q=None, backward_scale=None, stream=None) -> None:
    """w [E, n_in, n_out] -> the operand tiles and scales (fp8_weight_shapes) of x . W and, if given, of dy . W^T."""
    E, n_in, n_out = w.shape
    fwd = None if forward_q is None else _fp8_weights(forward_q, forward_scale, n_in, n_out, "forward_q")
    bwd = None if backward_q is None else _fp8_weights(backward_q, backward_scale, n_out, n_in, "backward_q")
    for f in (fwd, bwd):
        if f is not None and f.n_experts != E:
            raise ValueError(f"codes of {f.n_experts} experts for {E}")
    args = (_expect(w, "w", (E, n_in, n_out), w.dtype), _dtype(w, "w"), None if fwd is None else byref(fwd), None if bwd is None else byref(bwd))
    given = ((forward_q, forward_scale) if fwd is not None else ()) + ((backward_q, backward_scale) if bwd is not None else ())
    rc = lib.pgmoe_quantize_weights(*args, _stream_for(stream, w, *given))
    if rc:
        raise PgmoeError(rc, last_error())


def expert_matmul(x_q, x_scale, w_q, w_scale, expert_offsets, n_in, n_out, y, y_scale=None, relu=False, stream=None) -> None:
    """y[rows] = act(x[rows] . W_e) for the rows of every expert e; y [rows, n_out], or codes with y_scale."""
    x = _fp8_rows(x_q, x_scale, n_in, "x_q")
    w = _fp8_weights(w_q, w_scale, n_in, n_out, "w_q")
    offsets = _expect(expert_offsets, "expert_offsets", (w.n_experts + 1,), _i32)
    if y_scale is not None:
        out = _fp8_rows(y, y_scale, n_out, "y")
        args = (None, 0, out.dtype, byref(out))
    else:
        if y.shape != (x.rows, n_out):
            raise ValueError(f"y has shape {tuple(y.shape)}, not {(x.rows, n_out)}")
        args = (y.data_ptr(), _row_stride(y, "y"), _dtype(y, "y"), None)
    rc = lib.pgmoe_expert_matmul(byref(x), byref(w), offsets, 1 if relu else 0, *args, _stream_for(stream, x_q, x_scale, w_q, w_scale, expert_offsets, y, y_scale))
    if rc:
        raise PgmoeError(rc, last_error())


def expert_matmul_kernel_name(rows, n_experts, n_in, n_out, y_dtype=BF16, q_stride=0):
    """The kernel expert_matmul() launches for these sizes; q_stride: bytes from a row of codes to the next, 0: whole blocks."""
    x = FP8Rows(None, q_stride or FP8_BLOCK * fp8_blocks(n_in), None, rows, rows, n_in, E4M3)
    name = lib.pgmoe_expert_matmul_kernel_name(byref(x), byref(FP8Weights(None, None, n_experts, n_in, n_out)), y_dtype)
    return name.decode() if name is not None else None


class Context:
    """Owns a pgmoe_ctx*.  Methods take tensors (anything with data_ptr()) or raw addresses; without a stream they launch on
    the null stream, group_rows() with tensors on torch's current one."""

    def __init__(self, cfg: Config):
        self.cfg = cfg
        self._h = c_void_p()
        rc = lib.pgmoe_create(byref(self._h), byref(cfg))
        if rc:
            raise PgmoeError(rc, last_error())

    def close(self):
        if self._h:
            lib.pgmoe_destroy(self._h)
            self._h = c_void_p()

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc):
        if rc:
            raise PgmoeError(rc, last_error(self._h))

    @property
    def workspace_bytes(self) -> int:
        return int(lib.pgmoe_workspace_bytes(self._h))

    def pregate_topk(self, x, w_gate, bias, T, topk_idx, topk_prob, probs_out=None, stream=None):
        self._check(lib.pgmoe_pregate_topk(self._h, _ptr(x), _ptr(w_gate), _ptr(bias), T, _ptr(topk_idx),
                                           _ptr(topk_prob), _ptr(probs_out), _stream(stream)))

    def register_host_experts(self, host_base, expert_stride, block_stride):
        self._check(lib.pgmoe_register_host_experts(self._h, _ptr(host_base), expert_stride, block_stride))

    def register_resident_experts(self, dev_base, expert_stride, block_stride):
        self._check(lib.pgmoe_register_resident_experts(self._h, _ptr(dev_base), expert_stride, block_stride))

    def fetch_experts(self, block, topk_idx, T, compute_stream, copy_stream) -> int:
        n = c_int(0)
        self._check(lib.pgmoe_fetch_experts(self._h, block, _ptr(topk_idx), T, _stream(compute_stream),
                                            _stream(copy_stream), byref(n)))
        return n.value

    def fetch_experts_as_turn(self, block, topk_idx, T, stream, seq: int, wait_us: float):
        self._check(lib.pgmoe_fetch_experts_as_turn(self._h, block, _ptr(topk_idx), T, _stream(stream), seq, wait_us))

    @property
    def migration_engine(self) -> str:
        rc = lib.pgmoe_migration_engine(self._h)
        self._check(rc if rc < 0 else 0)
        return "copy_engine" if rc == 1 else "pull"

    def fetch_stats(self, block) -> FetchStats:
        st = FetchStats()
        self._check(lib.pgmoe_get_fetch_stats(self._h, block, byref(st)))
        return st

    def permute(self, x, topk_idx, T, x_perm, row_of, expert_offsets, stream=None):
        self._check(lib.pgmoe_permute(self._h, _ptr(x), _ptr(topk_idx), T, _ptr(x_perm), _ptr(row_of),
                                      _ptr(expert_offsets), _stream(stream)))

    def group_rows(self, topk_idx, T, row_of, expert_offsets, stream=None):
        """Without a stream: on torch's current one, as the operators it stands between, if the arguments are tensors."""
        tensors = topk_idx, row_of, expert_offsets
        on = _stream_for(stream, *tensors) if all(hasattr(t, "get_device") for t in tensors) else _stream(stream)
        self._check(lib.pgmoe_group_rows(self._h, _ptr(topk_idx), T, _ptr(row_of), _ptr(expert_offsets), on))

    def expert_ffn(self, block, x_perm, expert_offsets, n_rows, y_perm, workspace, stream=None):
        self._check(lib.pgmoe_expert_ffn(self._h, block, _ptr(x_perm), _ptr(expert_offsets), n_rows, _ptr(y_perm),
                                         _ptr(workspace), _stream(stream)))

    def expert_ffn_static(self, block, x_perm, expert_offsets, n_rows, y_perm, stream=None):
        self._check(lib.pgmoe_expert_ffn_static(self._h, block, _ptr(x_perm), _ptr(expert_offsets), n_rows, _ptr(y_perm),
                                                _stream(stream)))

    def combine(self, y_perm, row_of, topk_prob, T, y, x_res=None, x_next=None, stream=None):
        self._check(lib.pgmoe_combine(self._h, _ptr(y_perm), _ptr(row_of), _ptr(topk_prob), T, _ptr(y), _ptr(x_res),
                                      _ptr(x_next), _stream(stream)))

    def make_step_buffers(self, gate_w, gate_b, x_states, y_blocks, topk_idx, topk_prob, row_of, expert_offsets,
                          x_perm, y_perm, workspace) -> StepBuffers:
        L = self.cfg.n_blocks
        assert len(gate_w) == L
        gw = (c_void_p * L)(*[g.data_ptr() for g in gate_w])
        gb = None
        if gate_b is not None and any(b is not None for b in gate_b):
            gb = (c_void_p * L)(*[None if b is None else b.data_ptr() for b in gate_b])
        sb = StepBuffers(ctypes.cast(gw, POINTER(c_void_p)), ctypes.cast(gb, POINTER(c_void_p)) if gb else None,
                         _ptr(x_states), _ptr(y_blocks), _ptr(topk_idx), _ptr(topk_prob), _ptr(row_of),
                         _ptr(expert_offsets), _ptr(x_perm), _ptr(y_perm), _ptr(workspace))
        sb._keep = (gw, gb, gate_w, gate_b, x_states, y_blocks, topk_idx, topk_prob, row_of, expert_offsets, x_perm,
                    y_perm, workspace)
        return sb

    def stack_step(self, bufs: StepBuffers, T, compute_stream, copy_stream):
        self._check(lib.pgmoe_stack_step(self._h, byref(bufs), T, _stream(compute_stream), _stream(copy_stream)))

    def device_flags(self) -> int:
        f = c_uint32(0)
        self._check(lib.pgmoe_device_flags(self._h, byref(f)))
        return f.value

    def ffn_kernel_name(self, n_rows: int):
        name = lib.pgmoe_ffn_kernel_name(self._h, n_rows)
        return name.decode() if name is not None else None

    def ffn_timing_begin(self, max_launches: int):
        self._check(lib.pgmoe_ffn_timing_begin(self._h, max_launches))

    def ffn_timing_end(self):
        """-> (timed launches, sum of their event-to-event times in ms, per-pair event overhead in us)."""
        n, ms, oh = c_int(0), c_float(0.0), c_float(0.0)
        self._check(lib.pgmoe_ffn_timing_end(self._h, byref(n), byref(ms), byref(oh)))
        return n.value, ms.value, oh.value * 1e3

    def slot_address(self, block: int, slot: int) -> int:
        p = c_void_p()
        self._check(lib.pgmoe_slot_address(self._h, block, slot, byref(p)))
        return p.value

    def fetch_timing(self, enable: bool):
        self._check(lib.pgmoe_fetch_timing(self._h, 1 if enable else 0))

    def trace(self, enable: bool):
        self._check(lib.pgmoe_trace(self._h, 1 if enable else 0))

    def block_trace(self, block: int) -> BlockTrace:
        t = BlockTrace()
        self._check(lib.pgmoe_get_block_trace(self._h, block, byref(t)))
        return t

    def fetch_all_experts(self, block, compute_stream, copy_stream):
        self._check(lib.pgmoe_fetch_all_experts(self._h, block, _stream(compute_stream), _stream(copy_stream)))

    def set_schedule(self, schedule: int):
        self._check(lib.pgmoe_set_schedule(self._h, schedule))

    def check_streams(self, compute_stream, copy_stream) -> int:
        """Bit mask of the stream pairs that share a hardware queue (STREAMS_*); 0 = all side by side."""
        shared = c_int(0)
        self._check(lib.pgmoe_check_streams(self._h, _stream(compute_stream), _stream(copy_stream), byref(shared)))
        return shared.value

    def set_nonmoe_standin(self, microseconds: float):
        self._check(lib.pgmoe_set_nonmoe_standin(self._h, microseconds))
