"""Python face of the C-ABI library `libqsl.so` (see include/qsl.h): argument marshalling only.

Every step of the hot path runs in the HIP kernels behind the C ABI; torch is used for device
memory and for the current HIP stream.  Importing this module loads the library and raises if
it has not been built -- there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np
import torch

from .build import LIB_PATH

TOPK, RANDK = 0, 1
QSGD, SIGN_L1, SIGN_L2, FP32, QSGD_SCALED, SIGN_L3, SIGN_L4 = 0, 1, 2, 3, 4, 5, 6
FLAG_NO_FAST_PATH = 1
FLAG_NO_SMALL_PATH = 2
FLAG_OWN_V = 4
FLAG_NO_WARM_START = 8
FLAG_DENSE_FORMAT = 16

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}      # QSL_F32, QSL_BF16, QSL_F16
TOP_MAX = 128
TEACHER_MAX = 256
SIZE_END = 1 << 31                                                    # rows and classes stay below

OK, ERR_INVALID_ARG, ERR_BUFFER_TOO_SMALL, ERR_NONFINITE_INPUT, ERR_DEVICE, ERR_UNSUPPORTED = range(6)


class QslError(RuntimeError):
    def __init__(self, status, where):
        self.status = int(status)
        super().__init__(f"{where}: {_lib.qsl_status_string(status).decode()} (status {int(status)})")


class _Config(C.Structure):
    _fields_ = [("d", C.c_uint64), ("num_segments", C.c_uint32), ("seg_offset", C.POINTER(C.c_uint64)),
                ("seg_k", C.POINTER(C.c_uint32)), ("s", C.c_uint32), ("sparsifier", C.c_uint32),
                ("quantizer", C.c_uint32), ("seed", C.c_uint64), ("max_workers", C.c_uint32), ("flags", C.c_uint32)]


class _Logits(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride", C.c_uint64), ("rows", C.c_uint32), ("vocab", C.c_uint32), ("dtype", C.c_uint32),
                ("scale", C.c_float)]


class _Teacher(C.Structure):
    _fields_ = [("index", C.c_void_p), ("value", C.c_void_p), ("lse", C.c_void_p), ("top", C.c_uint32), ("scale", C.c_float)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it first (python -m paper_1906_02367_amd.build, or "
                          f"__graft_entry__.build()); this package has no fallback path")
    lib = C.CDLL(LIB_PATH)
    vp, u32, u64 = C.c_void_p, C.c_uint32, C.c_uint64
    lib.qsl_status_string.argtypes = [C.c_int]; lib.qsl_status_string.restype = C.c_char_p
    lib.qsl_create.argtypes = [C.POINTER(vp), C.POINTER(_Config), vp]; lib.qsl_create.restype = C.c_int
    lib.qsl_destroy.argtypes = [vp]; lib.qsl_destroy.restype = C.c_int
    lib.qsl_set_stream.argtypes = [vp, vp]; lib.qsl_set_stream.restype = C.c_int
    lib.qsl_msg_capacity_bytes.argtypes = [vp]; lib.qsl_msg_capacity_bytes.restype = C.c_size_t
    lib.qsl_compress.argtypes = [vp, vp, vp, vp, u32, u32, u64, vp, vp, vp, vp]; lib.qsl_compress.restype = C.c_int
    lib.qsl_compress_diff.argtypes = [vp, vp, vp, vp, vp, u32, u32, u64, vp, vp, vp, vp]; lib.qsl_compress_diff.restype = C.c_int
    lib.qsl_error_update.argtypes = [vp, vp, vp, vp, u32]; lib.qsl_error_update.restype = C.c_int
    lib.qsl_aggregate.argtypes = [vp, vp, C.POINTER(u32), u32, C.c_float, C.c_int, vp]; lib.qsl_aggregate.restype = C.c_int
    lib.qsl_aggregate_static.argtypes = [C.POINTER(_Config), vp, vp, C.POINTER(u32), u32, C.c_float, C.c_int, vp]
    lib.qsl_aggregate_static.restype = C.c_int
    lib.qsl_bits_sent.argtypes = [vp, vp, u32, C.POINTER(u64)]; lib.qsl_bits_sent.restype = C.c_int
    lib.qsl_device_status.argtypes = [vp]; lib.qsl_device_status.restype = C.c_int
    lib.qsl_debug_units.argtypes = [vp, C.POINTER(u32), u32, C.POINTER(u32)]; lib.qsl_debug_units.restype = C.c_int
    lib.qsl_timing_enable.argtypes = [vp, C.c_int]; lib.qsl_timing_enable.restype = C.c_int
    lib.qsl_timing_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(u32)]; lib.qsl_timing_read.restype = C.c_int
    lib.qsl_bits_index_free.argtypes = [C.POINTER(_Config), C.POINTER(u64)]; lib.qsl_bits_index_free.restype = C.c_int
    lib.qsl_plan_paths.argtypes = [C.POINTER(_Config), C.POINTER(u32)]; lib.qsl_plan_paths.restype = C.c_int
    zp, tp, sz = C.POINTER(_Logits), C.POINTER(_Teacher), C.c_size_t
    lib.qsl_logits_workspace_bytes.argtypes = [zp, u32]; lib.qsl_logits_workspace_bytes.restype = sz
    lib.qsl_token_logprobs.argtypes = [zp, vp, u32, vp, vp, vp, vp, vp, vp, vp, sz, vp]; lib.qsl_token_logprobs.restype = C.c_int
    lib.qsl_token_logprobs_backward.argtypes = [zp, vp, vp, vp, vp, vp, vp, vp, u64, vp, sz, vp]
    lib.qsl_token_logprobs_backward.restype = C.c_int
    lib.qsl_distill.argtypes = [zp, tp, vp, vp, vp, sz, vp]; lib.qsl_distill.restype = C.c_int
    lib.qsl_distill_backward.argtypes = [zp, tp, vp, vp, vp, vp, u64, vp, sz, vp]; lib.qsl_distill_backward.restype = C.c_int
    return lib


_lib = _load()

EXPORTED = ["qsl_create", "qsl_destroy", "qsl_set_stream", "qsl_msg_capacity_bytes", "qsl_compress",
            "qsl_compress_diff", "qsl_error_update", "qsl_aggregate", "qsl_aggregate_static", "qsl_bits_sent", "qsl_bits_index_free", "qsl_plan_paths",
            "qsl_device_status", "qsl_debug_units",
            "qsl_timing_enable", "qsl_timing_read", "qsl_status_string", "qsl_logits_workspace_bytes", "qsl_token_logprobs",
            "qsl_token_logprobs_backward", "qsl_distill", "qsl_distill_backward"]


def _check(status, where):
    if status != OK:
        raise QslError(status, where)


def _ptr(t, dtype=None, allow_none=False):
    if t is None:
        if allow_none:
            return None
        raise ValueError("tensor required")
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous device tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected dtype {dtype}, got {t.dtype}")
    return t.data_ptr()


def bits_index_free(d, seg_offset, seg_k, s, sparsifier, quantizer):
    """`qsl_bits_index_free`: bits of one Rand_k message without its indices (host only, no GPU needed)."""
    off = np.ascontiguousarray(seg_offset, dtype=np.uint64)
    k = np.ascontiguousarray(seg_k, dtype=np.uint32)
    cfg = _Config(int(d), int(k.size), off.ctypes.data_as(C.POINTER(C.c_uint64)), k.ctypes.data_as(C.POINTER(C.c_uint32)),
                  int(s), int(sparsifier), int(quantizer), 0, 1, 0)
    bits = C.c_uint64(0)
    _check(_lib.qsl_bits_index_free(C.byref(cfg), C.byref(bits)), "qsl_bits_index_free")
    return int(bits.value)


def plan_paths(d, seg_offset, seg_k, s, sparsifier, quantizer, flags=0):
    """`qsl_plan_paths`: the selection path of every segment (host only, no GPU needed)."""
    off = np.ascontiguousarray(seg_offset, dtype=np.uint64)
    k = np.ascontiguousarray(seg_k, dtype=np.uint32)
    cfg = _Config(int(d), int(k.size), off.ctypes.data_as(C.POINTER(C.c_uint64)), k.ctypes.data_as(C.POINTER(C.c_uint32)),
                  int(s), int(sparsifier), int(quantizer), 0, 1, int(flags))
    out = np.zeros(k.size, dtype=np.uint32)
    _check(_lib.qsl_plan_paths(C.byref(cfg), out.ctypes.data_as(C.POINTER(C.c_uint32))), "qsl_plan_paths")
    return out


def aggregate_static(d, k, s, sparsifier, quantizer, msg, out, scale, worker_list=None, accumulate=False):
    """`qsl_aggregate_static`: the master line without a context and without any allocation (one segment)."""
    off = np.array([0, int(d)], dtype=np.uint64)
    kk = np.array([int(k)], dtype=np.uint32)
    cfg = _Config(int(d), 1, off.ctypes.data_as(C.POINTER(C.c_uint64)), kk.ctypes.data_as(C.POINTER(C.c_uint32)),
                  int(s), int(sparsifier), int(quantizer), 0, 1, 0)
    if worker_list is None:
        R, lst = msg.shape[0], None
    else:
        lst = (C.c_uint32 * len(worker_list))(*[int(x) for x in worker_list])
        R = len(worker_list)
    stream = C.c_void_p(torch.cuda.current_stream(msg.device).cuda_stream)
    _check(_lib.qsl_aggregate_static(C.byref(cfg), stream, _ptr(msg, torch.uint8), lst, R, float(scale),
                                     int(bool(accumulate)), _ptr(out, torch.float32)), "qsl_aggregate_static")


def _rows_of(t, what):
    """Address and row stride of a [rows, vocab] tensor whose rows are contiguous."""
    if t.dim() != 2 or not t.is_cuda or t.dtype not in DTYPES:
        raise ValueError(f"{what}: expected a device tensor [rows, vocab] of float32, bfloat16 or float16")
    rows, vocab = t.shape
    if rows >= SIZE_END or vocab >= SIZE_END:                             # (ctypes would keep the lower 32 bits)
        raise ValueError(f"{what}: expected less than 2^31 rows and classes, got {list(t.shape)}")
    stride, step = t.stride()
    if (step != 1 and vocab != 1) or (rows > 1 and stride < vocab):
        raise ValueError(f"{what}: expected contiguous rows that do not overlap, got strides {t.stride()}")
    return t.data_ptr(), stride if rows > 1 else vocab


def _beside(t, what, device, dtype, shape):
    """Address of an argument that goes with logits on `device` (its index): there, contiguous, of that type and shape; None for None (which
    callers pass over for what is mostly not given: the call alone costs 40 ns)."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == shape and t.get_device() == device and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{what}: expected a contiguous {dtype} tensor {list(shape)} on cuda:{device}, got {t.dtype} {list(t.shape)} on {t.device}")


_current_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


def _on_logits(where, fn, logits, scale, top, workspace, *args, entries=False, kept=False):
    """Calls fn(rows, *args, workspace, its size, stream) on the logits' device and its current stream.  entries: `top` counts a teacher's
    entries, not alternatives; kept: the call has its statistics."""
    data, stride = _rows_of(logits, "logits")
    if top >= SIZE_END:
        raise ValueError(f"{where}: {top} alternatives or entries a row")
    rows, vocab = logits.shape
    z = C.byref(_Logits(data, stride, rows, vocab, DTYPES[logits.dtype], scale))
    if workspace is None and not kept:
        need = _lib.qsl_logits_workspace_bytes(z, 0 if entries else top)
        if need:
            if entries:
                need = _lib.qsl_logits_workspace_bytes(z, top)
            workspace = torch.empty(need, dtype=torch.uint8, device=logits.device)
    device = logits.get_device()
    at, size = (None, 0) if workspace is None else (_beside(workspace, "workspace", device, torch.uint8, (workspace.numel(),)), workspace.numel())
    if device == _current_device():
        st = fn(z, *args, at, size, _raw_stream(device))
    else:
        with torch.cuda.device(device):
            st = fn(z, *args, at, size, _raw_stream(device))
    if st != OK:
        raise QslError(st, where)


def logits_workspace_bytes(logits, top=0):
    """`qsl_logits_workspace_bytes` of these rows: what `workspace=` of the calls below has to hold (they allocate it if it is not given)."""
    data, stride = _rows_of(logits, "logits")
    if not 0 <= top < SIZE_END:
        return 0
    return int(_lib.qsl_logits_workspace_bytes(C.byref(_Logits(data, stride, logits.shape[0], logits.shape[1], DTYPES[logits.dtype], 1.0)), top))


def token_logprobs(logits, target=None, scale=1.0, logprob=None, entropy=None, lse=None, top_index=None, top_logprob=None,
                   stats=None, workspace=None):
    """`qsl_token_logprobs`: log probabilities of the given classes, entropy and best alternatives of every row of
    logits [rows, vocab], into those of the output tensors that are given."""
    N, dev = logits.shape[0], logits.get_device()
    some = top_index if top_index is not None else top_logprob
    top = 0 if some is None else some.shape[-1]
    f32 = torch.float32
    _on_logits("qsl_token_logprobs", _lib.qsl_token_logprobs, logits, scale, top, workspace, _beside(target, "target", dev, torch.int64, (N,)), top,
               _beside(logprob, "logprob", dev, f32, (N,)), None if entropy is None else _beside(entropy, "entropy", dev, f32, (N,)),
               None if lse is None else _beside(lse, "lse", dev, f32, (N,)), _beside(top_index, "top_index", dev, torch.int32, (N, top)),
               _beside(top_logprob, "top_logprob", dev, f32, (N, top)), None if stats is None else _beside(stats, "stats", dev, f32, (N, 4)))


def _gradient_rows(dlogits, logits):
    if dlogits.dtype is not logits.dtype or dlogits.shape != logits.shape or dlogits.get_device() != logits.get_device():
        raise ValueError("dlogits: expected the logits' type, shape and device")
    return _rows_of(dlogits, "dlogits")


def token_logprobs_backward(logits, target, dlogits, scale=1.0, grad_logprob=None, grad_entropy=None, stats=None, logprob=None,
                            entropy=None, workspace=None):
    """`qsl_token_logprobs_backward`: the gradient of sum(grad_logprob * logprob) + sum(grad_entropy * entropy) in the logits."""
    N, dev = logits.shape[0], logits.get_device()
    f32 = torch.float32
    out, dstride = _gradient_rows(dlogits, logits)
    _on_logits("qsl_token_logprobs_backward", _lib.qsl_token_logprobs_backward, logits, scale, 0, workspace,
               _beside(target, "target", dev, torch.int64, (N,)), _beside(grad_logprob, "grad_logprob", dev, f32, (N,)),
               None if grad_entropy is None else _beside(grad_entropy, "grad_entropy", dev, f32, (N,)),
               None if stats is None else _beside(stats, "stats", dev, f32, (N, 4)), _beside(logprob, "logprob", dev, f32, (N,)),
               None if entropy is None else _beside(entropy, "entropy", dev, f32, (N,)), out, dstride,
               kept=stats is not None)


def _teacher(logits, index, value, lse, scale):
    N, dev, top = logits.shape[0], logits.get_device(), index.shape[-1]
    return C.byref(_Teacher(_beside(index, "teacher_index", dev, torch.int32, (N, top)),
                            _beside(value, "teacher_value", dev, torch.float32, (N, top)),
                            None if lse is None else _beside(lse, "teacher_lse", dev, torch.float32, (N,)), top, scale))


def distill(logits, teacher_index, teacher_value, scale=1.0, teacher_scale=1.0, teacher_lse=None, loss=None, stats=None, workspace=None):
    """`qsl_distill`: the Kullback-Leibler divergence of every row from a teacher's top logits [rows, top]."""
    N, dev = logits.shape[0], logits.get_device()
    _on_logits("qsl_distill", _lib.qsl_distill, logits, scale, teacher_index.shape[-1], workspace,
               _teacher(logits, teacher_index, teacher_value, teacher_lse, teacher_scale), _beside(loss, "loss", dev, torch.float32, (N,)),
               None if stats is None else _beside(stats, "stats", dev, torch.float32, (N, 8)), entries=True)


def distill_backward(logits, teacher_index, teacher_value, dlogits, scale=1.0, teacher_scale=1.0, teacher_lse=None, grad_loss=None,
                     stats=None, loss=None, workspace=None):
    """`qsl_distill_backward`: the gradient of sum(grad_loss * loss) in the logits."""
    N, dev = logits.shape[0], logits.get_device()
    f32 = torch.float32
    out, dstride = _gradient_rows(dlogits, logits)
    _on_logits("qsl_distill_backward", _lib.qsl_distill_backward, logits, scale, teacher_index.shape[-1], workspace,
               _teacher(logits, teacher_index, teacher_value, teacher_lse, teacher_scale), _beside(grad_loss, "grad_loss", dev, f32, (N,)),
               None if stats is None else _beside(stats, "stats", dev, f32, (N, 8)), _beside(loss, "loss", dev, f32, (N,)), out, dstride,
               entries=True)


class Qsl:
    """One operator Q Comp_k (a `qsl_ctx`).  Methods mirror the C entry points one to one."""

    def __init__(self, d, seg_offset, seg_k, s, sparsifier, quantizer, seed, max_workers, flags=0, device=None):
        self.device = torch.device("cuda" if device is None else device)
        self._off = np.ascontiguousarray(seg_offset, dtype=np.uint64)
        self._k = np.ascontiguousarray(seg_k, dtype=np.uint32)
        self.d, self.L, self.K = int(d), int(self._k.size), int(self._k.sum())
        self.s, self.sparsifier, self.quantizer, self.seed = int(s), int(sparsifier), int(quantizer), int(seed)
        self.max_workers = int(max_workers)
        cfg = _Config(self.d, self.L, self._off.ctypes.data_as(C.POINTER(C.c_uint64)),
                      self._k.ctypes.data_as(C.POINTER(C.c_uint32)), self.s, self.sparsifier, self.quantizer,
                      self.seed, self.max_workers, int(flags))
        self._ctx = C.c_void_p()
        with torch.cuda.device(self.device):
            _check(_lib.qsl_create(C.byref(self._ctx), C.byref(cfg), self._stream()), "qsl_create")
        self.capacity = int(_lib.qsl_msg_capacity_bytes(self._ctx))

    def _stream(self):
        return C.c_void_p(torch.cuda.current_stream(self.device).cuda_stream)

    def close(self):
        if getattr(self, "_ctx", None) is not None and self._ctx.value:
            _lib.qsl_destroy(self._ctx)
            self._ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- allocation helpers (plumbing, not part of the C ABI) ---------------------------------
    def new_msg(self, R):
        return torch.empty(R, self.capacity, dtype=torch.uint8, device=self.device)

    # -- the C entry points -------------------------------------------------------------------
    def compress(self, m, delta, m_out, worker0, rnd, msg, msg_bits=None, sel_idx=None, sel_level=None):
        R = m.shape[0]
        assert m.shape == (R, self.d) and delta.shape == m.shape and (m_out is None or m_out.shape == m.shape)
        assert msg.shape == (R, self.capacity)
        _check(_lib.qsl_set_stream(self._ctx, self._stream()), "qsl_set_stream")
        _check(_lib.qsl_compress(self._ctx, _ptr(m, torch.float32), _ptr(delta, torch.float32),
                                 _ptr(m_out, torch.float32, True), int(worker0), R, int(rnd), _ptr(msg, torch.uint8),
                                 _ptr(msg_bits, torch.int64, True), _ptr(sel_idx, torch.int32, True),
                                 _ptr(sel_level, torch.int16, True)), "qsl_compress")

    def compress_diff(self, m, x, xhat_half, m_out, worker0, rnd, msg, msg_bits=None, sel_idx=None, sel_level=None):
        R = m.shape[0]
        assert m.shape == (R, self.d) and xhat_half.shape == m.shape and x.shape == (self.d,)
        assert m_out is None or m_out.shape == m.shape
        assert msg.shape == (R, self.capacity)
        _check(_lib.qsl_set_stream(self._ctx, self._stream()), "qsl_set_stream")
        _check(_lib.qsl_compress_diff(self._ctx, _ptr(m, torch.float32), _ptr(x, torch.float32),
                                      _ptr(xhat_half, torch.float32), _ptr(m_out, torch.float32, True), int(worker0), R,
                                      int(rnd), _ptr(msg, torch.uint8), _ptr(msg_bits, torch.int64, True),
                                      _ptr(sel_idx, torch.int32, True), _ptr(sel_level, torch.int16, True)),
               "qsl_compress_diff")

    def error_update(self, m, delta, msg):
        R = m.shape[0]
        assert m.shape == (R, self.d) and delta.shape == m.shape and msg.shape == (R, self.capacity)
        _check(_lib.qsl_set_stream(self._ctx, self._stream()), "qsl_set_stream")
        _check(_lib.qsl_error_update(self._ctx, _ptr(m, torch.float32), _ptr(delta, torch.float32),
                                     _ptr(msg, torch.uint8), R), "qsl_error_update")

    def aggregate(self, msg, out, scale, worker_list=None, accumulate=False):
        assert msg.shape[1] == self.capacity and out.shape == (self.d,)
        if worker_list is None:
            R, lst = msg.shape[0], None
        else:
            arr = (C.c_uint32 * len(worker_list))(*[int(x) for x in worker_list])
            R, lst = len(worker_list), arr
            assert max(worker_list) < msg.shape[0]
        _check(_lib.qsl_set_stream(self._ctx, self._stream()), "qsl_set_stream")
        _check(_lib.qsl_aggregate(self._ctx, _ptr(msg, torch.uint8), lst, R, float(scale), int(bool(accumulate)),
                                  _ptr(out, torch.float32)), "qsl_aggregate")

    def bits_sent(self, msg):
        R = msg.shape[0]
        out = (C.c_uint64 * R)()
        _check(_lib.qsl_set_stream(self._ctx, self._stream()), "qsl_set_stream")
        _check(_lib.qsl_bits_sent(self._ctx, _ptr(msg, torch.uint8), R, out), "qsl_bits_sent")
        return [int(x) for x in out]

    def device_status(self):
        return int(_lib.qsl_device_status(self._ctx))

    def debug_units(self):
        n = C.c_uint32()
        cap = self.max_workers * self.L
        buf = (C.c_uint32 * (8 * cap))()
        _check(_lib.qsl_debug_units(self._ctx, buf, cap, C.byref(n)), "qsl_debug_units")
        a = np.ctypeslib.as_array(buf).reshape(cap, 8)[: n.value].copy()
        return a

    def timing_enable(self, on=True):
        _check(_lib.qsl_timing_enable(self._ctx, int(on)), "qsl_timing_enable")

    def timing_read(self):
        ms, n = C.c_double(), C.c_uint32()
        _check(_lib.qsl_timing_read(self._ctx, C.byref(ms), C.byref(n)), "qsl_timing_read")
        return ms.value, n.value


def from_workload(wl, max_workers=None, flags=0, device=None) -> Qsl:
    if getattr(wl, "dense", False):
        flags |= FLAG_DENSE_FORMAT
    return Qsl(wl.d, wl.seg_offset, wl.seg_k, wl.s, wl.sparsifier, wl.quantizer, wl.seed,
               max_workers or wl.R, flags=flags, device=device)
