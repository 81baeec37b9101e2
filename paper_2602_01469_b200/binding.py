"""ctypes binding of libpeagle.so: argument marshalling only.

Every function here has the name and argument order of its C entry point in ``include/peagle.h``
and forwards device pointers of torch tensors (torch is used for device memory and streams,
nothing else).  There is no fallback: if the shared library is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import os
from bisect import bisect_left

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpeagle.so")

PEAGLE_OK = 0
STATUS = {
    "OK": 0, "NULL": -1, "BAD_SHAPE": -2, "BAD_RANGE": -3, "BAD_META": -4, "UNSUPPORTED_ARCH": -5,
    "WORKSPACE": -6, "TIMEOUT": -7, "TOO_LARGE": -8, "CUDA": -9, "ALIGN": -10,
}

EXPORTS = [
    "peagle_create", "peagle_destroy", "peagle_status_string", "peagle_last_cuda_error",
    "peagle_tile_shape", "peagle_poll_status", "peagle_launch_count", "peagle_attn_fwd",
    "peagle_attn_bwd", "peagle_attn_partitioned", "peagle_attn_partitioned_host",
    "peagle_assign_segments", "peagle_classify_tiles", "peagle_mask_dense",
    "peagle_timing_enable", "peagle_timing_read", "peagle_attn_fwd_static",
    "peagle_rope_qkv_fwd", "peagle_rope_qkv_bwd", "peagle_attn_partitioned_acc", "peagle_cast_grads",
    "peagle_gemm_bf16", "peagle_layer_partitioned", "peagle_selftest_wait_expiry",
    "peagle_norm_fwd", "peagle_norm_bwd", "peagle_token_logprobs_fwd", "peagle_token_logprobs_bwd",
    "peagle_adamw_step",
]

NORM = {"layer": 0, "rms": 1}  # peagle_norm


class peagle_range_t(ctypes.Structure):
    _fields_ = [("begin", ctypes.c_int32), ("end", ctypes.c_int32)]


class peagle_problem_t(ctypes.Structure):
    _fields_ = [
        ("num_seqs", ctypes.c_int32),
        ("cu_seqlens", ctypes.POINTER(ctypes.c_int32)),
        ("total_tokens", ctypes.c_int32),
        ("anchor", ctypes.c_void_p),
        ("depth", ctypes.c_void_p),
        ("K", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float),
    ]


class peagle_partition_t(ctypes.Structure):
    _fields_ = [
        ("seq", ctypes.c_int32),
        ("q", peagle_range_t),
        ("k", ctypes.POINTER(peagle_range_t)),
        ("nk", ctypes.c_int32),
    ]


class peagle_adamw_tensor_t(ctypes.Structure):
    _fields_ = [
        ("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("master", ctypes.c_void_p),
        ("m", ctypes.c_void_p), ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
        ("count", ctypes.c_int64), ("param_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32),
        ("weight_decay", ctypes.c_float),
    ]


class peagle_adamw_t(ctypes.Structure):
    _fields_ = [
        ("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
        ("step", ctypes.c_int64), ("lr_dev", ctypes.c_void_p), ("step_dev", ctypes.c_void_p),
        ("grad_scale_dev", ctypes.c_void_p), ("seed", ctypes.c_uint32),
    ]


def _argtypes(letters):
    """p: pointer, i: int32, l: int64, f: float."""
    kinds = {"p": ctypes.c_void_p, "i": ctypes.c_int32, "l": ctypes.c_int64, "f": ctypes.c_float}
    return [kinds[c] for c in letters]


# Entry points that short calls go through: with their types known, ctypes takes plain numbers.
_ARGTYPES = {
    "peagle_norm_fwd": _argtypes("piiiiiplppfplppp"),
    "peagle_norm_bwd": _argtypes("piiiiiplpppplplppp"),
    "peagle_token_logprobs_fwd": _argtypes("piiiplpfpppippp"),
    "peagle_token_logprobs_bwd": _argtypes("piiiplpfpppppl") + [ctypes.c_void_p],
    "peagle_adamw_step": _argtypes("pppip"),
}

_lib = None


def lib():
    """Loads libpeagle.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                               "(there is no CPU or PyTorch fallback)")
        L = ctypes.CDLL(LIB_PATH)
        L.peagle_status_string.restype = ctypes.c_char_p
        L.peagle_last_cuda_error.restype = ctypes.c_char_p
        L.peagle_last_cuda_error.argtypes = [ctypes.c_void_p]
        L.peagle_launch_count.restype = ctypes.c_int64
        L.peagle_launch_count.argtypes = [ctypes.c_void_p]
        for name, types in _ARGTYPES.items():
            getattr(L, name).argtypes = types
        _lib = L
    return _lib


class PeagleError(RuntimeError):
    def __init__(self, status: int, ctx=None):
        self.status = status
        msg = lib().peagle_status_string(status).decode()
        if ctx is not None and status == STATUS["CUDA"]:
            msg += ": " + lib().peagle_last_cuda_error(ctx).decode()
        super().__init__(f"peagle status {status}: {msg}")


def _check(rc: int, ctx=None):
    if rc != PEAGLE_OK:
        raise PeagleError(rc, ctx)


def _ptr(t):
    """Device (or host) address of a torch tensor / numpy array / None."""
    if t is None:
        return ctypes.c_void_p(0)
    if isinstance(t, np.ndarray):
        return ctypes.c_void_p(t.ctypes.data)
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        import torch
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    if hasattr(stream, "cuda_stream"):
        return ctypes.c_void_p(stream.cuda_stream)
    return ctypes.c_void_p(int(stream))


# ---- arguments of the operators around the layer.  Their calls can be as short as a few microseconds on the GPU, so
# the checks ask a tensor as little as they can.

def _current_stream(device):
    import torch
    return torch.cuda.current_stream(device).cuda_stream


def _know_torch():
    global _current_stream
    import torch
    # the same without the Python object around the handle, 0.1 instead of 1.3 us, where torch has it
    _current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _current_stream)
    _dtypes.update({torch.float32: 0, torch.bfloat16: 1})
    _f32[:], _i32[:], _i64[:] = [torch.float32], [torch.int32], [torch.int64]


def _refuse(status="BAD_SHAPE"):
    raise PeagleError(STATUS[status])


def _stream_on(ctx, stream):
    """The stream's handle; without one, the current stream of the context's own device."""
    if stream is None:
        return _current_stream(ctx.device)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


_dtypes = {}                       # peagle_dtype by torch dtype
_f32, _i32, _i64 = [], [], []      # the torch dtypes of vectors; filled, like _dtypes, when torch is there


def _dtype(t):
    """peagle_dtype of a tensor."""
    code = _dtypes.get(t.dtype)
    return code if code is not None else _refuse()


def _matrix(t, rows, cols, dtype, device):
    """Address and leading dimension of a [rows, cols] tensor on the context's device whose rows are contiguous."""
    if t.shape != (rows, cols) or t.dtype != dtype or t.get_device() != device:
        _refuse()
    ld, inner = t.stride()
    if inner != 1 and cols > 1 and rows:
        _refuse()
    return t.data_ptr(), ld if rows > 1 else max(ld, cols)


def _vector(t, n, dtypes, device):
    """Address of a contiguous vector of n elements, None of none."""
    if t is None:
        return None
    if t.shape != (n,) or t.dtype not in dtypes or t.get_device() != device or not t.is_contiguous():
        _refuse()
    return t.data_ptr()


class Problem:
    """Owns the host arrays a peagle_problem_t points to."""

    def __init__(self, cu_seqlens, anchor, depth, K, n_q_heads, n_kv_heads, head_dim,
                 softmax_scale):
        self.cu = np.ascontiguousarray(np.asarray(cu_seqlens, dtype=np.int32))
        self.anchor, self.depth = anchor, depth          # device tensors (host arrays for *_host)
        self.c = peagle_problem_t(
            len(self.cu) - 1, self.cu.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
            int(self.cu[-1]) if len(self.cu) else 0, _ptr(anchor), _ptr(depth), int(K),
            int(n_q_heads), int(n_kv_heads), int(head_dim), float(softmax_scale))

    def ref(self):
        return ctypes.byref(self.c)


class Partition:
    """Owns the host range array a peagle_partition_t points to."""

    def __init__(self, seq, q, k=None):
        k = [] if k is None else list(k)
        self.kr = (peagle_range_t * max(len(k), 1))(*[peagle_range_t(int(b), int(e)) for b, e in k])
        self.c = peagle_partition_t(int(seq), peagle_range_t(int(q[0]), int(q[1])),
                                    ctypes.cast(self.kr, ctypes.POINTER(peagle_range_t)) if k else None,
                                    len(k))

    def ref(self):
        return ctypes.byref(self.c)


def _partition_array(parts):
    arr = (peagle_partition_t * max(len(parts), 1))()
    for i, p in enumerate(parts):
        arr[i] = p.c
    return arr


ADAMW_BLOCK = 256  # elements that share a scale where states are held in 8 bits


class AdamWTensors:
    """The tensors of ``peagle_adamw_step``, put together once: owns the array a call passes and keeps the tensors
    alive.  Each item is a dict of ``param``, ``grad``, ``m``, ``v`` and, where they apply, ``master`` (fp32, for bf16
    parameters), ``m_scale`` and ``v_scale`` (states in 8 bits: m and v are float8_e4m3fn, a scale for every
    ADAMW_BLOCK elements), ``weight_decay``.  Contiguous device tensors; no two may share memory, but for gradients
    among themselves."""

    def __init__(self, items):
        import torch
        _know_torch()
        self.items = [dict(i) for i in items]
        self.device = self.items[0]["param"].device.index if self.items else None
        self.c = (peagle_adamw_tensor_t * max(len(self.items), 1))()
        written = []
        f32, codes, dev = torch.float32, torch.float8_e4m3fn, self.device

        def own(t, dtype, size, count):
            if t is None or t.dtype != dtype or t.get_device() != dev or t.numel() != count or not t.is_contiguous():
                _refuse()
            at = t.data_ptr()
            if count:
                written.append((at, at + size * count))
            return at

        for c, i in zip(self.c, self.items):
            p, get = i["param"], i.get
            n, code, master, m_scale, v_scale = p.numel(), _dtype(p), get("master"), get("m_scale"), get("v_scale")
            if m_scale is None and v_scale is None:
                c.m, c.v = own(get("m"), f32, 4, n), own(get("v"), f32, 4, n)
            elif m_scale is None or v_scale is None:
                _refuse()
            else:
                blocks = -(-n // ADAMW_BLOCK)
                c.m, c.v = own(get("m"), codes, 1, n), own(get("v"), codes, 1, n)
                c.m_scale, c.v_scale = own(m_scale, f32, 4, blocks), own(v_scale, f32, 4, blocks)
            if master is not None:
                c.master = own(master, f32, 4, n)
            c.param, c.count, c.param_dtype = own(p, p.dtype, 2 if code else 4, n), n, code
            c.weight_decay = float(get("weight_decay", 0.0))
        written.sort()
        if any(end > begin for (_, end), (begin, _) in zip(written, written[1:])):
            _refuse("BAD_RANGE")
        self._begins, self._ends = [begin for begin, _ in written], [end for _, end in written]
        self.set_grads([i["grad"] for i in self.items])

    def set_grads(self, grads):
        """Other gradients for the steps to come, in the order of the tensors.  All of them are taken, or none."""
        grads = list(grads)
        if len(grads) != len(self.items):
            _refuse()
        fresh = []
        for c, g in zip(self.c, grads):
            if g.get_device() != self.device or g.numel() != c.count or not g.is_contiguous():
                _refuse()
            at, code = g.data_ptr(), _dtype(g)
            before = bisect_left(self._begins, at + (2 if code else 4) * c.count) - 1
            if c.count and before >= 0 and self._ends[before] > at:
                _refuse("BAD_RANGE")
            fresh.append((at, code))
        for c, i, g, (at, code) in zip(self.c, self.items, grads, fresh):
            c.grad, c.grad_dtype, i["grad"] = at, code, g


class Context:
    def __init__(self, device: int = 0):
        self.h = ctypes.c_void_p()
        self.device = int(device)
        _know_torch()
        _check(lib().peagle_create(ctypes.byref(self.h), int(device)))

    def close(self):
        if self.h:
            lib().peagle_destroy(self.h)
            self.h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def peagle_tile_shape(ctx: Context, head_dim: int):
    bm, bn = ctypes.c_int(), ctypes.c_int()
    _check(lib().peagle_tile_shape(ctx.h, int(head_dim), ctypes.byref(bm), ctypes.byref(bn)))
    return bm.value, bn.value


def peagle_poll_status(ctx: Context, stream=None) -> int:
    return int(lib().peagle_poll_status(ctx.h, _stream(stream)))


def peagle_launch_count(ctx: Context) -> int:
    return int(lib().peagle_launch_count(ctx.h))


def peagle_timing_enable(ctx: Context, on: bool):
    _check(lib().peagle_timing_enable(ctx.h, int(bool(on))))


def peagle_timing_read(ctx: Context):
    """((forward ms, backward ms), (forward launches, backward launches)) since the last read."""
    ms = (ctypes.c_double * 2)()
    n = (ctypes.c_int64 * 2)()
    _check(lib().peagle_timing_read(ctx.h, ms, n), ctx.h)
    return (ms[0], ms[1]), (n[0], n[1])


def peagle_attn_fwd(ctx, prob: Problem, part: Partition, Q, K, V, O, LSE, stream=None):
    _check(lib().peagle_attn_fwd(ctx.h, prob.ref(), part.ref(), _ptr(Q), _ptr(K), _ptr(V), _ptr(O),
                                 _ptr(LSE), _stream(stream)), ctx.h)


def peagle_attn_fwd_static(device: int, prob: Problem, part: Partition, Q, K, V, O, LSE,
                           dev_status=None, stream=None):
    """Forward without any device allocation: the call's tile plan lives in a fixed array inside
    the library (4 MiB per GPU), so no context is needed.  ``dev_status`` is an optional int32
    device tensor that receives a device-side error code."""
    _check(lib().peagle_attn_fwd_static(int(device), prob.ref(), part.ref(), _ptr(Q), _ptr(K),
                                        _ptr(V), _ptr(O), _ptr(LSE), _ptr(dev_status),
                                        _stream(stream)))


def peagle_attn_bwd(ctx, prob: Problem, part: Partition, Q, K, V, O, dO, LSE, dQ, dK_acc, dV_acc,
                    stream=None):
    _check(lib().peagle_attn_bwd(ctx.h, prob.ref(), part.ref(), _ptr(Q), _ptr(K), _ptr(V), _ptr(O),
                                 _ptr(dO), _ptr(LSE), _ptr(dQ), _ptr(dK_acc), _ptr(dV_acc),
                                 _stream(stream)), ctx.h)


def peagle_attn_partitioned(ctx, prob: Problem, parts, Q, K, V, dO, O, LSE, dQ, dK, dV, stream=None):
    arr = _partition_array(parts)
    _check(lib().peagle_attn_partitioned(ctx.h, prob.ref(), arr, len(parts), _ptr(Q), _ptr(K),
                                         _ptr(V), _ptr(dO), _ptr(O), _ptr(LSE), _ptr(dQ), _ptr(dK),
                                         _ptr(dV), _stream(stream)), ctx.h)


def peagle_attn_partitioned_acc(ctx, prob: Problem, parts, Q, K, V, dO, O, LSE, dQ, dK_acc, dV_acc,
                                stream=None):
    """Forward + backward of ``parts`` adding into the caller's fp32 dK / dV accumulators."""
    arr = _partition_array(parts)
    _check(lib().peagle_attn_partitioned_acc(ctx.h, prob.ref(), arr, len(parts), _ptr(Q), _ptr(K),
                                             _ptr(V), _ptr(dO), _ptr(O), _ptr(LSE), _ptr(dQ),
                                             _ptr(dK_acc), _ptr(dV_acc), _stream(stream)), ctx.h)


def peagle_cast_grads(ctx, dK_acc, dV_acc, dK, dV, stream=None):
    """Rounds fp32 dK / dV sums to bf16."""
    _check(lib().peagle_cast_grads(ctx.h, _ptr(dK_acc), _ptr(dV_acc), ctypes.c_int64(dK_acc.numel()),
                                   _ptr(dK), _ptr(dV), _stream(stream)), ctx.h)


def peagle_attn_partitioned_host(ctx, prob: Problem, parts, Q, K, V, dO, O, LSE, dQ, dK, dV):
    """All tensors (and prob.anchor / prob.depth) are HOST memory here."""
    arr = _partition_array(parts)
    _check(lib().peagle_attn_partitioned_host(ctx.h, prob.ref(), arr, len(parts), _ptr(Q), _ptr(K),
                                              _ptr(V), _ptr(dO), _ptr(O), _ptr(LSE), _ptr(dQ),
                                              _ptr(dK), _ptr(dV)), ctx.h)


def peagle_rope_qkv_fwd(ctx, qkv, anchor, depth, Hq, Hkv, D, rope_base, Q, K, V, stream=None):
    """Rotary prologue: fused rows [T, (Hq + 2 Hkv) * D] -> Q, K (rotated), V (copied); device tensors."""
    _check(lib().peagle_rope_qkv_fwd(ctx.h, _ptr(qkv), _ptr(anchor), _ptr(depth),
                                     int(qkv.shape[0]), int(Hq), int(Hkv), int(D),
                                     ctypes.c_float(rope_base), _ptr(Q), _ptr(K), _ptr(V),
                                     _stream(stream)), ctx.h)


def peagle_rope_qkv_bwd(ctx, dQ, dK, dV, anchor, depth, Hq, Hkv, D, rope_base, d_qkv, stream=None):
    """Backward of the rotary prologue: dQ, dK, dV -> gradient of the fused rows; device tensors."""
    _check(lib().peagle_rope_qkv_bwd(ctx.h, _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(anchor), _ptr(depth),
                                     int(dQ.shape[0]), int(Hq), int(Hkv), int(D),
                                     ctypes.c_float(rope_base), _ptr(d_qkv), _stream(stream)), ctx.h)


def peagle_gemm_bf16(ctx, A, lda, a_t, B, ldb, b_t, C, ldc, c_f32_add, M, N, K, stream=None):
    """C[m][n] (+)= sum_k A(m,k) B(n,k); see include/peagle.h for the layouts."""
    _check(lib().peagle_gemm_bf16(ctx.h, _ptr(A), ctypes.c_int64(lda), int(a_t), _ptr(B),
                                  ctypes.c_int64(ldb), int(b_t), _ptr(C), ctypes.c_int64(ldc),
                                  int(c_f32_add), int(M), int(N), int(K), _stream(stream)), ctx.h)


def peagle_layer_partitioned(ctx, prob: Problem, parts, X, W, rope_base, dO, O, LSE, dX, dW, stream=None):
    """Projection -> rotary -> attention forward and backward, one pass per segment (device tensors)."""
    arr = _partition_array(parts)
    _check(lib().peagle_layer_partitioned(ctx.h, prob.ref(), arr, len(parts), _ptr(X), _ptr(W),
                                          int(X.shape[1]), ctypes.c_float(rope_base), _ptr(dO), _ptr(O),
                                          _ptr(LSE), _ptr(dX), _ptr(dW), _stream(stream)), ctx.h)


def peagle_norm_fwd(ctx, kind, X, weight, bias, eps, Y, mean=None, rstd=None, stream=None):
    """Layer norm (``NORM["layer"]``) or RMS norm (``NORM["rms"]``) of the rows of X into Y; weight, bias, and
    the fp32 statistics mean and rstd may be None.  Device tensors; rows of X and Y may lie apart."""
    if X.dim() != 2:
        _refuse()
    rows, cols = X.shape
    if (rows | cols) >> 31:  # the ABI's int32 would cut it off
        _refuse("TOO_LARGE")
    dtype, dev = _dtype(X), ctx.device
    w = weight if weight is not None else bias
    w_dtype = _dtype(w) if w is not None else 0
    if bias is not None and bias.dtype != w.dtype:
        _refuse()
    x, ldx = _matrix(X, rows, cols, X.dtype, dev)
    y, ldy = _matrix(Y, rows, cols, X.dtype, dev)
    rc = lib().peagle_norm_fwd(ctx.h, kind, dtype, w_dtype, rows, cols, x, ldx, _vector(weight, cols, _dtypes, dev),
                               _vector(bias, cols, _dtypes, dev), eps, y, ldy, _vector(mean, rows, _f32, dev),
                               _vector(rstd, rows, _f32, dev), _stream_on(ctx, stream))
    if rc:
        _check(rc, ctx.h)


def peagle_norm_bwd(ctx, kind, X, weight, mean, rstd, dY, dX, dweight_acc=None, dbias_acc=None, stream=None):
    """Backward of the norm: dX, and the gradients of weight and bias ADDED to fp32 sums."""
    if X.dim() != 2:
        _refuse()
    rows, cols = X.shape
    if (rows | cols) >> 31:  # the ABI's int32 would cut it off
        _refuse("TOO_LARGE")
    dtype, dev = _dtype(X), ctx.device
    w_dtype = _dtype(weight) if weight is not None else 0
    x, ldx = _matrix(X, rows, cols, X.dtype, dev)
    dy, lddy = _matrix(dY, rows, cols, X.dtype, dev)
    dx, lddx = _matrix(dX, rows, cols, X.dtype, dev)
    rc = lib().peagle_norm_bwd(ctx.h, kind, dtype, w_dtype, rows, cols, x, ldx, _vector(weight, cols, _dtypes, dev),
                               _vector(mean, rows, _f32, dev), _vector(rstd, rows, _f32, dev), dy, lddy, dx, lddx,
                               _vector(dweight_acc, cols, _f32, dev), _vector(dbias_acc, cols, _f32, dev),
                               _stream_on(ctx, stream))
    if rc:
        _check(rc, ctx.h)


def peagle_token_logprobs_fwd(ctx, logits, tokens, scale=1.0, logprob=None, lse=None, entropy=None, top_logprobs=None,
                              top_ids=None, stream=None):
    """Log probability of ``tokens`` (int32, -1 for none) under the rows of ``logits``, with log-sum-exp, entropy
    and the top alternatives; every output may be None.  The width of the top outputs says how many."""
    if logits.dim() != 2 or (top_logprobs is None) != (top_ids is None):
        _refuse()
    rows, vocab = logits.shape
    if (rows | vocab) >> 31:
        _refuse("TOO_LARGE")
    dtype, dev = _dtype(logits), ctx.device
    x, ld = _matrix(logits, rows, vocab, logits.dtype, dev)
    k, top, ids = 0, None, None
    if top_ids is not None:
        if top_ids.dim() != 2 or not top_ids.is_contiguous() or not top_logprobs.is_contiguous():
            _refuse()
        k = top_ids.size(1)
        if k >> 31:
            _refuse("TOO_LARGE")
        top = _matrix(top_logprobs, rows, k, _f32[0], dev)[0]
        ids = _matrix(top_ids, rows, k, _i32[0], dev)[0]
    rc = lib().peagle_token_logprobs_fwd(ctx.h, dtype, rows, vocab, x, ld, _vector(tokens, rows, _i32, dev), scale,
                                         _vector(logprob, rows, _f32, dev), _vector(lse, rows, _f32, dev),
                                         _vector(entropy, rows, _f32, dev), k, top, ids, _stream_on(ctx, stream))
    if rc:
        _check(rc, ctx.h)


def peagle_token_logprobs_bwd(ctx, logits, tokens, scale, lse, entropy, g_logprob, g_entropy, dlogits, stream=None):
    """Gradient of the logits from those of logprob and entropy (either may be None); ``dlogits`` may be ``logits``."""
    if logits.dim() != 2:
        _refuse()
    rows, vocab = logits.shape
    if (rows | vocab) >> 31:
        _refuse("TOO_LARGE")
    dtype, dev = _dtype(logits), ctx.device
    x, ld = _matrix(logits, rows, vocab, logits.dtype, dev)
    d, ldd = _matrix(dlogits, rows, vocab, logits.dtype, dev)
    rc = lib().peagle_token_logprobs_bwd(ctx.h, dtype, rows, vocab, x, ld, _vector(tokens, rows, _i32, dev), scale,
                                         _vector(lse, rows, _f32, dev), _vector(entropy, rows, _f32, dev),
                                         _vector(g_logprob, rows, _f32, dev), _vector(g_entropy, rows, _f32, dev), d, ldd,
                                         _stream_on(ctx, stream))
    if rc:
        _check(rc, ctx.h)


def peagle_adamw_step(ctx, tensors: AdamWTensors, lr, beta1, beta2, eps, step=1, seed=0, lr_dev=None, step_dev=None,
                      grad_scale=None, stream=None):
    """One AdamW step over ``tensors``, in place.  ``lr_dev`` (fp32), ``step_dev`` (int64) and ``grad_scale`` (fp32) are
    device tensors of shape [1] that replace lr, step and the gradients' factor 1."""
    dev = ctx.device
    if tensors.device is not None and tensors.device != dev:
        _refuse()
    how = peagle_adamw_t(lr, beta1, beta2, eps, step, _vector(lr_dev, 1, _f32, dev), _vector(step_dev, 1, _i64, dev),
                         _vector(grad_scale, 1, _f32, dev), seed & 0xFFFFFFFF)
    rc = lib().peagle_adamw_step(ctx.h, ctypes.addressof(how), ctypes.addressof(tensors.c), len(tensors.items),
                                 _stream_on(ctx, stream))
    if rc:
        _check(rc, ctx.h)


def peagle_selftest_wait_expiry(ctx, limit_ms: int = 20, stream=None):
    """Runs one bounded wait into its time limit; poll_status then reports TIMEOUT once."""
    _check(lib().peagle_selftest_wait_expiry(ctx.h, int(limit_ms), _stream(stream)), ctx.h)


def peagle_assign_segments(anchor, depth, K, boundaries):
    """Algorithm 1 on the host (no GPU needed): segment index of every token of one sequence."""
    anchor = np.ascontiguousarray(np.asarray(anchor, dtype=np.int32))
    depth = np.ascontiguousarray(np.asarray(depth, dtype=np.int32))
    b = np.ascontiguousarray(np.asarray(boundaries, dtype=np.int32))
    out = np.zeros(anchor.shape[0], np.int32)
    i32p = ctypes.POINTER(ctypes.c_int32)
    _check(lib().peagle_assign_segments(anchor.ctypes.data_as(i32p), depth.ctypes.data_as(i32p),
                                        int(anchor.shape[0]), int(K), b.ctypes.data_as(i32p),
                                        int(b.shape[0] - 1), out.ctypes.data_as(i32p)))
    return out


def peagle_classify_tiles(ctx, prob: Problem, part: Partition):
    nq, nk = ctypes.c_int32(), ctypes.c_int32()
    _check(lib().peagle_classify_tiles(ctx.h, prob.ref(), part.ref(), None, ctypes.byref(nq),
                                       ctypes.byref(nk)), ctx.h)
    out = np.zeros((nq.value, nk.value), np.uint8)
    _check(lib().peagle_classify_tiles(ctx.h, prob.ref(), part.ref(), _ptr(out), ctypes.byref(nq),
                                       ctypes.byref(nk)), ctx.h)
    return out


def peagle_mask_dense(ctx, prob: Problem, part: Partition):
    q_len = part.c.q.end - part.c.q.begin
    out = np.zeros((q_len, prob.c.total_tokens), np.uint8)
    _check(lib().peagle_mask_dense(ctx.h, prob.ref(), part.ref(), _ptr(out)), ctx.h)
    return out
