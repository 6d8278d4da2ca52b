"""ctypes binding of the BMLP C-ABI (include/bmlp.h).

Argument marshalling only: every step of training and evaluation runs in the
CUDA kernels of ``libbmlp.so``.  There is no fallback: if the library or a GB300
is missing, the calls raise.

Buffers may be torch tensors (CUDA or CPU) or numpy arrays; CPU/numpy buffers
are host pointers, which the library stages through its own device buffers.
``stream`` is a ``torch.cuda.Stream``, a raw ``cudaStream_t`` integer, or None
(torch's current stream when torch CUDA is initialised, else the legacy
default stream).
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
import sys
import threading

import numpy as np

from . import _build

BMLP_OK = 0
BMLP_EINVAL = -1
BMLP_ENOMEM = -2
BMLP_ECUDA = -3
BMLP_ETIMEOUT = -4
BMLP_ESTATE = -5
BMLP_ENODEV = -6
BMLP_EPOCH_END = 1
BMLP_FWD_AUTO, BMLP_FWD_POPC, BMLP_FWD_TCGEN05, BMLP_FWD_B1MMA, BMLP_FWD_S8MMA = 0, 1, 2, 3, 4
BMLP_GROUPS_CONTIGUOUS, BMLP_GROUPS_FIXED, BMLP_GROUPS_RESHUFFLED = 0, 1, 2
BMLP_F32, BMLP_F16, BMLP_BF16, BMLP_I32 = 0, 1, 2, 3
BMLP_INT8_MAX_K = 131071
PROFILE_KINDS = ("train_forward", "cls_select", "update", "eval_forward", "eval_out", "copy",
                 "r_events")

_ERRNAMES = {-1: "EINVAL", -2: "ENOMEM", -3: "ECUDA", -4: "ETIMEOUT", -5: "ESTATE", -6: "ENODEV"}


class BmlpError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("bmlp error %s (%d): %s" % (_ERRNAMES.get(code, "?"), code, msg))
        self.code = code


class bmlp_hparams(C.Structure):
    _fields_ = [("bs", C.c_int32), ("r_num", C.c_int32), ("r_den", C.c_int32),
                ("p_r0", C.c_double), ("gamma", C.POINTER(C.c_int32)), ("fwd_impl", C.c_int32),
                ("group_mode", C.c_int32)]


_lib = None
_lock = threading.Lock()
_vp = C.c_void_p
_i32p = C.POINTER(C.c_int32)
_i64p = C.POINTER(C.c_int64)
_f64p = C.POINTER(C.c_double)

# (name, restype, argtypes) of every entry point of include/bmlp.h
SIGNATURES = [
    ("bmlp_create", C.c_int, [_i32p, C.c_int32, C.c_int32, C.c_int16, C.c_uint64,
                              C.POINTER(bmlp_hparams), C.POINTER(_vp)]),
    ("bmlp_destroy", None, [_vp]),
    ("bmlp_train", C.c_int, [_vp, _vp, _vp, C.c_int64, C.c_uint32, _vp, _i64p]),
    ("bmlp_predict", C.c_int, [_vp, _vp, C.c_int64, _vp, _vp]),
    ("bmlp_get_state", C.c_int, [_vp, C.c_int32, _vp, _vp, _vp, _f64p, _i64p]),
    ("bmlp_set_state", C.c_int, [_vp, C.c_int32, _vp, C.c_double, C.c_int64]),
    ("bmlp_get_info", C.c_int, [_vp, _i32p, _i32p, _i32p, _i32p, _i32p, _i32p]),
    ("bmlp_last_error", C.c_char_p, [_vp]),
    ("bmlp_gamma_rule", C.c_int32, [C.c_int32]),
    ("bmlp_reinforce_tables", C.c_int, [C.c_double, C.c_int32, C.c_int32, _vp, _vp, _vp]),
    ("bmlp_debug_last_step", C.c_int, [_vp, C.c_int32, _vp, _vp, _vp, _vp]),
    ("bmlp_set_profiling", C.c_int, [_vp, C.c_int32]),
    ("bmlp_get_profile", C.c_int, [_vp, C.c_int32, _i64p, _f64p]),
    ("bmlp_reset_profile", C.c_int, [_vp]),
    ("bmlp_launch_count", C.c_int64, [_vp]),
    ("bmlp_predict_noalloc", C.c_int, [_vp, _vp, C.c_int64, _vp, _vp]),
    ("bmlp_layer_forward", C.c_int, [_vp, C.c_int32, _vp, C.c_int64, _vp, _vp]),
    ("bmlp_update_stats", C.c_int, [_vp, _vp, _vp, _vp, C.c_int32]),
    ("bmlp_predict_layers", C.c_int, [_vp, _vp, C.c_int64, _vp, _vp]),
    ("bmlp_layer_errors", C.c_int, [_vp, _i64p, C.c_int32]),
    ("bmlp_binarize_median", C.c_int, [_vp, C.c_int64, C.c_int32, _vp, _vp]),
    ("bmlp_expand_weights", C.c_int, [C.c_uint64, C.c_int32, C.c_int32, _vp, _vp]),
    ("bmlp_expand_sign", C.c_int, [_vp, C.c_int64, C.c_int32, _vp, C.c_int32, _vp, _vp]),
    ("bmlp_debug_expand_sign", C.c_int, [_vp, C.c_int64, C.c_int32, _vp, C.c_int32, _vp, _vp, C.c_int64]),
    ("bmlp_debug_wait_probe", C.c_int, [_vp, C.c_int32, C.c_double]),
    ("bmlp_engine_peak", C.c_int, [C.c_int32, C.c_int64, _f64p, _f64p]),
    ("bmlp_debug_fail_alloc", C.c_int, [C.c_int64]),
    ("bmlp_debug_fail_launch", C.c_int, [C.c_int64]),
    ("bmlp_debug_alloc_stats", C.c_int, [_i64p, _i64p]),
    ("bmlp_quantize_rows", C.c_int, [_vp, C.c_int32, C.c_int64, C.c_int64, C.c_int32, _vp, C.c_int64, _vp, _vp]),
    ("bmlp_norm_quantize", C.c_int, [_vp, C.c_int64, _vp, C.c_int64, _vp, C.c_int32, C.c_int64, C.c_int32,
                                     C.c_float, _vp, C.c_int64, _vp, C.c_int64, _vp, _vp]),
    ("bmlp_int8_matmul", C.c_int, [_vp, C.c_int64, _vp, _vp, C.c_int64, _vp, _vp, C.c_int64, C.c_int32, C.c_int32,
                                   _vp, C.c_int32, C.c_int64, _vp, C.c_int64, _vp]),
    ("bmlp_debug_int8_matmul", C.c_int, [_vp, C.c_int64, _vp, _vp, C.c_int64, _vp, _vp, C.c_int64, C.c_int32, C.c_int32,
                                   _vp, C.c_int32, C.c_int64, _vp, C.c_int64, _vp]),
    ("bmlp_int8_sign", C.c_int, [_vp, C.c_int64, _vp, C.c_int64, _vp, C.c_int64, C.c_int32, C.c_int32, _vp, _vp,
                                 C.c_int64, _vp]),
    ("bmlp_debug_int8_sign", C.c_int, [_vp, C.c_int64, _vp, C.c_int64, _vp, C.c_int64, C.c_int32, C.c_int32, _vp, _vp,
                                       C.c_int64, _vp]),
    ("bmlp_int8_workspace", C.c_int64, [C.c_int64, C.c_int32, C.c_int32]),
    ("bmlp_layer_forward_engine", C.c_int, [_vp, C.c_int32, C.c_int32, _vp, C.c_int64, _vp, _vp]),
]


def library_path() -> str:
    return _build.LIB


def lib(build_if_missing: bool = True):
    """Load libbmlp.so (building it with nvcc first if it is missing)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            path = _build.LIB
            if not os.path.exists(path):
                if not build_if_missing:
                    raise OSError("libbmlp.so is not built: run __graft_entry__.build()")
                _build.build()
            L = C.CDLL(path)
            for name, res, args in SIGNATURES:
                f = getattr(L, name)
                f.restype = res
                f.argtypes = args
            _lib = L   # last: the check above reads it without the lock
    return _lib


def _check(rc, h=None):
    if rc != BMLP_OK:
        msg = lib().bmlp_last_error(h)
        raise BmlpError(rc, msg.decode() if msg else "")


def _ptr(buf):
    """Raw pointer of a torch tensor or numpy array (must be contiguous)."""
    if buf is None:
        return None
    if isinstance(buf, np.ndarray):
        assert buf.flags["C_CONTIGUOUS"], "numpy buffer must be C-contiguous"
        return buf.ctypes.data
    if hasattr(buf, "data_ptr"):
        assert buf.is_contiguous(), "tensor must be contiguous"
        return buf.data_ptr()
    raise TypeError("expected a torch tensor or a numpy array, got %r" % type(buf))


# -- tensors of the 8-bit front end (torch is imported when the first one comes) --
_torch = _raw_stream = _get_device = None
_devices = 0                          # that torch sees
_real_types, _out_types = {}, {}      # torch dtype -> BMLP_* type


def _use_torch():
    global _torch, _raw_stream, _get_device, _devices
    import torch
    _real_types.update({torch.float32: BMLP_F32, torch.float16: BMLP_F16, torch.bfloat16: BMLP_BF16})
    _out_types.update(_real_types)
    _out_types[torch.int32] = BMLP_I32
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _get_device = getattr(torch._C, "_cuda_getDevice", None)
    _devices = torch.cuda.device_count()
    _torch = torch
    return torch


def _type(t, of, what):
    """BMLP_* type of a tensor's elements."""
    code = of.get(t.dtype)
    if code is None:
        raise TypeError("%s: expected a tensor of %s, got %s" % (what, ", ".join(map(str, of)), t.dtype))
    return code


def _rows(t, shape, what, dtype):
    """(pointer, row stride in elements) of a tensor of that shape whose rows are contiguous."""
    if t.shape != shape:
        raise ValueError("%s: expected shape %s, got %s" % (what, shape, tuple(t.shape)))
    if t.dtype is not dtype:
        raise TypeError("%s: expected %s, got %s" % (what, dtype, t.dtype))
    ld, step = t.stride()
    if step != 1 and shape[1] > 1:
        raise ValueError("%s: the elements of a row must be contiguous" % what)
    return t.data_ptr(), ld


def _int32(K, N=1):
    """ctypes would cut a K or N of more than 32 bits without a word."""
    raise BmlpError(BMLP_EINVAL, "K = %d or N = %d past 31 bits" % (K, N))


def _vector(t, n, what, dtype):
    """Pointer of a contiguous vector of n elements (None: NULL)."""
    if t is None:
        return None
    if t.shape != (n,) or t.dtype is not dtype or (n > 1 and t.stride(0) != 1):
        raise ValueError("%s: expected %d contiguous values of %s, got %s of %s"
                         % (what, n, dtype, tuple(t.shape), t.dtype))
    return t.data_ptr()


def _one_device(x, *others):
    """Refuses tensors of another device than the current one, where the kernels run.  (The
    library does too, by its pointers, and refuses host memory.)"""
    here = x.get_device()
    if here >= 0 and here != (_get_device or _torch.cuda.current_device)():
        raise ValueError("tensors on cuda:%d, which is not the current device" % here)
    for t in others:
        if t is not None and t.get_device() not in (here, -1):
            raise ValueError("tensors on different devices: cuda:%d and %s" % (t.get_device(), x.device))


def _tensor_stream(stream, t):
    """_stream(stream), where a tensor on the device says that CUDA is initialised."""
    if stream is None and _raw_stream is not None and _get_device is not None and t.is_cuda:
        return _raw_stream(_get_device())
    return _stream(stream)


def _stream(stream):
    if stream is None:
        torch = sys.modules.get("torch")   # not imported: not initialised either
        if torch is None or not torch.cuda.is_initialized():
            return None
        # (a Stream object takes 3 us to make, a third of the shortest calls)
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            return raw(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


# -- the C-ABI, one Python function per entry point ------------------------------

def bmlp_create(widths, classes, h_max=255, seed=0, bs=100, r=(1, 4), p_r0=0.5, gamma=None,
                fwd_impl=BMLP_FWD_AUTO, group_mode=BMLP_GROUPS_CONTIGUOUS):
    w = (C.c_int32 * len(widths))(*[int(v) for v in widths])
    hp = bmlp_hparams()
    hp.bs = bs
    hp.r_num, hp.r_den = int(r[0]), int(r[1])
    hp.p_r0 = float(p_r0)
    g = None
    if gamma is not None:
        g = (C.c_int32 * len(gamma))(*[int(v) for v in gamma])
        hp.gamma = C.cast(g, _i32p)
    hp.fwd_impl = fwd_impl
    hp.group_mode = group_mode
    h = _vp()
    rc = lib().bmlp_create(w, len(widths), classes, h_max, seed & (2 ** 64 - 1), C.byref(hp), C.byref(h))
    _check(rc, None)
    return h.value


def bmlp_destroy(h):
    lib().bmlp_destroy(h)


def bmlp_train(h, x_packed, labels, n=None, flags=0, stream=None, count_errors=False):
    n = labels.shape[0] if n is None else n
    err = C.c_int64(-1)
    rc = lib().bmlp_train(h, _ptr(x_packed), _ptr(labels), n, flags, _stream(stream),
                          C.byref(err) if count_errors else None)
    _check(rc, h)
    return int(err.value) if count_errors else None


def bmlp_predict(h, x_packed, labels_out, n=None, stream=None):
    n = labels_out.shape[0] if n is None else n
    _check(lib().bmlp_predict(h, _ptr(x_packed), n, _ptr(labels_out), _stream(stream)), h)


def bmlp_predict_noalloc(h, x_packed, labels_out, n=None, stream=None):
    """Allocation-free bmlp_predict for callers that cannot allocate device
    memory (device buffers only; n * ceil(max K_l / 64) <= 2^20)."""
    n = labels_out.shape[0] if n is None else n
    _check(lib().bmlp_predict_noalloc(h, _ptr(x_packed), n, _ptr(labels_out), _stream(stream)), h)


def bmlp_predict_layers(h, x_packed, labels_out, n=None, stream=None):
    """Early-exit predictions of every layer into labels_out (L x n, layer-major)."""
    n = labels_out.shape[-1] if n is None else n
    _check(lib().bmlp_predict_layers(h, _ptr(x_packed), n, _ptr(labels_out), _stream(stream)), h)


def bmlp_layer_errors(h, reset=False):
    """Local 01-loss counts of layers 1..L since creation or the last reset."""
    L = C.c_int32()
    lib().bmlp_get_info(h, C.byref(L), None, None, None, None, None)
    out = (C.c_int64 * L.value)()
    _check(lib().bmlp_layer_errors(h, out, 1 if reset else 0), h)
    return [int(v) for v in out]


def bmlp_binarize_median(x, out, stream=None):
    """Median binarisation of n x K fp32 patterns (device) into packed bits."""
    n, K = x.shape
    _check(lib().bmlp_binarize_median(_ptr(x), n, K, _ptr(out), _stream(stream)), None)


def bmlp_expand_weights(seed, K, D, E_out, stream=None):
    """The packed K x D +-1 expansion matrix (device, K x ceil(D/64) int64)."""
    _check(lib().bmlp_expand_weights(seed, K, D, _ptr(E_out), _stream(stream)), None)


def bmlp_expand_sign(x, E, K, out, stream=None):
    """Expansion layer: n x D uint8 patterns (device) -> packed sign(x E^T)."""
    n, D = x.shape
    _check(lib().bmlp_expand_sign(_ptr(x), n, D, _ptr(E), K, _ptr(out), _stream(stream)), None)


def bmlp_quantize_rows(x, q, scale, stream=None):
    """8-bit codes q (n x K int8) and scales (n fp32) of the rows of x (n x K
    fp32 / fp16 / bf16, on the device; row strides are kept)."""
    torch = _torch or _use_torch()
    shape = n, K = x.shape
    if K >> 31:
        _int32(K)
    if _devices > 1:
        _one_device(x, q, scale)
    px, ldx = _rows(x, shape, "x", x.dtype)
    pq, ldq = _rows(q, shape, "q", torch.int8)
    rc = (_lib or lib()).bmlp_quantize_rows(px, _type(x, _real_types, "x"), ldx, n, K, pq, ldq,
                                            _vector(scale, n, "scale", torch.float32), _tensor_stream(stream, x))
    if rc:
        _check(rc)


def bmlp_norm_quantize(x, gain, q, scale, res=None, sum_out=None, eps=1e-6, stream=None):
    """RMS norm of the rows of x + res times gain as 8-bit codes q (n x K int8)
    and scales (n fp32); sum_out (may be x or res): x + res in their type.
    gain, res, sum_out: x's type, each may be None."""
    torch = _torch or _use_torch()
    shape = n, K = x.shape
    if K >> 31:
        _int32(K)
    dtype = x.dtype
    if _devices > 1:
        _one_device(x, gain, q, scale, res, sum_out)
    px, ldx = _rows(x, shape, "x", dtype)
    pr, ldr = (None, 0) if res is None else _rows(res, shape, "res", dtype)
    ps, lds = (None, 0) if sum_out is None else _rows(sum_out, shape, "sum_out", dtype)
    pq, ldq = _rows(q, shape, "q", torch.int8)
    rc = (_lib or lib()).bmlp_norm_quantize(px, ldx, pr, ldr, _vector(gain, K, "gain", dtype),
                                            _type(x, _real_types, "x"), n, K, eps, ps, lds, pq, ldq,
                                            _vector(scale, n, "scale", torch.float32), _tensor_stream(stream, x))
    if rc:
        _check(rc)


def bmlp_int8_workspace(n, K, N):
    """Bytes of workspace with which the product of this size runs fastest."""
    return 0 if (K | N) >> 31 else int(lib().bmlp_int8_workspace(n, K, N))   # (0: refused)


_KEPT_WORKSPACE = 64 << 20     # bytes of the largest workspace that is kept for the next call
_KEPT_STREAMS = 4              # of the streams used last
_kept = threading.local()      # .at[device, stream]: this thread's, in the order of that stream


def bmlp_release_workspaces():
    """Give the workspaces that bmlp_int8_matmul and bmlp_int8_sign keep for the
    calling thread back to torch's allocator."""
    _kept.__dict__.clear()


def _on_stream(stream, a):
    """torch's current stream is the call's: a block that was freed on a stream is given out
    again at once, in the order of that stream alone."""
    if stream is None:
        return contextlib.nullcontext()
    raw = _stream(stream)
    if raw == _tensor_stream(None, a):
        return contextlib.nullcontext()
    cuda = _torch.cuda
    if isinstance(stream, cuda.Stream):
        return cuda.stream(stream)
    # (0 and 1: the legacy default stream)
    return cuda.stream(cuda.ExternalStream(raw, a.device) if raw > 1 else cuda.default_stream(a.device))


def _in_graph_pool(block):
    """Whether a block that was allocated in a capture stays the graph's."""
    at = block.data_ptr()
    return any(s["address"] <= at < s["address"] + s["total_size"] and tuple(s.get("segment_pool_id", (0, 0))) != (0, 0)
               for s in _torch.cuda.memory_snapshot())


def _block(size, a, stream):
    """A block of the call's stream.  None where there is no room for it; in a capture that is
    not torch's own, whose graph would write it while others have it; and in a capture with
    another allocator than torch's native one: what those allocate there is no device memory yet."""
    torch = _torch
    captured = torch.cuda.is_current_stream_capturing()
    with _on_stream(stream, a):
        capturing = torch.cuda.is_current_stream_capturing()
        if capturing and not (captured and torch.cuda.get_allocator_backend() == "native"):
            return None
        try:
            block = torch.empty(size, dtype=torch.uint8, device=a.device)
        except torch.cuda.OutOfMemoryError:
            return None
        return None if capturing and not _in_graph_pool(block) else block


def _workspace(L, workspace, n, K, N, a, stream):
    """(pointer, bytes) of the given workspace, or of one from torch's allocator where
    the size wants it: kept for the thread's next call on the same stream if it is small
    and the stream is torch's current one, not in a capture.  None where there is none to
    be had: the product runs without."""
    if workspace is not None:
        if not workspace.is_contiguous():
            raise ValueError("workspace: its bytes must be contiguous")
        return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace
    size = L.bmlp_int8_workspace(n, K, N)
    if size == 0 or not a.is_cuda:
        return None, 0, None
    torch = _torch
    keep = stream is None and size <= _KEPT_WORKSPACE and not torch.cuda.is_current_stream_capturing()
    if keep:
        at = _kept.__dict__.setdefault("at", {})
        key = a.device, _tensor_stream(None, a)
        workspace = at.pop(key, None)
        if workspace is not None and workspace.shape[0] >= size:
            at[key] = workspace      # (the last in the order of use)
            return workspace.data_ptr(), size, workspace
        workspace = at[key] = None   # (the smaller one goes back first)
        while len(at) > _KEPT_STREAMS:
            del at[next(iter(at))]
        workspace = at[key] = _block(size, a, None)
    else:
        workspace = _block(size, a, stream)
    if workspace is None:
        return None, 0, None
    return workspace.data_ptr(), size, workspace


def bmlp_int8_matmul(a, w, out, a_scale=None, w_scale=None, bias=None, stream=None, workspace=None, expired=False):
    """out (n x N fp32 / fp16 / bf16, or int32 without scales and bias) = a (n x K
    int8) times w (N x K int8) transposed, scaled per row and channel.
    workspace: a device tensor of bmlp_int8_workspace(n, K, N) bytes (None: one from
    torch's allocator; up to 64 MB of it stay with the thread for its next call on the
    stream, for the four streams used last, until bmlp_release_workspaces; where there is no room for it, and in a capture
    that torch does not make, the call runs without, slower).  expired: bmlp_debug_int8_matmul."""
    torch = _torch or _use_torch()
    L = _lib or lib()
    shape = n, K = a.shape
    N = w.shape[0]
    if (K | N) >> 31:
        _int32(K, N)
    if _devices > 1:
        _one_device(a, w, out, a_scale, w_scale, bias, workspace)
    pa, lda = _rows(a, shape, "a", torch.int8)
    pw, ldw = _rows(w, (N, K), "w", torch.int8)
    po, ldo = _rows(out, (n, N), "out", out.dtype)
    f32 = torch.float32
    ws, wsb, owner = _workspace(L, workspace, n, K, N, a, stream) if n > 32 or workspace is not None else (None, 0, None)
    call = L.bmlp_debug_int8_matmul if expired else L.bmlp_int8_matmul
    rc = call(pa, lda, _vector(a_scale, n, "a_scale", f32), pw, ldw, _vector(w_scale, N, "w_scale", f32),
              _vector(bias, N, "bias", f32), n, K, N, po, _type(out, _out_types, "out"), ldo, ws, wsb,
              _tensor_stream(stream, a))
    if rc:
        _check(rc)


def bmlp_int8_sign(a, w, out, threshold=None, stream=None, workspace=None, expired=False):
    """Packed +-1 words (n x ceil(N/64) int64) of a (n x K int8) times w (N x K
    int8) transposed against threshold (N int32; None: 0).  workspace: as for
    bmlp_int8_matmul.  expired: bmlp_debug_int8_sign."""
    torch = _torch or _use_torch()
    L = _lib or lib()
    shape = n, K = a.shape
    N = w.shape[0]
    if (K | N) >> 31:
        _int32(K, N)
    if _devices > 1:
        _one_device(a, w, out, threshold, workspace)
    pa, lda = _rows(a, shape, "a", torch.int8)
    pw, ldw = _rows(w, (N, K), "w", torch.int8)
    if out.shape != (n, (N + 63) // 64) or out.element_size() != 8 or not out.is_contiguous():
        raise ValueError("out: expected %d x %d contiguous 64-bit words" % (n, (N + 63) // 64))
    ws, wsb, owner = _workspace(L, workspace, n, K, N, a, stream) if n > 32 or workspace is not None else (None, 0, None)
    call = L.bmlp_debug_int8_sign if expired else L.bmlp_int8_sign
    rc = call(pa, lda, pw, ldw, _vector(threshold, N, "threshold", torch.int32), n, K, N,
              out.data_ptr(), ws, wsb, _tensor_stream(stream, a))
    if rc:
        _check(rc)


def bmlp_debug_expand_sign(x, E, K, out, expired_tile, stream=None):
    """bmlp_expand_sign with every CTA's wait for its tile expired_tile taken as
    expired."""
    n, D = x.shape
    _check(lib().bmlp_debug_expand_sign(_ptr(x), n, D, _ptr(E), K, _ptr(out), _stream(stream), int(expired_tile)), None)


def bmlp_debug_wait_probe(h, arrive, seconds=0.05, leave_pending=False):
    """Run the bounded-wait probe; raises BmlpError(BMLP_ETIMEOUT) if it expired.
    leave_pending: nothing arrives and the expiry is left for the next
    synchronising call to report."""
    a = -1 if leave_pending else (1 if arrive else 0)
    _check(lib().bmlp_debug_wait_probe(h, a, float(seconds)), h)


def bmlp_layer_forward(h, layer, a_in, a_out, n=None, stream=None):
    """a_out = sign(a_in W_layer), packed rows on the device."""
    n = a_out.shape[0] if n is None else n
    _check(lib().bmlp_layer_forward(h, layer, _ptr(a_in), n, _ptr(a_out), _stream(stream)), h)


def bmlp_layer_forward_engine(h, layer, engine, a_in, a_out, n=None, stream=None):
    """bmlp_layer_forward on the given engine (BMLP_FWD_POPC / TCGEN05 / B1MMA)."""
    n = a_out.shape[0] if n is None else n
    _check(lib().bmlp_layer_forward_engine(h, layer, engine, _ptr(a_in), n, _ptr(a_out),
                                           _stream(stream)), h)


def bmlp_debug_fail_alloc(nth):
    """Arm (nth >= 1) or disarm (0) the one-shot failure of the nth allocation."""
    _check(lib().bmlp_debug_fail_alloc(int(nth)), None)


def bmlp_debug_fail_launch(nth):
    """Arm (nth >= 1) or disarm (0) the one-shot failure of the nth training
    mini-batch that is launched kernel by kernel."""
    _check(lib().bmlp_debug_fail_launch(int(nth)), None)


def bmlp_debug_alloc_stats():
    """(allocations the library holds, their bytes), over all live handles."""
    n, b = C.c_int64(), C.c_int64()
    _check(lib().bmlp_debug_alloc_stats(C.byref(n), C.byref(b)), None)
    return n.value, b.value


def bmlp_engine_peak(engine, iters):
    """(bit-pairs per second over the device, ms of the timed launch) of one
    contraction unit's peak kernel."""
    bp, ms = C.c_double(), C.c_double()
    _check(lib().bmlp_engine_peak(engine, iters, C.byref(bp), C.byref(ms)), None)
    return bp.value, ms.value


def bmlp_update_stats(h, reset=False):
    """(rows visited, rows streamed, algorithmic bytes) of the update kernel."""
    r, st, by = C.c_int64(), C.c_int64(), C.c_int64()
    _check(lib().bmlp_update_stats(h, C.byref(r), C.byref(st), C.byref(by), 1 if reset else 0), h)
    return r.value, st.value, by.value


def bmlp_get_info(h):
    L = C.c_int32()
    lib().bmlp_get_info(h, C.byref(L), None, None, None, None, None)
    widths = (C.c_int32 * (L.value + 1))()
    gam = (C.c_int32 * L.value)()
    cls, bs, fwd = C.c_int32(), C.c_int32(), C.c_int32()
    _check(lib().bmlp_get_info(h, C.byref(L), widths, C.byref(cls), gam, C.byref(bs), C.byref(fwd)), h)
    return dict(L=L.value, widths=list(widths), classes=cls.value, gamma=list(gam), bs=bs.value,
                fwd_impl=fwd.value)


def bmlp_get_state(h, layer):
    """Returns (H int16 K_l x K_{l-1}, W uint64 K_l x nw, P int8 K_l x c, p_r, step)."""
    info = bmlp_get_info(h)
    Kin, Kout, c = info["widths"][layer - 1], info["widths"][layer], info["classes"]
    H = np.empty((Kout, Kin), np.int16)
    W = np.empty((Kout, (Kin + 63) // 64), np.uint64)
    P = np.empty((Kout, c), np.int8)
    pr = C.c_double()
    step = C.c_int64()
    _check(lib().bmlp_get_state(h, layer, H.ctypes.data, W.ctypes.data, P.ctypes.data,
                                C.byref(pr), C.byref(step)), h)
    return H, W, P, pr.value, step.value


def bmlp_set_state(h, layer, H=None, p_r=0.0, step=-1):
    Hc = None if H is None else np.ascontiguousarray(H, dtype=np.int16)
    _check(lib().bmlp_set_state(h, layer, None if Hc is None else Hc.ctypes.data, p_r, step), h)


def bmlp_debug_last_step(h, layer):
    info = bmlp_get_info(h)
    K, bs = info["widths"][layer], info["bs"]
    G = K // info["gamma"][layer - 1]
    Z = np.empty((bs, K), np.int16)
    A = np.empty((bs, (K + 63) // 64), np.uint64)
    mark = np.empty(bs, np.uint8)
    sel = np.empty((bs, G), np.int16)
    _check(lib().bmlp_debug_last_step(h, layer, Z.ctypes.data, A.ctypes.data, mark.ctypes.data,
                                      sel.ctypes.data), h)
    return Z, A, mark, sel


def bmlp_gamma_rule(K):
    return lib().bmlp_gamma_rule(K)


def bmlp_reinforce_tables(p_r, K, n):
    """Sampler thresholds of a block of n inputs: (any, first[n], gap[n-1])."""
    any_ = np.zeros(1, np.uint64)
    first = np.zeros(64, np.uint64)
    gap = np.zeros(64, np.uint64)
    _check(lib().bmlp_reinforce_tables(p_r, K, n, any_.ctypes.data, first.ctypes.data,
                                       gap.ctypes.data), None)
    return int(any_[0]), first[:n].copy(), gap[:max(n - 1, 0)].copy()


def bmlp_last_error(h=None):
    m = lib().bmlp_last_error(h)
    return m.decode() if m else ""


def bmlp_set_profiling(h, every=1):
    """every: 0 off, 1 every mini-batch, S every S-th mini-batch (True = 1)."""
    _check(lib().bmlp_set_profiling(h, int(every)), h)


def bmlp_get_profile(h):
    out = {}
    for i, name in enumerate(PROFILE_KINDS):
        n, ms = C.c_int64(), C.c_double()
        _check(lib().bmlp_get_profile(h, i, C.byref(n), C.byref(ms)), h)
        out[name] = (n.value, ms.value)
    return out


def bmlp_reset_profile(h):
    _check(lib().bmlp_reset_profile(h), h)


def bmlp_launch_count(h):
    return int(lib().bmlp_launch_count(h))


# -- convenience object -----------------------------------------------------------

class BMLP:
    """Owning wrapper of a bmlp_t handle."""

    def __init__(self, widths, classes, h_max=255, seed=0, bs=100, r=(1, 4), p_r0=0.5,
                 gamma=None, fwd_impl=BMLP_FWD_AUTO, group_mode=BMLP_GROUPS_CONTIGUOUS):
        self.h = bmlp_create(widths, classes, h_max, seed, bs, r, p_r0, gamma, fwd_impl,
                             group_mode)
        self.info = bmlp_get_info(self.h)

    def close(self):
        if getattr(self, "h", None):
            bmlp_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def train(self, x_packed, labels, epoch_end=False, stream=None, count_errors=False, n=None):
        return bmlp_train(self.h, x_packed, labels, n, BMLP_EPOCH_END if epoch_end else 0, stream,
                          count_errors)

    def predict(self, x_packed, labels_out, stream=None, n=None):
        bmlp_predict(self.h, x_packed, labels_out, n, stream)

    def predict_layers(self, x_packed, labels_out, stream=None, n=None):
        bmlp_predict_layers(self.h, x_packed, labels_out, n, stream)

    def layer_errors(self, reset=False):
        return bmlp_layer_errors(self.h, reset)

    def state(self, layer):
        return bmlp_get_state(self.h, layer)

    def set_state(self, layer, H=None, p_r=0.0, step=-1):
        bmlp_set_state(self.h, layer, H, p_r, step)
