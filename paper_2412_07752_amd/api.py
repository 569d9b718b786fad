"""Thin binding over libflashrnn.so (the C ABI of include/flashrnn.h), same entry-point names: ctypes, and for plain forward calls a native module
(csrc/flashrnn_binding.cpp) that makes the same checks.

Argument marshalling only: torch supplies device memory and the current HIP stream, every step of
the computation runs inside the library's kernels.  There is no fallback: if the library has not
been built (python -m paper_2412_07752_amd.build) every call raises.
"""
import ctypes
import functools
import os
import warnings

import torch

from .build import binding_stamp

FLASHRNN_LSTM, FLASHRNN_GRU, FLASHRNN_SLSTM, FLASHRNN_ELMAN, FLASHRNN_GRU4 = 0, 1, 2, 3, 4
FLASHRNN_F32, FLASHRNN_BF16 = 0, 1
FLASHRNN_I32, FLASHRNN_I64 = 2, 3
FLASHRNN_OK = 0
FLASHRNN_ERR_NULL, FLASHRNN_ERR_SHAPE, FLASHRNN_ERR_UNSUPPORTED = -1, -2, -3
FLASHRNN_ERR_WORKSPACE, FLASHRNN_ERR_LAUNCH, FLASHRNN_ERR_TIMEOUT, FLASHRNN_ERR_SCRATCH = -4, -5, -6, -7
FLASHRNN_STATIC_SCRATCH_BYTES = 16 << 20
STATIC_SCRATCH = "static"   # stands for FLASHRNN_STATIC_SCRATCH in flashrnn_check

# FLASHRNN_LIB=trace selects the library built with per-phase clock stamps (python -m paper_2412_07752_amd.build --trace)
_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)),
                         "libflashrnn_trace.so" if os.environ.get("FLASHRNN_LIB") == "trace" else "libflashrnn.so")
_lib = None
_native = None   # the native module, bound to the loaded library


class flashrnn_desc_t(ctypes.Structure):
    _fields_ = [("cell", ctypes.c_int), ("T", ctypes.c_int), ("B", ctypes.c_int), ("NH", ctypes.c_int), ("D", ctypes.c_int),
                ("io_dtype", ctypes.c_int), ("recurrent_grad_clip", ctypes.c_float)]


class flashrnn_embedding_desc_t(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_longlong), ("vocab", ctypes.c_int), ("width", ctypes.c_int), ("table_dtype", ctypes.c_int), ("io_dtype", ctypes.c_int),
                ("index_dtype", ctypes.c_int), ("scale", ctypes.c_float)]


class flashrnn_layer_norm_desc_t(ctypes.Structure):
    _fields_ = [("rows_outer", ctypes.c_longlong), ("rows_inner", ctypes.c_longlong), ("x_stride", ctypes.c_longlong), ("groups", ctypes.c_int), ("width", ctypes.c_int),
                ("x_dtype", ctypes.c_int), ("io_dtype", ctypes.c_int), ("dx_dtype", ctypes.c_int), ("param_dtype", ctypes.c_int), ("eps", ctypes.c_float)]


class flashrnn_cross_entropy_desc_t(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_longlong), ("logits_stride", ctypes.c_longlong), ("dlogits_stride", ctypes.c_longlong), ("classes", ctypes.c_int), ("io_dtype", ctypes.c_int),
                ("index_dtype", ctypes.c_int), ("grad_scale", ctypes.c_float)]


class FlashRNNError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


def library_path():
    return _LIB_PATH


def _load_native():
    """The native module, or None: every call then goes through ctypes."""
    try:
        from . import _flashrnn_binding as native
    except ImportError as e:
        why = str(e)
    else:
        built_for = getattr(native, "built_for", "an unknown torch")
        if built_for == binding_stamp():
            return native
        why = f"built for {built_for}, running {binding_stamp()}"
    warnings.warn(f"forward calls take a few microseconds more through ctypes, for want of the native binding ({why}): python -m paper_2412_07752_amd.build", RuntimeWarning, stacklevel=3)
    return None


def lib():
    """The loaded C-ABI library; raises if it was not built."""
    global _lib, _native
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2412_07752_amd.build` "
                               "(there is no CPU fallback)")
        L = ctypes.CDLL(_LIB_PATH)
        dp = ctypes.POINTER(flashrnn_desc_t)
        vp = ctypes.c_void_p
        L.flashrnn_num_states.argtypes = [ctypes.c_int]
        L.flashrnn_num_states.restype = ctypes.c_int
        L.flashrnn_num_gates.argtypes = [ctypes.c_int]
        L.flashrnn_num_gates.restype = ctypes.c_int
        L.flashrnn_gate_cache_bytes.argtypes = [dp]
        L.flashrnn_gate_cache_bytes.restype = ctypes.c_size_t
        L.flashrnn_workspace_bytes.argtypes = [dp]
        L.flashrnn_workspace_bytes.restype = ctypes.c_size_t
        L.flashrnn_fwd.argtypes = [dp] + [vp] * 8
        L.flashrnn_fwd.restype = ctypes.c_int
        L.flashrnn_fwd_static_scratch.argtypes = [dp] + [vp] * 7
        L.flashrnn_fwd_static_scratch.restype = ctypes.c_int
        L.flashrnn_bwd.argtypes = [dp] + [vp] * 12
        L.flashrnn_bwd.restype = ctypes.c_int
        L.flashrnn_bwd_recompute.argtypes = [dp] + [vp] * 12
        L.flashrnn_bwd_recompute.restype = ctypes.c_int
        L.flashrnn_recompute_workspace_bytes.argtypes = [dp]
        L.flashrnn_recompute_workspace_bytes.restype = ctypes.c_size_t
        L.flashrnn_check.argtypes = [dp, vp, vp]
        L.flashrnn_check.restype = ctypes.c_int
        L.flashrnn_plan.argtypes = [dp, ctypes.c_int] + [ctypes.POINTER(ctypes.c_int)] * 3
        L.flashrnn_plan.restype = ctypes.c_int
        L.flashrnn_plan_kernel.argtypes = [dp, ctypes.c_int] + [ctypes.POINTER(ctypes.c_int)] * 3
        L.flashrnn_plan_kernel.restype = ctypes.c_int
        L.flashrnn_profile_enable.argtypes = [ctypes.c_int]
        L.flashrnn_profile_enable.restype = ctypes.c_int
        L.flashrnn_profile_kernel_ms.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int)]
        L.flashrnn_profile_kernel_ms.restype = ctypes.c_int
        L.flashrnn_trace_phases.argtypes = [dp, vp, ctypes.c_int, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int), vp]
        L.flashrnn_trace_phases.restype = ctypes.c_int
        ep, np_, cp = (ctypes.POINTER(t) for t in (flashrnn_embedding_desc_t, flashrnn_layer_norm_desc_t, flashrnn_cross_entropy_desc_t))
        L.flashrnn_embedding_workspace_bytes.argtypes = [ep]
        L.flashrnn_embedding_workspace_bytes.restype = ctypes.c_size_t
        L.flashrnn_embedding_fwd.argtypes = [ep] + [vp] * 4
        L.flashrnn_embedding_fwd.restype = ctypes.c_int
        L.flashrnn_embedding_bwd.argtypes = [ep] + [vp] * 3 + [ctypes.c_int] + [vp] * 2
        L.flashrnn_embedding_bwd.restype = ctypes.c_int
        L.flashrnn_layer_norm_workspace_bytes.argtypes = [np_]
        L.flashrnn_layer_norm_workspace_bytes.restype = ctypes.c_size_t
        L.flashrnn_layer_norm_fwd.argtypes = [np_] + [vp] * 7
        L.flashrnn_layer_norm_fwd.restype = ctypes.c_int
        L.flashrnn_layer_norm_bwd.argtypes = [np_] + [vp] * 10
        L.flashrnn_layer_norm_bwd.restype = ctypes.c_int
        L.flashrnn_cross_entropy.argtypes = [cp] + [vp] * 7
        L.flashrnn_cross_entropy.restype = ctypes.c_int
        L.flashrnn_grad_clip_workspace_bytes.argtypes = [ctypes.c_int]
        L.flashrnn_grad_clip_workspace_bytes.restype = ctypes.c_size_t
        L.flashrnn_grad_clip.argtypes = [ctypes.c_int, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp]
        L.flashrnn_grad_clip.restype = ctypes.c_int
        L.flashrnn_status_string.argtypes = [ctypes.c_int]
        L.flashrnn_status_string.restype = ctypes.c_char_p
        native = _load_native()
        if native is not None:
            native.bind(*(ctypes.cast(f, vp).value for f in (L.flashrnn_fwd, L.flashrnn_fwd_static_scratch, L.flashrnn_num_states, L.flashrnn_num_gates)))
            native.bind_operators(*(ctypes.cast(f, vp).value for f in (
                L.flashrnn_embedding_fwd, L.flashrnn_embedding_bwd, L.flashrnn_embedding_workspace_bytes, L.flashrnn_layer_norm_fwd, L.flashrnn_layer_norm_bwd,
                L.flashrnn_layer_norm_workspace_bytes, L.flashrnn_cross_entropy, L.flashrnn_grad_clip, L.flashrnn_grad_clip_workspace_bytes)))
        _lib, _native = L, native
    return _lib


EXPORTS = ["flashrnn_num_states", "flashrnn_num_gates", "flashrnn_gate_cache_bytes", "flashrnn_workspace_bytes", "flashrnn_fwd",
           "flashrnn_fwd_static_scratch", "flashrnn_bwd", "flashrnn_bwd_recompute", "flashrnn_recompute_workspace_bytes", "flashrnn_check", "flashrnn_plan", "flashrnn_plan_kernel", "flashrnn_profile_enable", "flashrnn_profile_kernel_ms",
           "flashrnn_trace_phases", "flashrnn_status_string", "flashrnn_embedding_workspace_bytes", "flashrnn_embedding_fwd", "flashrnn_embedding_bwd", "flashrnn_layer_norm_workspace_bytes",
           "flashrnn_layer_norm_fwd", "flashrnn_layer_norm_bwd", "flashrnn_cross_entropy", "flashrnn_grad_clip_workspace_bytes", "flashrnn_grad_clip"]


def status_string(status):
    return lib().flashrnn_status_string(int(status)).decode()


@functools.lru_cache(maxsize=16)
def _cell_sizes(cell):
    return lib().flashrnn_num_states(cell), lib().flashrnn_num_gates(cell)


def flashrnn_num_states(cell):
    return _cell_sizes(int(cell))[0]


def flashrnn_num_gates(cell):
    return _cell_sizes(int(cell))[1]


def make_desc(cell, T, B, NH, D, io_dtype, recurrent_grad_clip=0.0):
    """recurrent_grad_clip: 0 = off, c > 0 clips R^T dg_t to [-c, c] per step, negative cuts it (backward only)."""
    return flashrnn_desc_t(int(cell), int(T), int(B), int(NH), int(D), int(io_dtype), float(recurrent_grad_clip))


@functools.lru_cache(maxsize=256)
def _desc_of(cell, T, B, NH, D, io_dtype, recurrent_grad_clip=0.0):
    """The descriptor of a call; the binding's own, never handed out, so that one serves all calls of a shape.  Plain numbers only: a caller's
    object (a tensor or an array that holds the clip) would be looked up by what it is, not by its value."""
    return make_desc(cell, T, B, NH, D, io_dtype, recurrent_grad_clip)


def flashrnn_gate_cache_bytes(desc):
    return lib().flashrnn_gate_cache_bytes(ctypes.byref(desc))


def flashrnn_workspace_bytes(desc):
    return lib().flashrnn_workspace_bytes(ctypes.byref(desc))


def flashrnn_plan(desc, backward=False):
    """(workgroups, CUs per head, waves per workgroup) of the launch the library would use.
    backward: False / 0 the forward call that saves its values, True / 1 the backward call, 2 the forward call that saves nothing."""
    a, b, c = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    rc = lib().flashrnn_plan(ctypes.byref(desc), int(backward), ctypes.byref(a), ctypes.byref(b), ctypes.byref(c))
    if rc != FLASHRNN_OK:
        raise FlashRNNError(rc, "flashrnn_plan")
    return a.value, b.value, c.value


def flashrnn_plan_kernel(desc, backward=False):
    """(staged: 0 / 1 / 2 = staged with the deep fetch, batch tile rows, workgroups per group) of the kernel that plan uses."""
    a, b, c = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    rc = lib().flashrnn_plan_kernel(ctypes.byref(desc), int(backward), ctypes.byref(a), ctypes.byref(b), ctypes.byref(c))
    if rc != FLASHRNN_OK:
        raise FlashRNNError(rc, "flashrnn_plan_kernel")
    return a.value, b.value, c.value


def flashrnn_profile_enable(on):
    """on: False / 0 = off, True / 1 = every call, n = every n-th call of each direction carries the two events."""
    rc = lib().flashrnn_profile_enable(int(on))
    if rc != FLASHRNN_OK:
        raise FlashRNNError(rc, "flashrnn_profile_enable")


def flashrnn_profile_kernel_ms(backward):
    """(mean ms, launches) of the persistent kernel of the recorded forward / backward calls."""
    ms, n = ctypes.c_float(), ctypes.c_int()
    rc = lib().flashrnn_profile_kernel_ms(int(bool(backward)), ctypes.byref(ms), ctypes.byref(n))
    if rc != FLASHRNN_OK:
        raise FlashRNNError(rc, "flashrnn_profile_kernel_ms")
    return ms.value, n.value


def flashrnn_trace_phases(desc, workspace, backward, stream=None):
    """(clocks per phase [8], waves recorded) of the last forward / backward call on `workspace`; trace builds only."""
    arr = (ctypes.c_double * 8)()
    n = ctypes.c_int()
    rc = lib().flashrnn_trace_phases(ctypes.byref(desc), _ptr(workspace), int(bool(backward)), arr, ctypes.byref(n), _stream(stream))
    if rc != FLASHRNN_OK:
        raise FlashRNNError(rc, "flashrnn_trace_phases")
    return list(arr), n.value


def _ptr(t):
    return None if t is None else t.data_ptr()


def _io_dtype(t):
    if t.dtype == torch.bfloat16:
        return FLASHRNN_BF16
    if t.dtype == torch.float32:
        return FLASHRNN_F32
    raise TypeError(f"I/O tensors must be bfloat16 or float32, got {t.dtype}")


def _chk(t, shape, dtype, name, optional=False):
    if t is not None and t.dtype is dtype and t.shape == shape and t.is_cuda and t.is_contiguous():
        return
    if t is None:
        if optional:
            return
        raise ValueError(f"{name} is required")
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device tensor")
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        raise ValueError(f"{name}: got {tuple(t.shape)} {t.dtype}, expected {tuple(shape)} {dtype}")


def _stream(stream):
    if stream is None:   # the current stream's handle, without a stream object around it
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def alloc_workspace(desc, device):
    n = flashrnn_workspace_bytes(desc)
    if n == 0:
        raise FlashRNNError(FLASHRNN_ERR_UNSUPPORTED, "flashrnn_workspace_bytes")
    # zero-filled once: a backward call on a workspace that no forward call has used must find clean error words
    return torch.zeros(n, dtype=torch.uint8, device=device)


def flashrnn_fwd_static_scratch(cell, Wx, R, b, states0=None, save_for_backward=True, stream=None, states=None, gate_cache=None):
    """flashrnn_fwd without a workspace: the library works in its own static device array (no allocation in the call
    when `states` and `gate_cache` are passed in).  Returns (states, gate_cache or None)."""
    if _native is not None and stream is None:
        rc = _native.fwd(cell, Wx, R, b, states0, save_for_backward, None, states, gate_cache)
        if rc == FLASHRNN_OK:
            return states, (gate_cache if save_for_backward else None)
        if rc < 0:
            raise FlashRNNError(rc, "flashrnn_fwd_static_scratch")
    T, B, G, NH, D = Wx.shape
    cell = int(cell)
    S, gates = _cell_sizes(cell)
    if G != gates:
        raise ValueError("gate axis of Wx does not match the cell")
    dt = Wx.dtype
    desc = _desc_of(cell, T, B, NH, D, _io_dtype(Wx))
    _chk(Wx, (T, B, G, NH, D), dt, "Wx")
    _chk(R, (NH, D, G, D), dt, "R")
    _chk(b, (NH, G, D), dt, "b")
    _chk(states0, (S, B, NH, D), torch.float32, "states0", optional=True)
    if states is None:
        states = torch.empty((T + 1, S, B, NH, D), dtype=torch.float32, device=Wx.device)
    _chk(states, (T + 1, S, B, NH, D), torch.float32, "states")
    if save_for_backward and gate_cache is None:
        gate_cache = torch.empty(max(flashrnn_gate_cache_bytes(desc), 16), dtype=torch.uint8, device=Wx.device)
    rc = lib().flashrnn_fwd_static_scratch(ctypes.byref(desc), _ptr(Wx), _ptr(R), _ptr(b), _ptr(states0), _ptr(states),
                                           _ptr(gate_cache) if save_for_backward else None, _stream(stream))
    if rc != FLASHRNN_OK:
        raise FlashRNNError(rc, "flashrnn_fwd_static_scratch")
    return states, (gate_cache if save_for_backward else None)


def flashrnn_fwd(cell, Wx, R, b, states0=None, save_for_backward=True, workspace=None, stream=None, states=None, gate_cache=None):
    """Forward pass.  Wx[T,B,G,NH,D], R[NH,D,G,D], b[NH,G,D] (bf16 or f32), states0[S,B,NH,D] f32 or None.  states0 may be
    a slot of `states`.
    Returns (states[T+1,S,B,NH,D] f32, gate_cache or None, workspace)."""
    if _native is not None and stream is None and workspace is not None:
        rc = _native.fwd(cell, Wx, R, b, states0, save_for_backward, workspace, states, gate_cache)
        if rc == FLASHRNN_OK:
            return states, (gate_cache if save_for_backward else None), workspace
        if rc < 0:
            raise FlashRNNError(rc, "flashrnn_fwd")
    T, B, G, NH, D = Wx.shape
    cell = int(cell)
    S, gates = _cell_sizes(cell)
    if G != gates:
        raise ValueError("gate axis of Wx does not match the cell")
    dt = Wx.dtype
    desc = _desc_of(cell, T, B, NH, D, _io_dtype(Wx))
    _chk(Wx, (T, B, G, NH, D), dt, "Wx")
    _chk(R, (NH, D, G, D), dt, "R")
    _chk(b, (NH, G, D), dt, "b")
    _chk(states0, (S, B, NH, D), torch.float32, "states0", optional=True)
    dev = Wx.device
    if states is None:
        states = torch.empty((T + 1, S, B, NH, D), dtype=torch.float32, device=dev)
    _chk(states, (T + 1, S, B, NH, D), torch.float32, "states")
    if save_for_backward and gate_cache is None:
        gate_cache = torch.empty(max(flashrnn_gate_cache_bytes(desc), 16), dtype=torch.uint8, device=dev)
    if workspace is None:
        workspace = alloc_workspace(desc, dev)
    rc = lib().flashrnn_fwd(ctypes.byref(desc), _ptr(Wx), _ptr(R), _ptr(b), _ptr(states0), _ptr(states),
                            _ptr(gate_cache) if save_for_backward else None, _ptr(workspace), _stream(stream))
    if rc != FLASHRNN_OK:
        raise FlashRNNError(rc, "flashrnn_fwd")
    return states, (gate_cache if save_for_backward else None), workspace


def flashrnn_bwd(cell, R, b, states, gate_cache, dH, dstates_last=None, workspace=None, stream=None, out=None,
                 recurrent_grad_clip=0.0):
    """BPTT.  dH[T,B,NH,D] (I/O dtype).  Returns (dWx[T,B,G,NH,D], dR[NH,D,G,D] f32, db[NH,G,D] f32,
    dstates0[S,B,NH,D] f32).  `out` may pass preallocated (dWx, dR, db, dstates0).  recurrent_grad_clip as in
    flashrnn_desc_t: 0 off, c > 0 clips R^T dg_t to [-c, c] per step, negative cuts it."""
    T, B, NH, D = dH.shape
    cell = int(cell)
    S, G = _cell_sizes(cell)
    dt = dH.dtype
    desc = _desc_of(cell, T, B, NH, D, _io_dtype(dH), float(recurrent_grad_clip))
    _chk(R, (NH, D, G, D), dt, "R")
    _chk(b, (NH, G, D), dt, "b")
    _chk(states, (T + 1, S, B, NH, D), torch.float32, "states")
    _chk(dstates_last, (S, B, NH, D), torch.float32, "dstates_last", optional=True)
    if gate_cache is None or gate_cache.numel() * gate_cache.element_size() < flashrnn_gate_cache_bytes(desc):
        raise ValueError("gate_cache missing or too small")
    dev = dH.device
    if out is None:
        dWx = torch.empty((T, B, G, NH, D), dtype=dt, device=dev)
        dR = torch.empty((NH, D, G, D), dtype=torch.float32, device=dev)
        db = torch.empty((NH, G, D), dtype=torch.float32, device=dev)
        ds0 = torch.empty((S, B, NH, D), dtype=torch.float32, device=dev)
    else:
        dWx, dR, db, ds0 = out
    if workspace is None:
        workspace = alloc_workspace(desc, dev)
    rc = lib().flashrnn_bwd(ctypes.byref(desc), _ptr(R), _ptr(b), _ptr(states), _ptr(gate_cache), _ptr(dH), _ptr(dstates_last),
                            _ptr(dWx), _ptr(dR), _ptr(db), _ptr(ds0), _ptr(workspace), _stream(stream))
    if rc != FLASHRNN_OK:
        raise FlashRNNError(rc, "flashrnn_bwd")
    return dWx, dR, db, ds0


def flashrnn_bwd_recompute(cell, Wx, R, b, states, dH, dstates_last=None, workspace=None, stream=None, out=None, recurrent_grad_clip=0.0):
    """BPTT without saved values: they are formed again from Wx, R, b and the states, window by window.  Arguments and
    results as flashrnn_bwd, with Wx[T,B,G,NH,D] in place of the gate cache; `workspace` needs
    flashrnn_recompute_workspace_bytes() bytes."""
    T, B, NH, D = dH.shape
    cell = int(cell)
    S, G = _cell_sizes(cell)
    dt = dH.dtype
    desc = _desc_of(cell, T, B, NH, D, _io_dtype(dH), float(recurrent_grad_clip))
    _chk(Wx, (T, B, G, NH, D), dt, "Wx")
    _chk(R, (NH, D, G, D), dt, "R")
    _chk(b, (NH, G, D), dt, "b")
    _chk(states, (T + 1, S, B, NH, D), torch.float32, "states")
    _chk(dstates_last, (S, B, NH, D), torch.float32, "dstates_last", optional=True)
    dev = dH.device
    if out is None:
        out = (torch.empty((T, B, G, NH, D), dtype=dt, device=dev), torch.empty((NH, D, G, D), dtype=torch.float32, device=dev),
               torch.empty((NH, G, D), dtype=torch.float32, device=dev), torch.empty((S, B, NH, D), dtype=torch.float32, device=dev))
    dWx, dR, db, ds0 = out
    if workspace is None:
        n = lib().flashrnn_recompute_workspace_bytes(ctypes.byref(desc))
        if n == 0:
            raise FlashRNNError(FLASHRNN_ERR_UNSUPPORTED, "flashrnn_recompute_workspace_bytes")
        workspace = torch.zeros(n, dtype=torch.uint8, device=dev)
    rc = lib().flashrnn_bwd_recompute(ctypes.byref(desc), _ptr(Wx), _ptr(R), _ptr(b), _ptr(states), _ptr(dH), _ptr(dstates_last),
                                      _ptr(dWx), _ptr(dR), _ptr(db), _ptr(ds0), _ptr(workspace), _stream(stream))
    if rc != FLASHRNN_OK:
        raise FlashRNNError(rc, "flashrnn_bwd_recompute")
    return dWx, dR, db, ds0, workspace


def flashrnn_check(desc, workspace, stream=None):
    """Synchronizes and raises FlashRNNError if a kernel of the last call reported a timeout."""
    ws = ctypes.c_void_p(1) if isinstance(workspace, str) and workspace == STATIC_SCRATCH else _ptr(workspace)
    rc = lib().flashrnn_check(ctypes.byref(desc), ws, _stream(stream))
    if rc != FLASHRNN_OK:
        raise FlashRNNError(rc, "flashrnn_check")


# ---- around the time-step loop -------------------------------------------------------------------------------------------------------------
def _index_dtype(t):
    if t.dtype == torch.int64:
        return FLASHRNN_I64
    if t.dtype == torch.int32:
        return FLASHRNN_I32
    raise TypeError(f"tokens and targets must be int64 or int32, got {t.dtype}")


def _done(rc, where, result):
    if rc != FLASHRNN_OK:
        raise FlashRNNError(rc, where)
    return result


def _same_device(first, **others):
    if first.is_cuda and first.device.index != torch.cuda.current_device():
        raise ValueError(f"the tensors are on {first.device}, the current device is cuda:{torch.cuda.current_device()}")
    for name, t in others.items():
        if t is not None and t.device != first.device:
            raise ValueError(f"{name} is on {t.device}, the other tensors on {first.device}")


def _sized_workspace(workspace, n, device):
    """The caller's workspace if it holds n bytes, a new one if there is none."""
    if workspace is None:
        return torch.empty(n, dtype=torch.uint8, device=device)
    if not workspace.is_cuda or not workspace.is_contiguous() or workspace.numel() * workspace.element_size() < n:
        raise ValueError(f"workspace must be a contiguous device tensor of at least {n} bytes")
    return workspace


def flashrnn_embedding_workspace_bytes(tokens, vocab, width):
    """Bytes of workspace of the gradient for this many tokens, words and columns."""
    d = flashrnn_embedding_desc_t(int(tokens), int(vocab), int(width), FLASHRNN_F32, FLASHRNN_F32, FLASHRNN_I64, 1.0)
    return lib().flashrnn_embedding_workspace_bytes(ctypes.byref(d))


def flashrnn_embedding_fwd(table, tokens, scale=1.0, dtype=None, out=None, stream=None):
    """out[..., :] = scale * table[tokens[...], :], in the table's type or in `dtype`.  table[vocab, width] bf16 or f32, tokens of any shape, int64 or int32;
    tokens outside the vocabulary give zeros."""
    if stream is not None:   # (what is allocated here belongs to that stream, too)
        with torch.cuda.stream(stream):
            return flashrnn_embedding_fwd(table, tokens, scale, dtype, out)
    if _native is not None and out is not None:
        rc = _native.embedding_fwd(table, tokens, scale, out)
        if rc <= 0:
            return _done(rc, "flashrnn_embedding_fwd", out)
    V, H = table.shape
    dtype = (table.dtype if dtype is None else dtype) if out is None else out.dtype
    _chk(table, (V, H), table.dtype, "table")
    _chk(tokens, tokens.shape, tokens.dtype, "tokens")
    if out is None:
        out = torch.empty((*tokens.shape, H), dtype=dtype, device=table.device)
    _chk(out, (*tokens.shape, H), dtype, "out")
    _same_device(table, tokens=tokens, out=out)
    d = flashrnn_embedding_desc_t(tokens.numel(), V, H, _io_dtype(table), _io_dtype(out), _index_dtype(tokens), float(scale))
    rc = lib().flashrnn_embedding_fwd(ctypes.byref(d), _ptr(table), _ptr(tokens), _ptr(out), _stream(None))
    if rc != FLASHRNN_OK:
        raise FlashRNNError(rc, "flashrnn_embedding_fwd")
    return out


def flashrnn_embedding_bwd(tokens, dout, vocab, scale=1.0, dtable=None, accumulate=False, workspace=None, stream=None):
    """dtable[v] = scale * sum of dout over the places of word v; dtable[vocab, width] f32.  accumulate: added to the dtable passed in, rows of words that do not
    occur untouched.  The same result on every run."""
    if stream is not None:   # (what is allocated here belongs to that stream, too)
        with torch.cuda.stream(stream):
            return flashrnn_embedding_bwd(tokens, dout, vocab, scale, dtable, accumulate, workspace)
    if _native is not None and dtable is not None:
        rc = _native.embedding_bwd(tokens, dout, vocab, scale, dtable, accumulate, workspace)
        if rc <= 0:
            return _done(rc, "flashrnn_embedding_bwd", dtable)
    H = dout.shape[-1]
    _chk(dout, (*tokens.shape, H), dout.dtype, "dout")
    _chk(tokens, tokens.shape, tokens.dtype, "tokens")
    if dtable is None:
        if accumulate:
            raise ValueError("dtable is required to accumulate into")
        dtable = torch.empty((int(vocab), H), dtype=torch.float32, device=dout.device)
    _chk(dtable, (int(vocab), H), torch.float32, "dtable")
    _same_device(dout, tokens=tokens, dtable=dtable, workspace=workspace)
    d = flashrnn_embedding_desc_t(tokens.numel(), int(vocab), H, FLASHRNN_F32, _io_dtype(dout), _index_dtype(tokens), float(scale))
    n = lib().flashrnn_embedding_workspace_bytes(ctypes.byref(d))
    workspace = _sized_workspace(workspace, n, dout.device)
    rc = lib().flashrnn_embedding_bwd(ctypes.byref(d), _ptr(tokens), _ptr(dout), _ptr(dtable), int(bool(accumulate)), _ptr(workspace), _stream(None))
    if rc != FLASHRNN_OK:
        raise FlashRNNError(rc, "flashrnn_embedding_bwd")
    return dtable


def _rows_of(x, inner):
    """(outer, inner, stride): x's leading axes as `outer` blocks of dense rows, `stride` elements apart; `inner` trailing axes are a row."""
    width = 1
    for n, step in zip(reversed(x.shape[-inner:]), reversed(x.stride()[-inner:])):
        if n != 1 and step != width:
            raise ValueError("the rows of x must be dense")
        width *= n
    outer, dense, stride, first = 1, 1, 0, True   # (from the last axis: dense so far, then one strided axis, then nothing but its continuation)
    for n, step in zip(reversed(x.shape[:-inner]), reversed(x.stride()[:-inner])):
        if n == 1:
            continue
        if first and step == dense * width:
            dense *= n
        elif first:
            outer, stride, first = n, step, False
        elif step == stride * outer:
            outer *= n
        else:
            raise ValueError("x must be dense but for one of its leading axes")
    return (0, 0, 0) if x.numel() == 0 else (outer, dense, stride)


def _norm_desc(x, weight, bias, io, dx, eps):
    if not x.is_cuda:
        raise ValueError("x must be a device tensor")
    params = weight if weight is not None else bias
    if params is None:
        groups, width, shape = 1, x.shape[-1], None
    else:
        shape = tuple(params.shape)
        if len(shape) not in (1, 2) or tuple(x.shape[-len(shape):]) != shape:
            raise ValueError(f"weight and bias are [D] or [NH, D], the last axes of x: got {shape} for x {tuple(x.shape)}")
        groups, width = (1, *shape)[-2:]
        for t, name in ((weight, "weight"), (bias, "bias")):
            _chk(t, shape, params.dtype, name, optional=True)
    outer, inner, stride = _rows_of(x, 1 if shape is None else len(shape))
    return flashrnn_layer_norm_desc_t(outer, inner, stride, groups, width, _io_dtype(x), _io_dtype(io), _io_dtype(dx), FLASHRNN_F32 if params is None else _io_dtype(params), float(eps))


def flashrnn_layer_norm_fwd(x, weight=None, bias=None, eps=1e-5, dtype=None, save_for_backward=True, y=None, mean=None, rstd=None, stream=None):
    """Layer norm over the last axis of x, in x's type or in `dtype`.  weight, bias: [D], or [NH, D] for x[..., NH, D] (head by head), or None.  x may have one leading
    axis that is not dense, as the hidden states states[1:, 0] of a flashrnn_fwd call; y may be a dense x, of its own type.  Returns (y, mean, rstd), the last two f32 of x.shape[:-1], or None, None."""
    if stream is not None:   # (what is allocated here belongs to that stream, too)
        with torch.cuda.stream(stream):
            return flashrnn_layer_norm_fwd(x, weight, bias, eps, dtype, save_for_backward, y, mean, rstd)
    if _native is not None and y is not None and (mean is not None and rstd is not None or not save_for_backward):
        if not save_for_backward:
            mean = rstd = None
        rc = _native.layer_norm_fwd(x, weight, bias, eps, y, mean, rstd)
        if rc <= 0:
            return _done(rc, "flashrnn_layer_norm_fwd", (y, mean, rstd))
    if y is None:
        y = torch.empty(x.shape, dtype=x.dtype if dtype is None else dtype, device=x.device)
    _chk(y, x.shape, y.dtype, "y")
    if save_for_backward:
        mean = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device) if mean is None else mean
        rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device) if rstd is None else rstd
        _chk(mean, x.shape[:-1], torch.float32, "mean")
        _chk(rstd, x.shape[:-1], torch.float32, "rstd")
    else:
        mean = rstd = None
    _same_device(x, weight=weight, bias=bias, y=y, mean=mean, rstd=rstd)
    d = _norm_desc(x, weight, bias, y, y, eps)
    rc = lib().flashrnn_layer_norm_fwd(ctypes.byref(d), _ptr(x), _ptr(weight), _ptr(bias), _ptr(y), _ptr(mean), _ptr(rstd), _stream(None))
    if rc != FLASHRNN_OK:
        raise FlashRNNError(rc, "flashrnn_layer_norm_fwd")
    return y, mean, rstd


def flashrnn_layer_norm_bwd(dy, x, mean, rstd, weight=None, dtype=None, param_grads=True, out=None, workspace=None, stream=None):
    """Gradient of flashrnn_layer_norm_fwd.  Returns (dx, dweight, dbias): dx dense, in dy's type or in `dtype`; the others f32 in weight's shape ([D] without a weight), or None
    where param_grads is false.  `out` may pass preallocated (dx, dweight, dbias); dx may be dy, or a dense x, of its own type."""
    if stream is not None:   # (what is allocated here belongs to that stream, too)
        with torch.cuda.stream(stream):
            return flashrnn_layer_norm_bwd(dy, x, mean, rstd, weight, dtype, param_grads, out, workspace)
    if _native is not None and out is not None:
        dx, dweight, dbias = out if param_grads else (out[0], None, None)
        rc = _native.layer_norm_bwd(dy, x, mean, rstd, weight, dx, dweight, dbias, workspace)
        if rc <= 0:
            return _done(rc, "flashrnn_layer_norm_bwd", (dx, dweight, dbias))
    _chk(dy, x.shape, dy.dtype, "dy")
    _chk(mean, x.shape[:-1], torch.float32, "mean")
    _chk(rstd, x.shape[:-1], torch.float32, "rstd")
    shape = x.shape[-1:] if weight is None else weight.shape
    if out is None:
        dx = torch.empty(x.shape, dtype=dy.dtype if dtype is None else dtype, device=x.device)
        dweight, dbias = (torch.empty(shape, dtype=torch.float32, device=x.device) if param_grads else None for _ in range(2))
    else:
        dx, dweight, dbias = out
        if not param_grads:
            dweight = dbias = None
    _chk(dx, x.shape, dx.dtype, "dx")
    _chk(dweight, shape, torch.float32, "dweight", optional=True)
    _chk(dbias, shape, torch.float32, "dbias", optional=True)
    _same_device(x, dy=dy, mean=mean, rstd=rstd, weight=weight, dx=dx, dweight=dweight, dbias=dbias, workspace=workspace)
    d = _norm_desc(x, weight, None, dy, dx, 0.0)
    if dweight is not None or dbias is not None:
        workspace = _sized_workspace(workspace, lib().flashrnn_layer_norm_workspace_bytes(ctypes.byref(d)), x.device)
    rc = lib().flashrnn_layer_norm_bwd(ctypes.byref(d), _ptr(dy), _ptr(x), _ptr(weight), _ptr(mean), _ptr(rstd), _ptr(dx), _ptr(dweight), _ptr(dbias), _ptr(workspace),
                                       _stream(None))
    if rc != FLASHRNN_OK:
        raise FlashRNNError(rc, "flashrnn_layer_norm_bwd")
    return dx, dweight, dbias


def _matrix(t, shape, dtype, name):
    """The distance of the rows of a matrix whose rows are dense."""
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or not t.is_cuda:
        raise ValueError(f"{name}: got {tuple(t.shape)} {t.dtype} on {t.device}, expected a device tensor {tuple(shape)} {dtype}")
    rows, columns = shape
    if columns > 1 and t.stride(1) != 1 or rows > 1 and t.stride(0) < columns:
        raise ValueError(f"the rows of {name} must be dense and must not overlap")
    return max(t.stride(0), columns) if rows > 1 else columns


def flashrnn_cross_entropy(logits, targets, dloss=None, grad_scale=1.0, gradient=True, loss=None, lse=None, dlogits=None, stream=None):
    """Cross entropy of every row of logits[rows, classes] against targets[rows] (int64 or int32; outside the classes: ignored, loss 0), and in the same pass the
    gradient of sum(grad_scale * dloss * loss).  dlogits may be `logits` itself; lse, where passed, takes the rows' log of the sum of exponentials.
    Returns (loss f32[rows], dlogits in logits' type, or None where gradient is false)."""
    if stream is not None:   # (what is allocated here belongs to that stream, too)
        with torch.cuda.stream(stream):
            return flashrnn_cross_entropy(logits, targets, dloss, grad_scale, gradient, loss, lse, dlogits)
    if _native is not None and loss is not None and (dlogits is not None or not gradient):
        if not gradient:
            dlogits = None
        rc = _native.cross_entropy(logits, targets, dloss, grad_scale, loss, lse, dlogits)
        if rc <= 0:
            return _done(rc, "flashrnn_cross_entropy", (loss, dlogits))
    N, V = logits.shape
    stride = _matrix(logits, (N, V), logits.dtype, "logits")
    _chk(targets, (N,), targets.dtype, "targets")
    _chk(dloss, (N,), torch.float32, "dloss", optional=True)
    _chk(lse, (N,), torch.float32, "lse", optional=True)
    if loss is None:
        loss = torch.empty(N, dtype=torch.float32, device=logits.device)
    _chk(loss, (N,), torch.float32, "loss")
    if not gradient:
        dlogits = None
    elif dlogits is None:
        dlogits = torch.empty((N, V), dtype=logits.dtype, device=logits.device)
    to_stride = V if dlogits is None else _matrix(dlogits, (N, V), logits.dtype, "dlogits")
    _same_device(logits, targets=targets, dloss=dloss, loss=loss, lse=lse, dlogits=dlogits)
    d = flashrnn_cross_entropy_desc_t(N, stride, to_stride, V, _io_dtype(logits), _index_dtype(targets), float(grad_scale))
    rc = lib().flashrnn_cross_entropy(ctypes.byref(d), _ptr(logits), _ptr(targets), _ptr(dloss), _ptr(loss), _ptr(lse), _ptr(dlogits), _stream(None))
    if rc != FLASHRNN_OK:
        raise FlashRNNError(rc, "flashrnn_cross_entropy")
    return loss, dlogits


def flashrnn_grad_clip(grads, max_norm, out=None, norm=None, workspace=None, stream=None):
    """The norm over all values of the tensors in `grads` (bf16 or f32, any mix), and the tensors scaled down so that it is max_norm at most: in place, or into the
    tensors of `out`.  max_norm = inf computes the norm alone (and copies into `out`).  Returns norm f32[1]."""
    if stream is not None:   # (what is allocated here belongs to that stream, too)
        with torch.cuda.stream(stream):
            return flashrnn_grad_clip(grads, max_norm, out, norm, workspace)
    if _native is not None and norm is not None:
        rc = _native.grad_clip(grads, max_norm, out, norm, workspace, out is not None or max_norm != float("inf"))
        if rc <= 0:
            return _done(rc, "flashrnn_grad_clip", norm)
    grads = list(grads)
    n = len(grads)
    to = grads if out is None else list(out)
    if len(to) != n:
        raise ValueError(f"{n} gradients, {len(to)} tensors for them")
    if norm is None:
        if n == 0:
            raise ValueError("norm is required where there are no gradients")
        norm = torch.empty(1, dtype=torch.float32, device=grads[0].device)
    _chk(norm, (1,), torch.float32, "norm")
    _same_device(norm, workspace=workspace)
    for i, (g, o) in enumerate(zip(grads, to)):
        _chk(g, g.shape, g.dtype, f"grads[{i}]")
        if o is not g:
            _chk(o, g.shape, g.dtype, f"out[{i}]")
        _same_device(norm, grads=g, out=o)
    workspace = _sized_workspace(workspace, lib().flashrnn_grad_clip_workspace_bytes(n), norm.device)
    vp = ctypes.c_void_p * n
    ins = vp(*[g.data_ptr() for g in grads])
    outs = None if out is None and max_norm == float("inf") else vp(*[o.data_ptr() for o in to])
    rc = lib().flashrnn_grad_clip(n, ins, outs, (ctypes.c_longlong * n)(*[g.numel() for g in grads]), (ctypes.c_int * n)(*[_io_dtype(g) for g in grads]), float(max_norm),
                                  _ptr(norm), _ptr(workspace), _stream(None))
    if rc != FLASHRNN_OK:
        raise FlashRNNError(rc, "flashrnn_grad_clip")
    return norm
