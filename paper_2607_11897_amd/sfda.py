"""Thin Python binding of libsfda (ctypes).  Argument marshalling only: every step of the
computation runs in the HIP kernels behind the C ABI declared in include/sfda.h.

Tensors are torch tensors on the GPU, contiguous, with complex values stored as a trailing
axis of 2 (re, im) -- float32 (``torch.view_as_real`` of complex64 gives this layout) or
bfloat16.  torch is used for device memory and streams only.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from typing import Optional, Tuple

HERE = os.path.dirname(os.path.abspath(__file__))
# the in-tree build; SFDA_LIBRARY names another build to load (the sanitizer pass uses it)
LIB_PATH = os.environ.get("SFDA_LIBRARY") or os.path.join(HERE, "libsfda.so")

SFDA_F32, SFDA_BF16 = 0, 1
STATUS = {0: "SFDA_OK", 1: "SFDA_ERR_NULL", 2: "SFDA_ERR_SHAPE", 3: "SFDA_ERR_CHUNK",
          4: "SFDA_ERR_DTYPE", 5: "SFDA_ERR_ALIGN", 6: "SFDA_ERR_ALIAS", 7: "SFDA_ERR_HIP",
          8: "SFDA_ERR_SCRATCH"}
NOALLOC_SCRATCH_BYTES = 32 * 1024 * 1024      # SFDA_NOALLOC_SCRATCH_BYTES
EXPORTS = ("sfda_chunk_fwd", "sfda_chunk_fwd_sliced", "sfda_chunk_fwd_gated", "sfda_chunk_fwd_decoupled",
           "sfda_chunk_fwd_factored", "sfda_chunk_fwd_decoupled_factored",
           "sfda_chunk_fwd_factored_workspace_bytes", "sfda_chunk_fwd_segmented", "sfda_chunk_fwd_segmented_noalloc",
           "sfda_chunk_fwd_segmented_workspace_bytes", "sfda_chunk_fwd_auto_segments",
           "sfda_chunk_bwd", "sfda_chunk_bwd_workspace_bytes",
           "sfda_chunk_bwd_auto_workspace_bytes", "sfda_chunk_fwd_auto_factored",
           "sfda_chunk_solve_monitor",
           "sfda_step", "sfda_status_string", "sfda_abi_version",
           "sfda_rotary", "sfda_decay_attn_fwd", "sfda_decay_attn_fwd_workspace_bytes", "sfda_decay_attn_bwd",
           "sfda_decay_attn_bwd_workspace_bytes", "sfda_decay_attn_step", "sfda_group_norm", "sfda_group_norm_bwd",
           "sfda_group_norm_bwd_workspace_bytes",
           "sfda_rotary_axes", "sfda_delta_attn_fwd", "sfda_delta_attn_fwd_workspace_bytes", "sfda_delta_attn_bwd",
           "sfda_delta_attn_bwd_workspace_bytes", "sfda_delta_attn_step", "sfda_layer_norm", "sfda_layer_norm_bwd",
           "sfda_layer_norm_bwd_workspace_bytes")

_lib = None


class SfdaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = load_library().sfda_status_string(status).decode()
        super().__init__(f"{where}: {STATUS.get(status, status)} ({msg})")


@contextlib.contextmanager
def library(path: str):
    """Run the binding against another build of the library at `path` (the LDS-poison
    debug build in its test) for the duration of a with-block, then go back to the one
    loaded before.  Nothing may be in flight on the device when the block ends."""
    global _lib
    saved = _lib
    _lib = None
    try:
        yield load_library(path)
    finally:
        _lib = saved


def load_library(path: str = LIB_PATH):
    """Load libsfda.so; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"libsfda.so not found at {path}: build it with "
                           "`python -m paper_2607_11897_amd.build` (no CPU fallback exists)")
    lib = ctypes.CDLL(path)
    vp, i = ctypes.c_void_p, ctypes.c_int
    lib.sfda_chunk_fwd.argtypes = [vp] * 9 + [i] * 6 + [i, i, vp]
    lib.sfda_chunk_fwd.restype = i
    lib.sfda_chunk_fwd_sliced.argtypes = [vp] * 9 + [i] * 7 + [i, i, vp]
    lib.sfda_chunk_fwd_sliced.restype = i
    f = ctypes.c_float
    lib.sfda_chunk_fwd_gated.argtypes = [vp] * 9 + [i] * 6 + [f] * 4 + [i, i, vp]
    lib.sfda_chunk_fwd_gated.restype = i
    lib.sfda_chunk_fwd_decoupled.argtypes = [vp] * 11 + [i] * 6 + [i, i, vp]
    lib.sfda_chunk_fwd_decoupled.restype = i
    lib.sfda_chunk_fwd_factored.argtypes = [vp] * 9 + [i] * 6 + [i, i, vp, ctypes.c_size_t, vp]
    lib.sfda_chunk_fwd_factored.restype = i
    lib.sfda_chunk_fwd_decoupled_factored.argtypes = [vp] * 11 + [i] * 6 + [i, i, vp, ctypes.c_size_t, vp]
    lib.sfda_chunk_fwd_decoupled_factored.restype = i
    lib.sfda_chunk_fwd_factored_workspace_bytes.argtypes = [i] * 7
    lib.sfda_chunk_fwd_factored_workspace_bytes.restype = ctypes.c_size_t
    lib.sfda_chunk_fwd_segmented.argtypes = [vp] * 9 + [i] * 7 + [i, i, vp, ctypes.c_size_t, vp]
    lib.sfda_chunk_fwd_segmented.restype = i
    lib.sfda_chunk_fwd_segmented_noalloc.argtypes = [vp] * 9 + [i] * 7 + [i, i, vp]
    lib.sfda_chunk_fwd_segmented_noalloc.restype = i
    lib.sfda_chunk_fwd_segmented_workspace_bytes.argtypes = [i] * 7
    lib.sfda_chunk_fwd_segmented_workspace_bytes.restype = ctypes.c_size_t
    lib.sfda_chunk_fwd_auto_segments.argtypes = [i] * 7
    lib.sfda_chunk_solve_monitor.argtypes = [vp] * 6 + [i] * 5 + [vp]
    lib.sfda_chunk_solve_monitor.restype = i
    lib.sfda_chunk_fwd_auto_segments.restype = i
    lib.sfda_chunk_bwd.argtypes = [vp] * 16 + [i] * 6 + [i, i, vp, ctypes.c_size_t, vp]
    lib.sfda_chunk_bwd.restype = i
    lib.sfda_chunk_bwd_workspace_bytes.argtypes = [i] * 6
    lib.sfda_chunk_bwd_workspace_bytes.restype = ctypes.c_size_t
    lib.sfda_chunk_fwd_auto_factored.argtypes = [i] * 8
    lib.sfda_chunk_fwd_auto_factored.restype = i
    lib.sfda_chunk_bwd_auto_workspace_bytes.argtypes = [i] * 7
    lib.sfda_chunk_bwd_auto_workspace_bytes.restype = ctypes.c_size_t
    lib.sfda_step.argtypes = [vp] * 8 + [i] * 4 + [i, i, vp]
    lib.sfda_step.restype = i
    sz, ll = ctypes.c_size_t, ctypes.c_longlong
    lib.sfda_rotary.argtypes = [vp] * 5 + [i, ll, ll] + [vp] * 2 + [i] * 9 + [vp, i, vp]
    lib.sfda_decay_attn_fwd.argtypes = [vp] * 8 + [i] * 5 + [f, vp, i, vp, sz, vp]
    lib.sfda_decay_attn_bwd.argtypes = [vp] * 12 + [i] * 5 + [f, vp, i, vp, sz, vp]
    lib.sfda_decay_attn_step.argtypes = [vp] * 6 + [i] * 4 + [f, vp, i, vp]
    lib.sfda_group_norm.argtypes = [vp] * 5 + [i] * 5 + [f, vp, i, vp]
    lib.sfda_group_norm_bwd.argtypes = [vp] * 9 + [i] * 5 + [f, vp, i, vp, sz, vp]
    lib.sfda_rotary_axes.argtypes = [vp] * 5 + [i, ll, ll] + [vp] + [i] * 2 + [vp] * 2 + [i] * 8 + [vp, i, vp]
    lib.sfda_delta_attn_fwd.argtypes = [vp] * 9 + [i] * 6 + [f, vp, i, vp, sz, vp]
    lib.sfda_delta_attn_bwd.argtypes = [vp] * 15 + [i] * 6 + [f, vp, i, vp, sz, vp]
    lib.sfda_delta_attn_step.argtypes = [vp] * 7 + [i] * 5 + [f, vp, i, vp]
    lib.sfda_layer_norm.argtypes = [vp] * 6 + [i] * 3 + [f, vp, i, vp]
    lib.sfda_layer_norm_bwd.argtypes = [vp] * 7 + [i] * 3 + [f, vp, i, vp, sz, vp]
    for fn in (lib.sfda_rotary, lib.sfda_decay_attn_fwd, lib.sfda_decay_attn_bwd, lib.sfda_decay_attn_step,
               lib.sfda_group_norm, lib.sfda_group_norm_bwd, lib.sfda_rotary_axes, lib.sfda_delta_attn_fwd,
               lib.sfda_delta_attn_bwd, lib.sfda_delta_attn_step, lib.sfda_layer_norm, lib.sfda_layer_norm_bwd):
        fn.restype = i
    for fn, n in ((lib.sfda_delta_attn_fwd_workspace_bytes, 6), (lib.sfda_delta_attn_bwd_workspace_bytes, 7),
                  (lib.sfda_layer_norm_bwd_workspace_bytes, 4)):
        fn.argtypes = [i] * n
        fn.restype = sz
    for fn in (lib.sfda_decay_attn_fwd_workspace_bytes, lib.sfda_decay_attn_bwd_workspace_bytes,
               lib.sfda_group_norm_bwd_workspace_bytes):
        fn.argtypes = [i] * (5 if fn is lib.sfda_group_norm_bwd_workspace_bytes else 6)
        fn.restype = sz
    lib.sfda_status_string.argtypes = [i]
    lib.sfda_status_string.restype = ctypes.c_char_p
    lib.sfda_abi_version.restype = i
    _lib = lib
    return lib


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.float32:
        return SFDA_F32
    if t.dtype == torch.bfloat16:
        return SFDA_BF16
    raise TypeError(f"unsupported dtype {t.dtype} (float32 or bfloat16)")


def _check(named: dict) -> None:
    """Every given tensor has its expected shape and sits on the first tensor's GPU: the
    library receives bare pointers and sizes, so a short buffer or a host pointer would
    only show up as a fault inside a kernel.  `named` maps a name to (tensor or None,
    expected shape)."""
    # one pass where everything is as it should be (a call of a microsecond's kernel is bound by
    # what happens here); whatever is not is named by the passes below
    index = None
    for t, shape in named.values():
        if t is None:
            continue
        if index is None:
            index = t.get_device()
        if t.shape != shape or not t.is_cuda or t.get_device() != index:
            break
    else:
        return
    dev = None
    for name, (t, shape) in named.items():
        if t is None:
            continue
        if tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    for name, (t, _) in named.items():
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError(f"{name} must be a GPU tensor (got {t.device})")
        if dev is None:
            dev = t.device
        elif t.device != dev:
            raise ValueError(f"{name} is on {t.device}, the other tensors on {dev}")


def _need_f32(**named) -> None:
    """States (S0, S_T, dS_T, S) are complex float32 whatever the inputs' dtype: the library
    reads and writes m * n * 8 bytes per head there, so a half-width buffer would be
    overrun."""
    import torch
    for name, t in named.items():
        if t is not None and t.dtype != torch.float32:
            raise TypeError(f"{name} must be float32 (got {t.dtype})")


def _dims(q, v, nd):
    if q.dim() != nd or v.dim() != nd:
        raise ValueError(f"q and v must have {nd} dimensions")
    return q.shape


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous")
    return t.data_ptr()


def _stream(stream):
    import torch
    if stream is None:              # (torch.cuda.current_stream() builds a Stream: 2.7 us against 0.2)
        return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))
    return ctypes.c_void_p(stream.cuda_stream)


def _workspace(nbytes: int, device, stream):
    """A workspace from torch's allocator, owned by the stream it is used on (so that its memory
    is given to later work of that stream only)."""
    import torch
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    if not isinstance(stream, torch.cuda.Stream):       # any object with a cuda_stream handle
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _try_workspace(nbytes: int, device, stream):
    """_workspace, or None where the device's memory is full (the paths that need less run then)."""
    import torch
    try:
        return _workspace(nbytes, device, stream)
    except torch.OutOfMemoryError:
        return None


def chunk_fwd(q, k, v, alpha, theta, beta, S0=None, C: int = 64, *, o=None, S_T=None,
              out_dtype=None, want_state: bool = True, slice: Optional[int] = None,
              segments="auto", workspace=None, stream=None) -> Tuple:
    """SFDA chunkwise forward.  q, k: [B,H,T,m,2]; v: [B,H,T,n,2]; alpha, theta: [B,H,T,m];
    beta: [B,H,T] (all float32 or all bfloat16); S0: [B,H,m,n,2] float32 or None.
    Returns (o [B,H,T,n,2] in out_dtype, S_T [B,H,m,n,2] float32 or None).
    slice: value columns per workgroup (sfda_chunk_fwd_sliced); segments: G parallel
    segments per head (sfda_chunk_fwd_segmented; `workspace` a uint8 device tensor of at
    least segmented_workspace_bytes(...) bytes, allocated here when not given), None for one
    scan per head (sfda_chunk_fwd), or "auto" (the default, without a slice): sfda_chunk_fwd_factored
    where sfda_chunk_fwd_auto_factored says so, else the count sfda_chunk_fwd_auto_segments
    suggests: segments when the heads alone would leave most compute units idle.  Workspaces not
    given come from torch's allocator."""
    import torch
    lib = load_library()
    B, H, T, m, _ = _dims(q, v, 5)
    n = v.shape[3]
    in_code = _dtype_code(q)
    for t in (k, v, alpha, theta, beta):
        if t.dtype != q.dtype:
            raise TypeError("q, k, v, alpha, theta, beta must share one dtype")
    out_dtype = q.dtype if out_dtype is None else out_dtype
    if o is None:
        o = torch.empty((B, H, T, n, 2), dtype=out_dtype, device=q.device)
    if S_T is None and want_state:
        S_T = torch.empty((B, H, m, n, 2), dtype=torch.float32, device=q.device)
    _need_f32(S0=S0, S_T=S_T)
    _dtype_code(o)
    _check(dict(q=(q, (B, H, T, m, 2)), k=(k, (B, H, T, m, 2)), v=(v, (B, H, T, n, 2)),
                alpha=(alpha, (B, H, T, m)), theta=(theta, (B, H, T, m)), beta=(beta, (B, H, T)),
                S0=(S0, (B, H, m, n, 2)), o=(o, (B, H, T, n, 2)), S_T=(S_T, (B, H, m, n, 2)),
                workspace=(workspace, tuple(workspace.shape) if workspace is not None else ())))
    args = [_ptr(q), _ptr(k), _ptr(v), _ptr(alpha), _ptr(theta), _ptr(beta), _ptr(S0),
            _ptr(o), _ptr(S_T), B, H, T, m, n, C]
    if isinstance(segments, str):
        if segments != "auto":
            raise ValueError(f"segments must be an int, None or 'auto', not {segments!r}")
        segments = None
        nfac = 0
        # (a slice asks for sfda_chunk_fwd_sliced; a workspace the caller sized for segments keeps them)
        if workspace is None and slice is None and lib.sfda_chunk_fwd_auto_factored(B, H, T, m, n, C, in_code, 0):
            nfac = lib.sfda_chunk_fwd_factored_workspace_bytes(B, H, T, m, n, in_code, 0)
        ws = _try_workspace(nfac, q.device, stream) if nfac else None
        if ws is not None:
            st = lib.sfda_chunk_fwd_factored(*args, in_code, _dtype_code(o), _ptr(ws), nfac, _stream(stream))
            if st != 0:
                raise SfdaError(st, "sfda_chunk_fwd_factored")
            return o, S_T
        if slice is None and q.is_cuda:
            if q.get_device() == torch.cuda.current_device():
                G = int(lib.sfda_chunk_fwd_auto_segments(B, H, T, m, n, C, in_code))
            else:
                with torch.cuda.device(q.device):
                    G = int(lib.sfda_chunk_fwd_auto_segments(B, H, T, m, n, C, in_code))
            segments = G if G > 1 else None
    if segments is not None:
        nws = lib.sfda_chunk_fwd_segmented_workspace_bytes(B, H, T, m, n, segments, in_code)
        if workspace is None:
            workspace = _workspace(max(nws, 1), q.device, stream)
        st = lib.sfda_chunk_fwd_segmented(*args, segments, in_code, _dtype_code(o), _ptr(workspace),
                                          workspace.numel() * workspace.element_size(), _stream(stream))
        if st != 0:
            raise SfdaError(st, "sfda_chunk_fwd_segmented")
        return o, S_T
    if slice is None:
        st = lib.sfda_chunk_fwd(*args, in_code, _dtype_code(o), _stream(stream))
    else:
        st = lib.sfda_chunk_fwd_sliced(*args, slice, in_code, _dtype_code(o), _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_chunk_fwd")
    return o, S_T


def chunk_fwd_segmented_noalloc(q, k, v, alpha, theta, beta, S0=None, C: int = 64, *, segments: int,
                                o=None, S_T=None, out_dtype=None, want_state: bool = True,
                                stream=None) -> Tuple:
    """chunk_fwd with `segments` parallel segments per head whose workspace is the library's
    static scratch (sfda_chunk_fwd_segmented_noalloc: the call allocates no device memory;
    o and S_T are allocated here only when not given).  Shapes and results as chunk_fwd."""
    import torch
    lib = load_library()
    B, H, T, m, _ = _dims(q, v, 5)
    n = v.shape[3]
    in_code = _dtype_code(q)
    for t in (k, v, alpha, theta, beta):
        if t.dtype != q.dtype:
            raise TypeError("q, k, v, alpha, theta, beta must share one dtype")
    out_dtype = q.dtype if out_dtype is None else out_dtype
    if o is None:
        o = torch.empty((B, H, T, n, 2), dtype=out_dtype, device=q.device)
    if S_T is None and want_state:
        S_T = torch.empty((B, H, m, n, 2), dtype=torch.float32, device=q.device)
    _need_f32(S0=S0, S_T=S_T)
    _dtype_code(o)
    _check(dict(q=(q, (B, H, T, m, 2)), k=(k, (B, H, T, m, 2)), v=(v, (B, H, T, n, 2)),
                alpha=(alpha, (B, H, T, m)), theta=(theta, (B, H, T, m)), beta=(beta, (B, H, T)),
                S0=(S0, (B, H, m, n, 2)), o=(o, (B, H, T, n, 2)), S_T=(S_T, (B, H, m, n, 2))))
    st = lib.sfda_chunk_fwd_segmented_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(alpha), _ptr(theta), _ptr(beta),
                                              _ptr(S0), _ptr(o), _ptr(S_T), B, H, T, m, n, C, segments,
                                              in_code, _dtype_code(o), _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_chunk_fwd_segmented_noalloc")
    return o, S_T


def chunk_fwd_gated(q, k_raw, v, a, b, c, S0=None, C: int = 64, *, alpha_min: float,
                    alpha_max: float, theta_max: float, eps: float, o=None, S_T=None,
                    out_dtype=None, want_state: bool = True, stream=None) -> Tuple:
    """SFDA chunkwise forward on pre-activations (sfda_chunk_fwd_gated): alpha, theta, beta
    and the keys are formed inside the kernel from a, b [B,H,T,m], c [B,H,T] and the raw
    keys k_raw [B,H,T,m,2].  Shapes and results otherwise as chunk_fwd."""
    import torch
    lib = load_library()
    B, H, T, m, _ = _dims(q, v, 5)
    n = v.shape[3]
    in_code = _dtype_code(q)
    for t in (k_raw, v, a, b, c):
        if t.dtype != q.dtype:
            raise TypeError("q, k_raw, v, a, b, c must share one dtype")
    out_dtype = q.dtype if out_dtype is None else out_dtype
    if o is None:
        o = torch.empty((B, H, T, n, 2), dtype=out_dtype, device=q.device)
    if S_T is None and want_state:
        S_T = torch.empty((B, H, m, n, 2), dtype=torch.float32, device=q.device)
    _need_f32(S0=S0, S_T=S_T)
    _dtype_code(o)
    _check(dict(q=(q, (B, H, T, m, 2)), k_raw=(k_raw, (B, H, T, m, 2)), v=(v, (B, H, T, n, 2)),
                a=(a, (B, H, T, m)), b=(b, (B, H, T, m)), c=(c, (B, H, T)),
                S0=(S0, (B, H, m, n, 2)), o=(o, (B, H, T, n, 2)), S_T=(S_T, (B, H, m, n, 2))))
    st = lib.sfda_chunk_fwd_gated(_ptr(q), _ptr(k_raw), _ptr(v), _ptr(a), _ptr(b), _ptr(c), _ptr(S0),
                                  _ptr(o), _ptr(S_T), B, H, T, m, n, C, float(alpha_min),
                                  float(alpha_max), float(theta_max), float(eps), in_code,
                                  _dtype_code(o), _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_chunk_fwd_gated")
    return o, S_T


def chunk_fwd_decoupled(q, k, r, v, alpha, theta, eta, beta, S0=None, C: int = 32, *, o=None,
                        S_T=None, out_dtype=None, want_state: bool = True, stream=None) -> Tuple:
    """Write-decoupled forward (sfda_chunk_fwd_decoupled_factored, its workspace from torch's
    allocator): erase along k with strengths eta [B,H,T], write along r [B,H,T,m,2] with
    strengths beta [B,H,T].  Shapes and results otherwise as chunk_fwd."""
    import torch
    lib = load_library()
    B, H, T, m, _ = _dims(q, v, 5)
    n = v.shape[3]
    in_code = _dtype_code(q)
    for t in (k, r, v, alpha, theta, eta, beta):
        if t.dtype != q.dtype:
            raise TypeError("q, k, r, v, alpha, theta, eta, beta must share one dtype")
    out_dtype = q.dtype if out_dtype is None else out_dtype
    if o is None:
        o = torch.empty((B, H, T, n, 2), dtype=out_dtype, device=q.device)
    if S_T is None and want_state:
        S_T = torch.empty((B, H, m, n, 2), dtype=torch.float32, device=q.device)
    _need_f32(S0=S0, S_T=S_T)
    _dtype_code(o)
    _check(dict(q=(q, (B, H, T, m, 2)), k=(k, (B, H, T, m, 2)), r=(r, (B, H, T, m, 2)),
                v=(v, (B, H, T, n, 2)), alpha=(alpha, (B, H, T, m)), theta=(theta, (B, H, T, m)),
                eta=(eta, (B, H, T)), beta=(beta, (B, H, T)), S0=(S0, (B, H, m, n, 2)),
                o=(o, (B, H, T, n, 2)), S_T=(S_T, (B, H, m, n, 2))))
    args = [_ptr(q), _ptr(k), _ptr(r), _ptr(v), _ptr(alpha), _ptr(theta), _ptr(eta), _ptr(beta), _ptr(S0),
            _ptr(o), _ptr(S_T), B, H, T, m, n, C, in_code, _dtype_code(o)]
    ws = None
    if lib.sfda_chunk_fwd_auto_factored(B, H, T, m, n, C, in_code, 1):
        nws = lib.sfda_chunk_fwd_factored_workspace_bytes(B, H, T, m, n, in_code, 1)
        ws = _try_workspace(nws, q.device, stream)
    if ws is not None:
        st = lib.sfda_chunk_fwd_decoupled_factored(*args, _ptr(ws), nws, _stream(stream))
    else:
        st = lib.sfda_chunk_fwd_decoupled(*args, _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_chunk_fwd_decoupled")
    return o, S_T


def chunk_bwd(q, k, v, alpha, theta, beta, S0, dO, dS_T=None, C: int = 64, *,
              want_dS0: bool = True, workspace=None, stream=None) -> dict:
    """Gradients of a real loss through the chunkwise forward (sfda_chunk_bwd), given
    dO = dL/do [B,H,T,n,2] (o's dtype) and dS_T = dL/dS_T [B,H,m,n,2] float32 or None.
    Inputs as chunk_fwd.  Returns dq, dk, dv, dalpha, dtheta, dbeta in the inputs' dtype and
    dS0 (float32, or None without want_dS0); complex gradients are dL/dRe + i dL/dIm.
    `workspace`: a uint8 device tensor of at least bwd_workspace_bytes(...) bytes (fastest at
    bwd_auto_workspace_bytes(...), which is allocated here when none is given)."""
    import torch
    lib = load_library()
    B, H, T, m, _ = _dims(q, v, 5)
    n = v.shape[3]
    in_code = _dtype_code(q)
    for t in (k, v, alpha, theta, beta):
        if t.dtype != q.dtype:
            raise TypeError("q, k, v, alpha, theta, beta must share one dtype")
    _need_f32(S0=S0, dS_T=dS_T)
    _dtype_code(dO)
    _check(dict(q=(q, (B, H, T, m, 2)), k=(k, (B, H, T, m, 2)), v=(v, (B, H, T, n, 2)),
                alpha=(alpha, (B, H, T, m)), theta=(theta, (B, H, T, m)), beta=(beta, (B, H, T)),
                S0=(S0, (B, H, m, n, 2)), dO=(dO, (B, H, T, n, 2)), dS_T=(dS_T, (B, H, m, n, 2))))
    g = dict(dq=torch.empty_like(q), dk=torch.empty_like(k), dv=torch.empty_like(v),
             dalpha=torch.empty_like(alpha), dtheta=torch.empty_like(theta), dbeta=torch.empty_like(beta),
             dS0=torch.empty((B, H, m, n, 2), dtype=torch.float32, device=q.device) if want_dS0 else None)
    if workspace is None:
        nws = lib.sfda_chunk_bwd_auto_workspace_bytes(B, H, T, m, n, C, in_code)
        workspace = _try_workspace(max(nws, 1), q.device, stream)
        if workspace is None:
            nws = lib.sfda_chunk_bwd_workspace_bytes(B, H, T, m, n, C)
            workspace = _workspace(max(nws, 1), q.device, stream)
    else:
        _check(dict(q=(q, (B, H, T, m, 2)), workspace=(workspace, tuple(workspace.shape))))
    st = lib.sfda_chunk_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(alpha), _ptr(theta), _ptr(beta), _ptr(S0),
                            _ptr(dO), _ptr(dS_T), _ptr(g["dq"]), _ptr(g["dk"]), _ptr(g["dv"]),
                            _ptr(g["dalpha"]), _ptr(g["dtheta"]), _ptr(g["dbeta"]), _ptr(g["dS0"]),
                            B, H, T, m, n, C, in_code, _dtype_code(dO), _ptr(workspace),
                            workspace.numel() * workspace.element_size(), _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_chunk_bwd")
    return g


def bwd_workspace_bytes(B: int, H: int, T: int, m: int, n: int, C: int) -> int:
    return int(load_library().sfda_chunk_bwd_workspace_bytes(B, H, T, m, n, C))


def bwd_auto_workspace_bytes(B: int, H: int, T: int, m: int, n: int, C: int, dtype: str = "f32") -> int:
    """The workspace at which chunk_bwd is fastest (sfda_chunk_bwd_auto_workspace_bytes); dtype:
    the inputs' ("f32" or "bf16")."""
    code = {"f32": SFDA_F32, "bf16": SFDA_BF16}[dtype]
    return int(load_library().sfda_chunk_bwd_auto_workspace_bytes(B, H, T, m, n, C, code))


def chunk_solve_monitor(k, alpha, theta, beta, stream=None) -> Tuple:
    """The triangular solve of every 16-token block checked on its own
    (sfda_chunk_solve_monitor): returns (residual, lnorm), float32 [B, H, ceil(T / 16)],
    the max-abs entry of (I + D_beta L') N - I and ||D_beta L'||_F.  k: [B,H,T,m,2];
    alpha, theta: [B,H,T,m]; beta: [B,H,T] (float32 or bfloat16)."""
    import torch
    lib = load_library()
    if k.dim() != 5 or k.shape[-1] != 2:
        raise ValueError(f"k must be [B,H,T,m,2], not {tuple(k.shape)}")
    B, H, T, m = k.shape[0], k.shape[1], k.shape[2], k.shape[3]
    code = _dtype_code(k)
    for t in (alpha, theta, beta):
        if t.dtype != k.dtype:
            raise TypeError("k, alpha, theta, beta must share one dtype")
    _check(dict(k=(k, (B, H, T, m, 2)), alpha=(alpha, (B, H, T, m)), theta=(theta, (B, H, T, m)),
                beta=(beta, (B, H, T))))
    nb = (T + 15) // 16
    residual = torch.empty((B, H, nb), dtype=torch.float32, device=k.device)
    lnorm = torch.empty((B, H, nb), dtype=torch.float32, device=k.device)
    st = lib.sfda_chunk_solve_monitor(_ptr(k), _ptr(alpha), _ptr(theta), _ptr(beta), _ptr(residual),
                                      _ptr(lnorm), B, H, T, m, code, _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_chunk_solve_monitor")
    return residual, lnorm


def auto_segments(B: int, H: int, T: int, m: int, n: int, C: int = 64, dtype: str = "f32") -> int:
    """sfda_chunk_fwd_auto_segments on the current device (1: one scan per head); dtype: the
    inputs' ("f32" or "bf16")."""
    code = {"f32": SFDA_F32, "bf16": SFDA_BF16}[dtype]
    return int(load_library().sfda_chunk_fwd_auto_segments(B, H, T, m, n, C, code))


def segmented_workspace_bytes(B: int, H: int, T: int, m: int, n: int, G: int, dtype: str = "f32") -> int:
    """Workspace of sfda_chunk_fwd_segmented; dtype: the inputs' ("f32" or "bf16")."""
    code = {"f32": SFDA_F32, "bf16": SFDA_BF16}[dtype]
    return int(load_library().sfda_chunk_fwd_segmented_workspace_bytes(B, H, T, m, n, G, code))


def step(q, k, v, alpha, theta, beta, S, *, o=None, out_dtype=None, stream=None):
    """One decode token per head.  q, k: [B,H,m,2]; v: [B,H,n,2]; alpha, theta: [B,H,m];
    beta: [B,H]; S: [B,H,m,n,2] float32, updated in place.  Returns o [B,H,n,2]."""
    import torch
    lib = load_library()
    B, H, m, _ = _dims(q, v, 4)
    n = v.shape[2]
    in_code = _dtype_code(q)
    for t in (k, v, alpha, theta, beta):
        if t.dtype != q.dtype:
            raise TypeError("q, k, v, alpha, theta, beta must share one dtype")
    _need_f32(S=S)
    out_dtype = q.dtype if out_dtype is None else out_dtype
    if o is None:
        o = torch.empty((B, H, n, 2), dtype=out_dtype, device=q.device)
    _dtype_code(o)
    _check(dict(q=(q, (B, H, m, 2)), k=(k, (B, H, m, 2)), v=(v, (B, H, n, 2)), alpha=(alpha, (B, H, m)),
                theta=(theta, (B, H, m)), beta=(beta, (B, H)), S=(S, (B, H, m, n, 2)), o=(o, (B, H, n, 2))))
    st = lib.sfda_step(_ptr(q), _ptr(k), _ptr(v), _ptr(alpha), _ptr(theta), _ptr(beta),
                       _ptr(S), _ptr(o), B, H, m, n, in_code, _dtype_code(o), _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_step")
    return o


# ------------------------------------------------------------------ operators around the attention
# Activations may have any strides with a contiguous last axis; float32 states, tables and weights are contiguous.

_ACT = {"none": 0, "silu": 1}
_STRIDES = {n: ctypes.c_longlong * n for n in (7, 8, 12, 18, 21, 33)}


def _rows(t) -> Optional[int]:
    """The pointer of an activation whose last axis is contiguous."""
    if t is None:
        return None
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError("the last axis of an activation must be contiguous")
    return t.data_ptr()


def _fit(*pairs) -> None:
    """_check of (name, tensor or None, shape) triples; in one pass where everything is as it should be."""
    index = pairs[0][1].get_device()
    if index >= 0:
        for _, t, shape in pairs:
            if t is not None and (t.shape != shape or t.get_device() != index):
                break
        else:
            return
    _check({name: (t, shape) for name, t, shape in pairs})


def _same_dtype(x, **named) -> int:
    code = _dtype_code(x)
    for name, t in named.items():
        if t is not None and t.dtype != x.dtype:
            raise TypeError(f"{name} must be {x.dtype} as the other activations (got {t.dtype})")
    return code


def _int32(name, t) -> None:
    import torch
    if t is not None and t.dtype != torch.int32:
        raise TypeError(f"{name} must be int32 (got {t.dtype})")


def _strides(outer: int, *tensors):
    """The strides of the outer axes, tensor after tensor, or None where all of them are contiguous."""
    for t in tensors:
        if not t.is_contiguous():
            return _STRIDES[outer * len(tensors)](*[s for t in tensors for s in t.stride()[:outer]])
    return None


def _empty(shape, dtype, device, stream):
    """An output, from the memory of the stream that writes it."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _empty_as(x, shape, stream):
    """An output of x's type and a shape of its own or x's."""
    import torch
    if stream is None and x.shape == shape and x.is_contiguous():
        return torch.empty_like(x)
    return _empty(shape, x.dtype, x.device, stream)


def rotary_tables(positions: int, rot: int, *, base: float = 10000.0, scaling: Optional[dict] = None, device="cuda"):
    """The tables of `rotary`: cos and sin [positions, rot / 2] float32 of position * frequency, formed in
    float64, frequency_i = base^(-2i / rot).  `scaling` stretches them past the length L that a
    model was trained at, by a factor s:
      dict(kind="linear", factor=s)              positions divided by s
      dict(kind="ntk", factor=s)                 base * s^(rot / (rot - 2)): the fastest pair keeps its frequency,
                                                 the slowest is divided by s
      dict(kind="yarn", factor=s, length=L, fast=32, slow=1, amplitude=None)
                                                 pairs that turn more than `fast` times over L keep their frequency,
                                                 those that turn less than `slow` times are divided by s, linear in the
                                                 pair's number between (from the whole number below the pair of `fast`
                                                 turns to the one above that of `slow`, rot - 1 at most); both tables
                                                 times the amplitude (0.1 log s + 1 if None)."""
    import math
    import torch
    if rot < 2 or rot % 2 or positions < 1:
        raise ValueError(f"rot must be even and at least 2, positions at least 1 (got {rot}, {positions})")
    pair = torch.arange(rot // 2, dtype=torch.float64)
    freq = base ** (-2.0 * pair / rot)
    amplitude = 1.0
    if scaling is not None:
        kind, s = scaling["kind"], float(scaling["factor"])
        if not s > 0:
            raise ValueError(f"the factor must be positive (got {s})")
        if kind == "linear":
            freq = freq / s
        elif kind == "ntk":
            if rot < 4:
                raise ValueError("ntk scaling needs at least two pairs")
            freq = (base * s ** (rot / (rot - 2))) ** (-2.0 * pair / rot)
        elif kind == "yarn":
            length = float(scaling["length"])
            # the (fractional) pair that turns n times over the length
            at = lambda n: rot * math.log(length / (2 * math.pi * n)) / (2 * math.log(base))  # noqa: E731
            low = max(math.floor(at(float(scaling.get("fast", 32)))), 0)
            # (an end past the last pair stays there: that pair turns more than `slow` times and is divided in part only)
            high = min(math.ceil(at(float(scaling.get("slow", 1)))), rot - 1)
            keep = 1.0 - ((pair - low) / max(high - low, 1e-3)).clamp(0.0, 1.0)
            freq = freq * keep + freq / s * (1.0 - keep)
            amplitude = scaling.get("amplitude")
            amplitude = (0.1 * math.log(s) + 1.0 if s > 1 else 1.0) if amplitude is None else float(amplitude)
        else:
            raise ValueError(f"scaling must be linear, ntk or yarn, not {kind!r}")
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * freq
    return tuple((amplitude * t).to(torch.float32).to(device) for t in (angle.cos(), angle.sin()))


def rotary(q, k, cos, sin, positions=None, *, offset: int = 0, interleaved: bool = False, inverse: bool = False,
           q_out=None, k_out=None, stream=None) -> Tuple:
    """Queries and keys turned by their tokens' positions (sfda_rotary).  q: [B,Hq,T,D]; k: [B,Hk,T,D] or None (float32 or
    bfloat16, any strides with a contiguous last axis); cos, sin: [P, rot / 2] float32 (rotary_tables): the first
    rot channels turn, as pairs (i, i + rot / 2) or, interleaved, (2i, 2i + 1); positions: int32 or int64 [T] or [B,T],
    else offset, offset + 1, ....  inverse turns back: the gradient of the outputs becomes that of the inputs.
    Returns (q_out, k_out), new contiguous tensors if not given; q_out=q, k_out=k turns in place."""
    import torch
    lib = load_library()
    if q.dim() != 4 or cos.dim() != 2:
        raise ValueError("q must be [B,H,T,D] and cos [P, rot / 2]")
    B, Hq, T, D = q.shape
    Hk = 0 if k is None else k.shape[1]
    code = _same_dtype(q, k=k, q_out=q_out, k_out=k_out)
    _need_f32(cos=cos, sin=sin)
    P, half = cos.shape
    tq, tk = (B, Hq, T, D), (B, Hk, T, D)
    if q_out is None:
        q_out = _empty_as(q, tq, stream)
    if k is None:
        k_out = None
    elif k_out is None:
        k_out = _empty_as(k, tk, stream)
    bits, pstride = 0, 0
    if positions is not None:
        if positions.dtype not in (torch.int32, torch.int64):
            raise TypeError(f"positions must be int32 or int64 (got {positions.dtype})")
        bits = 32 if positions.dtype == torch.int32 else 64
        pstride = positions.stride(0) if positions.dim() == 2 and B > 1 else 0
    _fit(("q", q, tq), ("k", k, tk), ("cos", cos, (P, half)), ("sin", sin, (P, half)), ("q_out", q_out, tq),
         ("k_out", k_out, tk), ("positions", positions, (T,) if positions is not None and positions.dim() == 1 else (B, T)))
    kk, ko = (q, q_out) if k is None else (k, k_out)
    st = lib.sfda_rotary(_rows(q), _rows(k), _ptr(cos), _ptr(sin), _rows(positions), bits, pstride, offset, _rows(q_out),
                         _rows(k_out), B, Hq, Hk, T, D, 2 * half, P, interleaved, inverse,
                         _strides(3, q, kk, q_out, ko), code, _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_rotary")
    return q_out, k_out


def decay_attn_fwd(q, k, v, log_decay, S0=None, *, scale: float = 1.0, lengths=None, o=None, S_T=None,
                   want_state: bool = True, workspace=None, stream=None) -> Tuple:
    """Linear attention with one decay for each head (sfda_decay_attn_fwd): S_t = exp(log_decay) S_(t-1) + k_t v_t^T,
    o_t = scale S_t^T q_t.  q, k: [B,H,T,dk]; v: [B,H,T,dv] (float32 or bfloat16, any strides with a contiguous last
    axis: a [B,T,H,D] projection is passed as its transpose(1, 2)); log_decay: [H] float32; S0: [B,H,dk,dv] float32
    or None; lengths: [B] int32 or None (all T).  Returns (o [B,H,T,dv], S_T [B,H,dk,dv] float32 or None).  `workspace`: a
    uint8 device tensor (fastest with decay_attn_fwd_workspace_bytes(...) bytes, which are allocated here if it is None)."""
    import torch
    lib = load_library()
    if q.dim() != 4 or v.dim() != 4:
        raise ValueError("q and v must have 4 dimensions")
    B, H, T, dk = q.shape
    dv = v.shape[3]
    code = _same_dtype(q, k=k, v=v, o=o)
    tk, tv, ts = (B, H, T, dk), (B, H, T, dv), (B, H, dk, dv)
    if o is None:
        o = _empty_as(v, tv, stream)
    if S_T is None and want_state:
        S_T = _empty((B, H, dk, dv), torch.float32, q.device, stream)
    _need_f32(S0=S0, S_T=S_T, log_decay=log_decay)
    _int32("lengths", lengths)
    _fit(("q", q, tk), ("k", k, tk), ("v", v, tv), ("log_decay", log_decay, (H,)), ("lengths", lengths, (B,)), ("S0", S0, ts),
         ("o", o, tv), ("S_T", S_T, ts), ("workspace", workspace, workspace.shape if workspace is not None else ()))
    if workspace is None:
        nws = lib.sfda_decay_attn_fwd_workspace_bytes(B, H, T, dk, dv, code)
        workspace = _try_workspace(nws, q.device, stream) if nws else None
    st = lib.sfda_decay_attn_fwd(_rows(q), _rows(k), _rows(v), _ptr(log_decay), _ptr(lengths), _ptr(S0), _rows(o), _ptr(S_T),
                                 B, H, T, dk, dv, scale, _strides(3, q, k, v, o), code, _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(),
                                 _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_decay_attn_fwd")
    return o, S_T


def decay_attn_bwd(q, k, v, log_decay, S0, dO, dS_T=None, *, scale: float = 1.0, lengths=None, want_dS0: bool = True,
                   dq=None, dk=None, dv=None, workspace=None, stream=None) -> dict:
    """Gradients of a real loss through decay_attn_fwd (sfda_decay_attn_bwd), given dO = dL/do [B,H,T,dv] (the inputs'
    dtype, any strides) and dS_T = dL/dS_T [B,H,dk,dv] float32 or None.  Inputs as decay_attn_fwd; the decays are constants.
    Returns dq, dk, dv (new contiguous tensors if not given) and dS0 (float32, or None without want_dS0)."""
    import torch
    lib = load_library()
    if q.dim() != 4 or v.dim() != 4:
        raise ValueError("q and v must have 4 dimensions")
    B, H, T, nk = q.shape
    nv = v.shape[3]
    code = _same_dtype(q, k=k, v=v, dO=dO, dq=dq, dk=dk, dv=dv)
    tk, tv, ts = (B, H, T, nk), (B, H, T, nv), (B, H, nk, nv)
    dq = _empty_as(q, tk, stream) if dq is None else dq
    dk = _empty_as(k, tk, stream) if dk is None else dk
    dv = _empty_as(v, tv, stream) if dv is None else dv
    dS0 = _empty((B, H, nk, nv), torch.float32, q.device, stream) if want_dS0 else None
    _need_f32(S0=S0, dS_T=dS_T, log_decay=log_decay)
    _int32("lengths", lengths)
    _fit(("q", q, tk), ("k", k, tk), ("v", v, tv), ("log_decay", log_decay, (H,)), ("lengths", lengths, (B,)), ("S0", S0, ts),
         ("dO", dO, tv), ("dS_T", dS_T, ts), ("dq", dq, tk), ("dk", dk, tk), ("dv", dv, tv),
         ("workspace", workspace, workspace.shape if workspace is not None else ()))
    if workspace is None:
        nws = lib.sfda_decay_attn_bwd_workspace_bytes(B, H, T, nk, nv, code)
        workspace = _try_workspace(nws, q.device, stream) if nws else None
    strides = _strides(3, q, k, v, dO, dq, dk, dv)
    st = lib.sfda_decay_attn_bwd(_rows(q), _rows(k), _rows(v), _ptr(log_decay), _ptr(lengths), _ptr(S0), _rows(dO), _ptr(dS_T),
                                 _rows(dq), _rows(dk), _rows(dv), _ptr(dS0), B, H, T, nk, nv, scale, strides, code,
                                 _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(),
                                 _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_decay_attn_bwd")
    return dict(dq=dq, dk=dk, dv=dv, dS0=dS0)


def decay_attn_fwd_workspace_bytes(B: int, H: int, T: int, dk: int, dv: int, dtype: str = "f32") -> int:
    """The workspace at which decay_attn_fwd is fastest; dtype: the activations' ("f32" or "bf16")."""
    code = {"f32": SFDA_F32, "bf16": SFDA_BF16}[dtype]
    return int(load_library().sfda_decay_attn_fwd_workspace_bytes(B, H, T, dk, dv, code))


def decay_attn_bwd_workspace_bytes(B: int, H: int, T: int, dk: int, dv: int, dtype: str = "f32") -> int:
    """The workspace at which decay_attn_bwd is fastest; dtype: the activations' ("f32" or "bf16")."""
    code = {"f32": SFDA_F32, "bf16": SFDA_BF16}[dtype]
    return int(load_library().sfda_decay_attn_bwd_workspace_bytes(B, H, T, dk, dv, code))


def decay_attn_step(q, k, v, log_decay, S, *, scale: float = 1.0, o=None, stream=None):
    """One token of decay_attn_fwd (sfda_decay_attn_step).  q, k: [B,H,dk]; v: [B,H,dv] (any strides with a contiguous
    last axis); S: [B,H,dk,dv] float32, updated in place.  Returns o [B,H,dv]."""
    lib = load_library()
    if q.dim() != 3 or v.dim() != 3:
        raise ValueError("q and v must have 3 dimensions")
    B, H, dk = q.shape
    dv = v.shape[2]
    code = _same_dtype(q, k=k, v=v, o=o)
    tk, tv = (B, H, dk), (B, H, dv)
    if o is None:
        o = _empty_as(v, tv, stream)
    _need_f32(S=S, log_decay=log_decay)
    _fit(("q", q, tk), ("k", k, tk), ("v", v, tv), ("log_decay", log_decay, (H,)), ("S", S, (B, H, dk, dv)), ("o", o, tv))
    st = lib.sfda_decay_attn_step(_rows(q), _rows(k), _rows(v), _ptr(log_decay), _ptr(S), _rows(o), B, H, dk, dv, scale,
                                  _strides(2, q, k, v, o), code, _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_decay_attn_step")
    return o


def group_norm(x, weight=None, bias=None, gate=None, *, activation: str = "none", eps: float = 1e-5, y=None, stream=None):
    """Every token's heads normalised over their channels, scaled and activated (sfda_group_norm): n = x^ weight + bias,
    y = act(n), or n act(gate) with a gate; activation "none" or "silu".  x: [B,H,T,D] (any strides with a contiguous last
    axis; a channels-last [B,T,C] is passed as view(B,T,H,D).transpose(1, 2)); gate: [B,T,H*D]; weight, bias: [H*D]
    float32 or None.  Returns y [B,T,H*D]."""
    lib = load_library()
    if x.dim() != 4:
        raise ValueError("x must have 4 dimensions")
    B, H, T, D = x.shape
    code = _same_dtype(x, gate=gate, y=y)
    if activation not in _ACT:
        raise ValueError(f"activation must be 'none' or 'silu', not {activation!r}")
    if y is None:
        y = _empty((B, T, H * D), x.dtype, x.device, stream)
    _need_f32(weight=weight, bias=bias)
    tc, w = (B, T, H * D), (H * D,)
    _fit(("x", x, (B, H, T, D)), ("weight", weight, w), ("bias", bias, w), ("gate", gate, tc), ("y", y, tc))
    g = y if gate is None else gate
    st = lib.sfda_group_norm(_rows(x), _ptr(weight), _ptr(bias), _rows(gate), _rows(y), B, H, T, D, _ACT[activation], eps,
                             _STRIDES[7](*x.stride()[:3], *g.stride()[:2], *y.stride()[:2]), code, _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_group_norm")
    return y


def group_norm_bwd(dy, x, weight=None, bias=None, gate=None, *, activation: str = "none", eps: float = 1e-5, dx=None,
                   dgate=None, workspace=None, stream=None) -> dict:
    """Gradients of a real loss through group_norm (sfda_group_norm_bwd), given dy = dL/dy [B,T,H*D].  Returns dx (new and
    contiguous if not given), dgate, dweight, dbias (float32); None for what was not given.  `workspace`: a uint8 device
    tensor of at least sfda_group_norm_bwd_workspace_bytes, allocated here if None."""
    import torch
    lib = load_library()
    if x.dim() != 4:
        raise ValueError("x must have 4 dimensions")
    B, H, T, D = x.shape
    code = _same_dtype(x, dy=dy, gate=gate, dx=dx, dgate=dgate)
    if activation not in _ACT:
        raise ValueError(f"activation must be 'none' or 'silu', not {activation!r}")
    if dx is None:
        dx = _empty((B, H, T, D), x.dtype, x.device, stream)
    if gate is None:
        dgate = None
    elif dgate is None:
        dgate = _empty((B, T, H * D), x.dtype, x.device, stream)
    dweight = None if weight is None else _empty((H * D,), torch.float32, x.device, stream)
    dbias = None if bias is None else _empty((H * D,), torch.float32, x.device, stream)
    _need_f32(weight=weight, bias=bias)
    tc, w = (B, T, H * D), (H * D,)
    _fit(("x", x, (B, H, T, D)), ("dy", dy, tc), ("weight", weight, w), ("bias", bias, w), ("gate", gate, tc), ("dx", dx, (B, H, T, D)),
         ("dgate", dgate, tc), ("workspace", workspace, workspace.shape if workspace is not None else ()))
    if workspace is None and (dweight is not None or dbias is not None):
        workspace = _workspace(lib.sfda_group_norm_bwd_workspace_bytes(B, H, T, D, code), x.device, stream)
    g, dg = (dy, dy) if gate is None else (gate, dgate)
    st = lib.sfda_group_norm_bwd(_rows(dy), _rows(x), _ptr(weight), _ptr(bias), _rows(gate), _rows(dx), _rows(dgate),
                                 _ptr(dweight), _ptr(dbias), B, H, T, D, _ACT[activation], eps,
                                 _STRIDES[12](*x.stride()[:3], *g.stride()[:2], *dy.stride()[:2], *dx.stride()[:3],
                                                          *dg.stride()[:2]),
                                 code, _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(),
                                 _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_group_norm_bwd")
    return dict(dx=dx, dgate=dgate, dweight=dweight, dbias=dbias)


def rotary_axes(q, k, cos, sin, positions, sections, *, cyclic: bool = False, interleaved: bool = False, inverse: bool = False,
                q_out=None, k_out=None, stream=None) -> Tuple:
    """rotary for tokens with a position on each of several axes (sfda_rotary_axes): positions int32 or int64 [A,T] or [A,B,T];
    sections: how many pairs follow each of the A (1 to 4) axes, in runs, or with cyclic dealt to the axes in turn; their sum is
    rot / 2, the width of cos and sin.  A pair's angle is that of its own column of the tables: rotary_tables(P, rot) runs one set of
    frequencies through all axes; torch.cat of the axes' own tables along the columns gives each axis its own (with runs).
    Other arguments and the result as rotary's."""
    import torch
    lib = load_library()
    if q.dim() != 4 or cos.dim() != 2:
        raise ValueError("q must be [B,H,T,D] and cos [P, rot / 2]")
    B, Hq, T, D = q.shape
    Hk = 0 if k is None else k.shape[1]
    code = _same_dtype(q, k=k, q_out=q_out, k_out=k_out)
    _need_f32(cos=cos, sin=sin)
    A, (P, half) = len(sections), cos.shape
    if sum(sections) != half:
        raise ValueError(f"sections {tuple(sections)} must add up to the {half} pairs of the tables")
    if positions.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"positions must be int32 or int64 (got {positions.dtype})")
    tq, tk = (B, Hq, T, D), (B, Hk, T, D)
    if q_out is None:
        q_out = _empty_as(q, tq, stream)
    if k is None:
        k_out = None
    elif k_out is None:
        k_out = _empty_as(k, tk, stream)
    bits = 32 if positions.dtype == torch.int32 else 64
    astride = positions.stride(0) if A > 1 and positions.dim() > 1 else 0
    pstride = positions.stride(1) if positions.dim() == 3 and B > 1 else 0
    _fit(("q", q, tq), ("k", k, tk), ("cos", cos, (P, half)), ("sin", sin, (P, half)), ("q_out", q_out, tq),
         ("k_out", k_out, tk), ("positions", positions, (A, T) if positions.dim() == 2 else (A, B, T)))
    kk, ko = (q, q_out) if k is None else (k, k_out)
    st = lib.sfda_rotary_axes(_rows(q), _rows(k), _ptr(cos), _ptr(sin), _rows(positions), bits, astride, pstride,
                              (ctypes.c_int * A)(*sections), A, cyclic, _rows(q_out), _rows(k_out), B, Hq, Hk, T, D, P, interleaved,
                              inverse, _strides(3, q, kk, q_out, ko), code, _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_rotary_axes")
    return q_out, k_out


def _scalars(t) -> Optional[int]:
    """The pointer of a [B,H,T] tensor, of any strides."""
    return None if t is None else t.data_ptr()


def _heads_of(q, v) -> Tuple[int, int]:
    """Value heads and key heads, which have to divide them."""
    H, Hk = v.shape[1], q.shape[1]
    if Hk == 0 and H > 0 or Hk > 0 and H % Hk:
        raise ValueError(f"the heads of v ({H}) must be a multiple of those of q and k ({Hk})")
    return H, Hk


def delta_attn_fwd(q, k, v, log_decay, beta, S0=None, *, scale: float = 1.0, lengths=None, o=None, S_T=None,
                   want_state: bool = True, workspace=None, stream=None) -> Tuple:
    """Linear attention with the gated delta rule (sfda_delta_attn_fwd): with a_t = exp(log_decay_t),
    S_t = a_t S_(t-1) + k_t u_t^T, u_t = beta_t (v_t - a_t S_(t-1)^T k_t), o_t = scale S_t^T q_t.  q, k: [B,Hk,T,dk]; v: [B,H,T,dv]
    (float32 or bfloat16, any strides with a contiguous last axis: a [B,T,H,D] projection is passed as its transpose(1, 2));
    H a multiple of Hk; log_decay, beta: [B,H,T] float32 of any strides; S0: [B,H,dk,dv] float32 or None; lengths: [B] int32 or
    None (all T).  Returns (o [B,H,T,dv], S_T [B,H,dk,dv] float32 or None).  `workspace`: a uint8 device tensor; with
    delta_attn_fwd_workspace_bytes(...) bytes all heads run at once, with less (one head's at least, a B H-th) in passes over them, with
    the same results.  If it is None it is allocated here, as much as the device has room for."""
    import torch
    lib = load_library()
    if q.dim() != 4 or v.dim() != 4:
        raise ValueError("q and v must have 4 dimensions")
    H, Hk = _heads_of(q, v)
    B, _, T, dk = q.shape
    dv = v.shape[3]
    code = _same_dtype(q, k=k, v=v, o=o)
    tk, tv, tg, ts = (B, Hk, T, dk), (B, H, T, dv), (B, H, T), (B, H, dk, dv)
    if o is None:
        o = _empty_as(v, tv, stream)
    if S_T is None and want_state:
        S_T = _empty(ts, torch.float32, q.device, stream)
    _need_f32(S0=S0, S_T=S_T, log_decay=log_decay, beta=beta)
    _int32("lengths", lengths)
    _fit(("q", q, tk), ("k", k, tk), ("v", v, tv), ("log_decay", log_decay, tg), ("beta", beta, tg), ("lengths", lengths, (B,)),
         ("S0", S0, ts), ("o", o, tv), ("S_T", S_T, ts), ("workspace", workspace, workspace.shape if workspace is not None else ()))
    if workspace is None:
        nws = lib.sfda_delta_attn_fwd_workspace_bytes(B, H, T, dk, dv, code)
        n = B * H                       # heads of a pass
        while nws and workspace is None:
            part = nws // (B * H) * n
            workspace = _try_workspace(part, q.device, stream) if n > 1 else _workspace(part, q.device, stream)
            n = (n + 3) // 4
    st = lib.sfda_delta_attn_fwd(_rows(q), _rows(k), _rows(v), _scalars(log_decay), _scalars(beta), _ptr(lengths), _ptr(S0), _rows(o),
                                 _ptr(S_T), B, H, Hk, T, dk, dv, scale, _strides(3, q, k, v, log_decay, beta, o), code,
                                 _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(),
                                 _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_delta_attn_fwd")
    return o, S_T


def delta_attn_bwd(q, k, v, log_decay, beta, S0, dO, dS_T=None, *, scale: float = 1.0, lengths=None, want_dS0: bool = True,
                   dq=None, dk=None, dv=None, workspace=None, stream=None) -> dict:
    """Gradients of a real loss through delta_attn_fwd (sfda_delta_attn_bwd), given dO = dL/do [B,H,T,dv] (the inputs' dtype, any
    strides) and dS_T = dL/dS_T [B,H,dk,dv] float32 or None.  Inputs as delta_attn_fwd.  Returns dq, dk (summed over the value heads
    that share a key head), dv (new contiguous tensors if not given), dlog_decay, dbeta [B,H,T] float32 and dS0 (float32, or None
    without want_dS0).  `workspace`: a uint8 device tensor; with delta_attn_bwd_workspace_bytes(...) bytes all heads run at once,
    with less in passes over groups of heads, with the same results.  If it is None it is allocated here, at most 8 GiB
    where that holds the least that a call needs."""
    import torch
    lib = load_library()
    if q.dim() != 4 or v.dim() != 4:
        raise ValueError("q and v must have 4 dimensions")
    H, Hk = _heads_of(q, v)
    B, _, T, nk = q.shape
    nv = v.shape[3]
    code = _same_dtype(q, k=k, v=v, dO=dO, dq=dq, dk=dk, dv=dv)
    tk, tv, tg, ts = (B, Hk, T, nk), (B, H, T, nv), (B, H, T), (B, H, nk, nv)
    dq = _empty_as(q, tk, stream) if dq is None else dq
    dk = _empty_as(k, tk, stream) if dk is None else dk
    dv = _empty_as(v, tv, stream) if dv is None else dv
    dg, db = (_empty(tg, torch.float32, q.device, stream) for _ in range(2))
    dS0 = _empty(ts, torch.float32, q.device, stream) if want_dS0 else None
    _need_f32(S0=S0, dS_T=dS_T, log_decay=log_decay, beta=beta)
    _int32("lengths", lengths)
    _fit(("q", q, tk), ("k", k, tk), ("v", v, tv), ("log_decay", log_decay, tg), ("beta", beta, tg), ("lengths", lengths, (B,)),
         ("S0", S0, ts), ("dO", dO, tv), ("dS_T", dS_T, ts), ("dq", dq, tk), ("dk", dk, tk), ("dv", dv, tv),
         ("workspace", workspace, workspace.shape if workspace is not None else ()))
    if workspace is None and B * H > 0:
        nws = lib.sfda_delta_attn_bwd_workspace_bytes(B, H, Hk, T, nk, nv, code)
        least = lib.sfda_delta_attn_bwd_workspace_bytes(1, H // Hk, 1, T, nk, nv, code)
        nws = max(min(nws, 8 << 30), least)
        workspace = _try_workspace(nws, q.device, stream) if nws > least else None
        if workspace is None and least > 0:
            workspace = _workspace(least, q.device, stream)
    st = lib.sfda_delta_attn_bwd(_rows(q), _rows(k), _rows(v), _scalars(log_decay), _scalars(beta), _ptr(lengths), _ptr(S0), _rows(dO),
                                 _ptr(dS_T), _rows(dq), _rows(dk), _rows(dv), _scalars(dg), _scalars(db), _ptr(dS0), B, H, Hk, T, nk, nv,
                                 scale, _strides(3, q, k, v, log_decay, beta, dO, dq, dk, dv, dg, db), code, _ptr(workspace),
                                 0 if workspace is None else workspace.numel() * workspace.element_size(), _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_delta_attn_bwd")
    return dict(dq=dq, dk=dk, dv=dv, dlog_decay=dg, dbeta=db, dS0=dS0)


def delta_attn_fwd_workspace_bytes(B: int, H: int, T: int, dk: int, dv: int, dtype: str = "f32") -> int:
    """The workspace at which delta_attn_fwd runs all heads at once; the least is a B H-th of it.  dtype: the activations' ("f32" or
    "bf16")."""
    code = {"f32": SFDA_F32, "bf16": SFDA_BF16}[dtype]
    return int(load_library().sfda_delta_attn_fwd_workspace_bytes(B, H, T, dk, dv, code))


def delta_attn_bwd_workspace_bytes(B: int, H: int, Hk: int, T: int, dk: int, dv: int, dtype: str = "f32") -> int:
    """The workspace at which delta_attn_bwd runs all heads at once; the least is that of B = 1, H / Hk value heads and one key
    head.  dtype: the activations' ("f32" or "bf16")."""
    code = {"f32": SFDA_F32, "bf16": SFDA_BF16}[dtype]
    return int(load_library().sfda_delta_attn_bwd_workspace_bytes(B, H, Hk, T, dk, dv, code))


def delta_attn_step(q, k, v, log_decay, beta, S, *, scale: float = 1.0, o=None, stream=None):
    """One token of delta_attn_fwd (sfda_delta_attn_step).  q, k: [B,Hk,dk]; v: [B,H,dv] (any strides with a contiguous last axis);
    log_decay, beta: [B,H] float32 of any strides; S: [B,H,dk,dv] float32, updated in place.  Returns o [B,H,dv]."""
    lib = load_library()
    if q.dim() != 3 or v.dim() != 3:
        raise ValueError("q and v must have 3 dimensions")
    H, Hk = _heads_of(q, v)
    B, _, dk = q.shape
    dv = v.shape[2]
    code = _same_dtype(q, k=k, v=v, o=o)
    tk, tv, tg = (B, Hk, dk), (B, H, dv), (B, H)
    if o is None:
        o = _empty_as(v, tv, stream)
    _need_f32(S=S, log_decay=log_decay, beta=beta)
    _fit(("q", q, tk), ("k", k, tk), ("v", v, tv), ("log_decay", log_decay, tg), ("beta", beta, tg), ("S", S, (B, H, dk, dv)), ("o", o, tv))
    st = lib.sfda_delta_attn_step(_rows(q), _rows(k), _rows(v), _scalars(log_decay), _scalars(beta), _ptr(S), _rows(o), B, H, Hk, dk, dv,
                                  scale, _strides(2, q, k, v, log_decay, beta, o), code, _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_delta_attn_step")
    return o


def layer_norm(x, weight=None, bias=None, residual=None, *, eps: float = 1e-5, y=None, total=None, stream=None) -> Tuple:
    """Rows normalised over their channels, after the residual sum where there is one (sfda_layer_norm): total = x + residual, rounded
    to the type; y = (total - mean) / sqrt(var + eps) weight + bias.  x, residual: [B,T,D] (any strides with a contiguous last axis);
    weight, bias: [D] float32 or None.  Returns (y, total), total None without a residual; total=residual or total=x keeps the
    stream in place."""
    lib = load_library()
    if x.dim() != 3:
        raise ValueError("x must have 3 dimensions")
    B, T, D = x.shape
    code = _same_dtype(x, residual=residual, y=y, total=total)
    if y is None:
        y = _empty_as(x, x.shape, stream)
    if residual is None:
        total = None
    elif total is None:
        total = _empty_as(x, x.shape, stream)
    _need_f32(weight=weight, bias=bias)
    _fit(("x", x, (B, T, D)), ("weight", weight, (D,)), ("bias", bias, (D,)), ("residual", residual, (B, T, D)), ("y", y, (B, T, D)),
         ("total", total, (B, T, D)))
    r, t = (x, y) if residual is None else (residual, total)
    st = lib.sfda_layer_norm(_rows(x), _ptr(weight), _ptr(bias), _rows(residual), _rows(y), _rows(total), B, T, D, eps,
                             _strides(2, x, r, y, t), code, _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_layer_norm")
    return y, total


def layer_norm_bwd(dy, x, weight=None, bias=None, dtotal=None, *, eps: float = 1e-5, dx=None, workspace=None, stream=None) -> dict:
    """Gradients of a real loss through layer_norm (sfda_layer_norm_bwd), given dy = dL/dy [B,T,D], x (the total, where there was a
    residual) and, or None, dtotal: what reaches the total by other ways.  Returns dx, the gradient of x and of the residual alike (new
    if not given; dx=dy or dx=dtotal is allowed), dweight and dbias (float32; None for what was not given).  `workspace`: a
    uint8 device tensor of at least sfda_layer_norm_bwd_workspace_bytes, allocated here if None."""
    import torch
    lib = load_library()
    if x.dim() != 3:
        raise ValueError("x must have 3 dimensions")
    B, T, D = x.shape
    code = _same_dtype(x, dy=dy, dtotal=dtotal, dx=dx)
    if dx is None:
        dx = _empty_as(x, x.shape, stream)
    dweight = None if weight is None else _empty((D,), torch.float32, x.device, stream)
    dbias = None if bias is None else _empty((D,), torch.float32, x.device, stream)
    _need_f32(weight=weight, bias=bias)
    _fit(("x", x, (B, T, D)), ("dy", dy, (B, T, D)), ("weight", weight, (D,)), ("bias", bias, (D,)), ("dtotal", dtotal, (B, T, D)),
         ("dx", dx, (B, T, D)), ("workspace", workspace, workspace.shape if workspace is not None else ()))
    if workspace is None and (dweight is not None or dbias is not None):
        workspace = _workspace(lib.sfda_layer_norm_bwd_workspace_bytes(B, T, D, code), x.device, stream)
    st = lib.sfda_layer_norm_bwd(_rows(dy), _rows(x), _ptr(weight), _rows(dtotal), _rows(dx), _ptr(dweight), _ptr(dbias), B, T, D, eps,
                                 _strides(2, dy, x, dy if dtotal is None else dtotal, dx), code, _ptr(workspace),
                                 0 if workspace is None else workspace.numel() * workspace.element_size(), _stream(stream))
    if st != 0:
        raise SfdaError(st, "sfda_layer_norm_bwd")
    return dict(dx=dx, dweight=dweight, dbias=dbias)
