"""ctypes binding of the Fastmax C ABI (include/fastmax.h).

Argument marshalling only: every step of the computation runs in the HIP
library.  Tensors are PyTorch device tensors (they supply memory and the
stream); the library must be built (``python -m paper_2402_07901_amd.build``)
and fails loudly when it is missing.
"""
from __future__ import annotations

import contextlib
import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
# the sanitizer tier (tests/test_sanitize.py) points FASTMAX_LIB at the build
# whose host code carries AddressSanitizer/UBSan
LIB_PATH = os.environ.get("FASTMAX_LIB", os.path.join(_HERE, "libfastmax.so"))

F32 = 0
BF16 = 1

OK = 0
EINVAL = -1
EUNSUPPORTED = -2
ENULL = -3
EALIGN = -4
EWORKSPACE = -5
EHIP = -6

_lib = None


class Strides(ctypes.Structure):
    """fastmax_strides_t: strides in elements."""
    _fields_ = [("batch", ctypes.c_longlong), ("token", ctypes.c_longlong),
                ("head", ctypes.c_longlong)]


class Rope(ctypes.Structure):
    """fastmax_rope_t: norm and rotation of query and key rows."""
    _fields_ = [("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("pos", ctypes.c_void_p),
                ("table_rows", ctypes.c_int), ("rot", ctypes.c_int), ("axes", ctypes.c_int),
                ("sections", ctypes.c_int * 4), ("interleaved", ctypes.c_int),
                ("wq", ctypes.c_void_p), ("wk", ctypes.c_void_p), ("eps", ctypes.c_float)]


class FastmaxError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {strerror(code)} (code {code})")
        self.code = code


def lib():
    """The loaded libfastmax.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} not found: build it with `python -m paper_2402_07901_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        L.fastmax_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i]
        L.fastmax_workspace_bytes.restype = sz
        L.fastmax_fwd.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, i, i, vp, sz, vp]
        L.fastmax_fwd.restype = i
        L.fastmax_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, i, i,
                                  vp, sz, vp]
        L.fastmax_bwd.restype = i
        f = ctypes.c_float
        L.fastmax_fwd_scaled.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, i, f, i, vp, sz, vp]
        L.fastmax_fwd_scaled.restype = i
        L.fastmax_bwd_scaled.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, i, f,
                                         i, vp, sz, vp]
        L.fastmax_bwd_scaled.restype = i
        u64 = ctypes.c_uint64
        L.fastmax_dropout_mask_words.argtypes = [i]
        L.fastmax_dropout_mask_words.restype = sz
        L.fastmax_dropout_mask.argtypes = [vp, i, i, i, i, f, u64, vp]
        L.fastmax_dropout_mask.restype = i
        L.fastmax_dropout_workspace_bytes.argtypes = [i, i, i, i, i, i, i]
        L.fastmax_dropout_workspace_bytes.restype = sz
        L.fastmax_fwd_dropout.argtypes = [vp, vp, vp, vp, vp, vp, f, i, i, i, i, i, f, i, vp, sz,
                                          vp]
        L.fastmax_fwd_dropout.restype = i
        L.fastmax_bwd_dropout.argtypes = [vp, vp, vp, vp, vp, vp, vp, f, vp, vp, vp, i, i, i, i,
                                          i, f, i, vp, sz, vp]
        L.fastmax_bwd_dropout.restype = i
        L.fastmax_fwd_noalloc.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, i, f, i, vp]
        L.fastmax_fwd_noalloc.restype = i
        L.fastmax_set_scan_segments.argtypes = [i]
        L.fastmax_set_scan_segments.restype = i
        st, rope = vp, ctypes.POINTER(Rope)     # fastmax_strides_t arrays, NULL: contiguous
        L.fastmax_rope_fwd.argtypes = [vp, vp, vp, st, vp, vp, vp, i, i, i, i, i, rope, i, vp]
        L.fastmax_rope_fwd.restype = i
        L.fastmax_rope_workspace_bytes.argtypes = [i, i, i, i, i, i]
        L.fastmax_rope_workspace_bytes.restype = sz
        L.fastmax_rope_bwd.argtypes = [vp, vp, st, vp, vp, vp, vp, vp, vp, st, vp, vp, i, i, i, i,
                                       i, rope, i, vp, sz, vp]
        L.fastmax_rope_bwd.restype = i
        L.fastmax_cache_append.argtypes = [vp, vp, vp, st, vp, vp, vp, st, vp, i, i, i, i, i, i,
                                           rope, i, vp]
        L.fastmax_cache_append.restype = i
        L.fastmax_paged_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i, i, i]
        L.fastmax_paged_workspace_bytes.restype = sz
        L.fastmax_paged_fwd.argtypes = [vp, st, vp, vp, st, vp, vp, vp, vp, i, i, i, i, i, i, i, i,
                                        i, i, i, f, i, i, i, vp, sz, vp]
        L.fastmax_paged_fwd.restype = i
        L.fastmax_cache_append_q8.argtypes = [vp, vp, vp, st, vp, vp, vp, vp, vp, st, vp, i, i, i,
                                              i, i, i, rope, i, vp]
        L.fastmax_cache_append_q8.restype = i
        L.fastmax_cache_read_q8.argtypes = [vp, vp, vp, vp, st, vp, vp, vp, i, i, i, i, i, i, vp]
        L.fastmax_cache_read_q8.restype = i
        L.fastmax_paged_q8_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i, i, i]
        L.fastmax_paged_q8_workspace_bytes.restype = sz
        L.fastmax_paged_fwd_q8.argtypes = [vp, st, vp, vp, vp, vp, st, vp, vp, vp, vp, i, i, i, i, i,
                                           i, i, i, i, i, i, f, i, i, i, vp, sz, vp]
        L.fastmax_paged_fwd_q8.restype = i
        L.fastmax_packed_workspace_bytes.argtypes = [i, i, i, i, i, i, i]
        L.fastmax_packed_workspace_bytes.restype = sz
        L.fastmax_packed_fwd.argtypes = [vp, vp, vp, st, vp, vp, vp, i, i, i, i, i, i, i, f, i, vp,
                                         sz, vp]
        L.fastmax_packed_fwd.restype = i
        L.fastmax_packed_bwd.argtypes = [vp, vp, vp, st, vp, vp, vp, vp, vp, vp, vp, st, i, i, i, i,
                                         i, i, i, f, i, vp, sz, vp]
        L.fastmax_packed_bwd.restype = i
        L.fastmax_strerror.argtypes = [i]
        L.fastmax_strerror.restype = ctypes.c_char_p
        L.fastmax_version.restype = ctypes.c_char_p
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().fastmax_strerror(int(code)).decode()


def version() -> str:
    return lib().fastmax_version().decode()


# fastmax_set_scan_segments modes
SCAN_SEGMENTS_AUTO, SCAN_SEGMENTS_OFF, SCAN_SEGMENTS_ON, SCAN_SEGMENTS_REBUILD = 0, 1, 2, 3


def set_scan_segments(mode: int) -> int:
    """Process-wide segment mode of the causal MFMA scans; returns the previous one."""
    return lib().fastmax_set_scan_segments(int(mode))


def workspace_bytes(B, H, N, D, p, causal, dt, backward=False) -> int:
    return int(lib().fastmax_workspace_bytes(B, H, N, D, p, int(causal), dt, int(backward)))


# Calls of a few microseconds on the GPU wait for the host: pointers and
# streams go to ctypes as plain ints, the device is switched only when another
# one is current, and the usual arguments pass one comparison each (small
# float32 forward, host time per call 17.3 -> 12.8 us).
def _ptr(t):
    if t is None:
        return None
    return t.data_ptr() if hasattr(t, "data_ptr") else t


def _stream(stream):
    """The stream argument as a handle: ``stream`` as given (a torch stream or
    a raw handle), else the current device's current stream."""
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def _stream_of(stream, device):
    """``stream``, or the handle of ``device``'s current stream when None."""
    if stream is None:
        import torch
        return torch._C._cuda_getCurrentRawStream(device.index)
    return stream


_HERE_ALREADY = contextlib.nullcontext()


def _on(device):
    """Context that makes ``device`` current for a library call (the library
    runs its kernels, and requires its stream to be, on the current device)."""
    import torch
    if device.index == torch.cuda.current_device():
        return _HERE_ALREADY
    return torch.cuda.device(device)


def _dtype_code(t):
    import torch
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def fastmax_fwd_raw(q, k, v, out, g, B, H, N, D, p, causal, dt, workspace, ws_bytes, stream,
                    scale=None):
    """Direct call of fastmax_fwd (fastmax_fwd_scaled when ``scale`` is given)
    with raw pointers/ints; returns the code."""
    if scale is None:
        return lib().fastmax_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(g), B, H, N, D, p,
                                 int(causal), dt, _ptr(workspace), ws_bytes, _stream(stream))
    return lib().fastmax_fwd_scaled(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(g), B, H, N, D,
                                    p, int(causal), float(scale), dt, _ptr(workspace), ws_bytes,
                                    _stream(stream))


def fastmax_bwd_raw(q, k, v, out, dout, g, dq, dk, dv, B, H, N, D, p, causal, dt, workspace,
                    ws_bytes, stream, scale=None):
    if scale is None:
        return lib().fastmax_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(dout), _ptr(g),
                                 _ptr(dq), _ptr(dk), _ptr(dv), B, H, N, D, p, int(causal), dt,
                                 _ptr(workspace), ws_bytes, _stream(stream))
    return lib().fastmax_bwd_scaled(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(dout), _ptr(g),
                                    _ptr(dq), _ptr(dk), _ptr(dv), B, H, N, D, p, int(causal),
                                    float(scale), dt, _ptr(workspace), ws_bytes,
                                    _stream(stream))


# the library's per-GPU scratch size for fastmax_fwd_noalloc (include/fastmax.h)
NOALLOC_MAX_WORKSPACE_BYTES = 64 << 20


def fastmax_fwd_noalloc_raw(q, k, v, out, g, B, H, N, D, p, causal, dt, stream, scale=1.0):
    """Direct call of fastmax_fwd_noalloc with raw pointers/ints; returns the code."""
    return lib().fastmax_fwd_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(g), B, H, N, D,
                                     p, int(causal), float(scale), dt, _stream(stream))


def fastmax_fwd_noalloc(q, k, v, out, g=None, p=2, causal=False, stream=None, scale=None):
    """fastmax_fwd into caller-provided ``out`` (and ``g``) with the library's
    per-GPU scratch as workspace: nothing is allocated."""
    B, H, N, D = _check_args(q, k=(k, "like_q"), v=(v, "like_q"), out=(out, "like_q"),
                             g=(g, "g"))
    with _on(q.device):
        rc = fastmax_fwd_noalloc_raw(q, k, v, out, g, B, H, N, D, p, causal, _dtype_code(q),
                                     _stream_of(stream, q.device), 1.0 if scale is None else scale)
    if rc != OK:
        raise FastmaxError(rc, "fastmax_fwd_noalloc")
    return out, g


def _check_args(q, **tensors):
    """Shape, dtype, layout and device checks the C ABI cannot make (it sees
    pointers only): q is a contiguous [B, H, N, D] tensor on a GPU; every
    other tensor is contiguous, on q's device, with the shape and dtype
    its entry names ("like_q": q's; "g": float32 [B, H, N]; "bits": int32
    [B, H, N, words]; "workspace": any dtype).  Returns (B, H, N, D)."""
    import torch
    if q.dim() != 4:
        raise ValueError(f"q must be [B, H, N, D], got shape {tuple(q.shape)}")
    shape, dtype, device = q.shape, q.dtype, q.device
    B, H, N, D = shape
    if not q.is_contiguous():
        raise ValueError("q must be contiguous")
    for name, (t, kind) in tensors.items():
        if t is None:
            continue
        if kind == "like_q":
            want, wdtype = shape, dtype
        elif kind == "g":
            want, wdtype = (B, H, N), torch.float32
        elif kind == "bits":
            want, wdtype = (B, H, N, mask_words(D)), torch.int32
        else:                                   # "workspace"
            want, wdtype = t.shape, t.dtype
        if t.shape != want:
            raise ValueError(f"{name} must have shape {tuple(want)}, got {tuple(t.shape)}")
        if t.dtype != wdtype:
            raise ValueError(f"{name} must be {wdtype}, got {t.dtype}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        if t.device != device:
            raise ValueError(f"{name} is on {t.device}, q on {device}")
    if device.type != "cuda":
        raise ValueError(f"the tensors must be on a GPU, q is on {device}")
    return B, H, N, D


def _alloc_ws(nbytes, device):
    import torch
    if nbytes == 0:
        return None
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def fastmax_fwd(q, k, v, p=2, causal=False, out=None, g=None, want_g=True, workspace=None,
                stream=None, scale=None):
    """O = Fastmax(q, k, v) for [B, H, N, D] device tensors; returns (O, G).
    ``scale``: score scale (weights f_p(scale * q^.k^)); None = the definition."""
    import torch
    B, H, N, D = _check_args(q, k=(k, "like_q"), v=(v, "like_q"), out=(out, "like_q"),
                             g=(g, "g"), workspace=(workspace, "workspace"))
    dt = _dtype_code(q)
    if out is None:
        out = torch.empty_like(q)
    if g is None and want_g:
        g = torch.empty((B, H, N), dtype=torch.float32, device=q.device)
    need = workspace_bytes(B, H, N, D, p, causal, dt, False)
    if workspace is None:
        workspace = _alloc_ws(need, q.device)
    ws_n = 0 if workspace is None else workspace.numel() * workspace.element_size()
    with _on(q.device):
        rc = fastmax_fwd_raw(q, k, v, out, g, B, H, N, D, p, causal, dt, workspace, ws_n,
                             _stream_of(stream, q.device), scale)
    if rc != OK:
        raise FastmaxError(rc, "fastmax_fwd")
    return out, g


def fastmax_bwd(q, k, v, out, dout, g, p=2, causal=False, dq=None, dk=None, dv=None,
                workspace=None, stream=None, scale=None):
    """Gradients (dq, dk, dv) of sum(dout * O); ``scale`` as in the forward."""
    import torch
    B, H, N, D = _check_args(q, k=(k, "like_q"), v=(v, "like_q"), out=(out, "like_q"),
                             dout=(dout, "like_q"), g=(g, "g"), dq=(dq, "like_q"),
                             dk=(dk, "like_q"), dv=(dv, "like_q"),
                             workspace=(workspace, "workspace"))
    dt = _dtype_code(q)
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(q) if dk is None else dk
    dv = torch.empty_like(q) if dv is None else dv
    need = workspace_bytes(B, H, N, D, p, causal, dt, True)
    if workspace is None:
        workspace = _alloc_ws(need, q.device)
    ws_n = 0 if workspace is None else workspace.numel() * workspace.element_size()
    with _on(q.device):
        rc = fastmax_bwd_raw(q, k, v, out, dout, g, dq, dk, dv, B, H, N, D, p, causal, dt,
                             workspace, ws_n, _stream_of(stream, q.device), scale)
    if rc != OK:
        raise FastmaxError(rc, "fastmax_bwd")
    return dq, dk, dv


# ---------------------------------------------------------------------------
# Quadratic-term dropout (Sec. 2.4, dropout paragraph; Fig. 2), p = 2.  Keep
# bits are an int32 tensor [B, H, N, mask_words(D)] holding the uint32 words.
# ---------------------------------------------------------------------------
def mask_words(D) -> int:
    """uint32 words per token of a keep-bit row (0 for an unsupported D)."""
    return int(lib().fastmax_dropout_mask_words(int(D)))


def fastmax_dropout_mask_raw(bits, B, H, N, D, rate, seed, stream):
    return lib().fastmax_dropout_mask(_ptr(bits), B, H, N, D, float(rate),
                                      ctypes.c_uint64(int(seed)), _stream(stream))


def dropout_mask(B, H, N, D, rate, seed, device="cuda", stream=None):
    """Philox4x32-10 keep bits for the quadratic features of every key token."""
    import torch
    bits = torch.empty((B, H, N, mask_words(D)), dtype=torch.int32, device=device)
    with _on(bits.device):
        rc = fastmax_dropout_mask_raw(bits, B, H, N, D, rate, seed,
                                      _stream_of(stream, bits.device))
    if rc != OK:
        raise FastmaxError(rc, "fastmax_dropout_mask")
    return bits


def dropout_workspace_bytes(B, H, N, D, causal, dt, backward=False) -> int:
    return int(lib().fastmax_dropout_workspace_bytes(B, H, N, D, int(causal), dt,
                                                     int(bool(backward))))


def fastmax_fwd_dropout_raw(q, k, v, out, g, bits, rate, B, H, N, D, causal, scale, dt,
                            workspace, ws_bytes, stream):
    return lib().fastmax_fwd_dropout(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(g), _ptr(bits),
                                     float(rate), B, H, N, D, int(causal), float(scale), dt,
                                     _ptr(workspace), ws_bytes, _stream(stream))


def fastmax_bwd_dropout_raw(q, k, v, out, dout, g, bits, rate, dq, dk, dv, B, H, N, D, causal,
                            scale, dt, workspace, ws_bytes, stream):
    return lib().fastmax_bwd_dropout(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(dout), _ptr(g),
                                     _ptr(bits), float(rate), _ptr(dq), _ptr(dk), _ptr(dv), B, H,
                                     N, D, int(causal), float(scale), dt, _ptr(workspace),
                                     ws_bytes, _stream(stream))


def fastmax_fwd_dropout(q, k, v, bits, rate, causal=False, scale=None, out=None, g=None,
                        workspace=None, stream=None):
    """Forward with the quadratic features of the keys masked by ``bits``
    (kept ones scaled by 1/(1 - rate)); returns (O, G)."""
    import torch
    B, H, N, D = _check_args(q, k=(k, "like_q"), v=(v, "like_q"), bits=(bits, "bits"),
                             out=(out, "like_q"), g=(g, "g"),
                             workspace=(workspace, "workspace"))
    dt = _dtype_code(q)
    out = torch.empty_like(q) if out is None else out
    if g is None:
        g = torch.empty((B, H, N), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = _alloc_ws(dropout_workspace_bytes(B, H, N, D, causal, dt, False), q.device)
    ws_n = 0 if workspace is None else workspace.numel() * workspace.element_size()
    with _on(q.device):
        rc = fastmax_fwd_dropout_raw(q, k, v, out, g, bits, rate, B, H, N, D, causal,
                                     1.0 if scale is None else scale, dt, workspace, ws_n,
                                     _stream_of(stream, q.device))
    if rc != OK:
        raise FastmaxError(rc, "fastmax_fwd_dropout")
    return out, g


def fastmax_bwd_dropout(q, k, v, out, dout, g, bits, rate, causal=False, scale=None, dq=None,
                        dk=None, dv=None, workspace=None, stream=None):
    """Gradients (dq, dk, dv) of sum(dout * O) for the forward with the same bits."""
    import torch
    B, H, N, D = _check_args(q, k=(k, "like_q"), v=(v, "like_q"), out=(out, "like_q"),
                             dout=(dout, "like_q"), g=(g, "g"), bits=(bits, "bits"),
                             dq=(dq, "like_q"), dk=(dk, "like_q"), dv=(dv, "like_q"),
                             workspace=(workspace, "workspace"))
    dt = _dtype_code(q)
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(q) if dk is None else dk
    dv = torch.empty_like(q) if dv is None else dv
    if workspace is None:
        workspace = _alloc_ws(dropout_workspace_bytes(B, H, N, D, causal, dt, True), q.device)
    ws_n = 0 if workspace is None else workspace.numel() * workspace.element_size()
    with _on(q.device):
        rc = fastmax_bwd_dropout_raw(q, k, v, out, dout, g, bits, rate, dq, dk, dv, B, H, N, D,
                                     causal, 1.0 if scale is None else scale, dt, workspace,
                                     ws_n, _stream_of(stream, q.device))
    if rc != OK:
        raise FastmaxError(rc, "fastmax_bwd_dropout")
    return dq, dk, dv


# ---------------------------------------------------------------------------
# Around the attention: norm and rotation of a projection's rows, shared heads,
# a paged cache and the attention of new tokens over it.
# ---------------------------------------------------------------------------
# These calls may take less time on the GPU than on the host, so the usual
# arguments pass one comparison each and what is wrong is found out after; a
# tensor's dtype and device index (``dev``) are asked for once.
_t = None   # torch, once a call has brought tensors


def _torch():
    global _t
    if _t is None:
        import torch
        _t = torch
    return _t


def _wrong(name, t, shape, dtype, q):
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.device != q.device:
        raise ValueError(f"{name} is on {t.device}, not on {q.device}")


def _rows_of(name, t, shape, dtype, dev, q):
    """Checks token rows: dtype, q's device, the given shape, D contiguous (the
    library checks the other strides)."""
    if t.shape != shape or t.dtype != dtype or t.get_device() != dev or t.stride(-1) != 1:
        _wrong(name, t, shape, dtype, q)
        raise ValueError(f"{name}'s channels must be contiguous")


def _whole(name, t, shape, dtype, dev, q):
    """Checks a contiguous tensor of a given dtype and shape on q's device."""
    if t.shape != shape or t.dtype != dtype or t.get_device() != dev or not t.is_contiguous():
        _wrong(name, t, shape, dtype, q)
        raise ValueError(f"{name} must be contiguous")


_LL3, _LL6, _LL9 = (ctypes.c_longlong * n for n in (3, 6, 9))   # one, two, three strides


def _rope_of(q, tokens, pos, cos, sin, wq, wk, eps, sections, interleaved):
    """The fastmax_rope_t of a call whose rows are q's; ``tokens``: q's
    leading sizes."""
    torch, dev = _torch(), q.get_device()
    p = c = s = gq = gk = None
    rows = rot = 0
    axes, parts = 1, ()
    if (cos is None) != (sin is None) or (cos is None) != (pos is None):
        raise ValueError("pos, cos and sin go together")
    if cos is not None:
        shape = cos.shape
        if len(shape) != 2:
            raise ValueError(f"cos must be [rows, rot / 2], got shape {tuple(shape)}")
        _whole("cos", cos, shape, torch.float32, dev, q)
        _whole("sin", sin, shape, torch.float32, dev, q)
        if pos.dim() > len(tokens):
            axes = pos.shape[-1]
            tokens = (*tokens, axes)
        _whole("pos", pos, tokens, torch.int32, dev, q)
        if axes != 1:
            if not 1 <= axes <= 4:
                raise ValueError(f"1 to 4 axes of positions, got {axes}")
            if sections is None or len(sections) != axes:
                raise ValueError(f"{axes} axes of positions need as many sections")
            parts = tuple(sections)
        p, c, s = pos.data_ptr(), cos.data_ptr(), sin.data_ptr()
        rows, rot = shape[0], 2 * shape[1]
    if wq is not None and wk is not None:
        D = q.shape[-1:]
        _whole("wq", wq, D, torch.float32, dev, q)
        _whole("wk", wk, D, torch.float32, dev, q)
        gq, gk = wq.data_ptr(), wk.data_ptr()
    elif wq is not wk:
        raise ValueError("wq and wk go together")
    return Rope(c, s, p, rows, rot, axes, parts, 1 if interleaved else 0, gq, gk, eps)


def _of(name, given, n):
    """Checks that the caller's outputs, if there are any, are n tensors."""
    if given is not None and len(given) != n:
        raise ValueError(f"{name} must be {n} tensors, got {len(given)}")


def _on_gpu(q, dims, what):
    if q.dim() != dims:
        raise ValueError(f"q must be {what}, got shape {tuple(q.shape)}")
    if not q.is_cuda:
        raise ValueError(f"the tensors must be on a GPU, q is on {q.device}")
    if q.stride(-1) != 1:
        raise ValueError("q's channels must be contiguous")


@contextlib.contextmanager
def _owner(stream, device):
    """Context in which what a call allocates belongs to the stream it runs on:
    memory that another stream still uses is not handed to it, nor its own to
    others while it runs."""
    torch = _torch()
    if not hasattr(stream, "cuda_stream"):
        # handle 0 is the null stream; torch would make a stream of its own of it
        stream = (torch.cuda.ExternalStream(stream, device=device) if stream
                  else torch.cuda.default_stream(device))
    with torch.cuda.stream(stream):
        yield


def _new(q, shapes, stream, dtype=None):
    """Uninitialised tensors like q (of ``dtype``) for a call on ``stream``; a
    shape None gives None."""
    if stream is None:
        return [x if x is None else q.new_empty(x, dtype=dtype) for x in shapes]
    with _owner(stream, q.device):
        return [x if x is None else q.new_empty(x, dtype=dtype) for x in shapes]


def _workspace(q, given, nbytes, stream):
    """(tensor, bytes) of a call's workspace: the caller's, checked, or
    ``nbytes()`` of its own."""
    if given is not None:
        _whole("workspace", given, given.shape, given.dtype, q.get_device(), q)
        return given, given.numel() * given.element_size()
    n = nbytes()
    return (_new(q, [(n,)], stream, _torch().uint8)[0], n) if n else (None, 0)


def _run(what, fn, dev, stream, *args):
    """fn(*args, stream) on device ``dev``, the stream None meaning its current one."""
    torch = _torch()
    handle = torch._C._cuda_getCurrentRawStream(dev) if stream is None else _stream(stream)
    if dev == torch.cuda.current_device():
        rc = fn(*args, handle)
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, handle)
    if rc != OK:
        raise FastmaxError(rc, what)


def fastmax_rope_fwd(q, k, v, pos, cos, sin, wq=None, wk=None, eps=1e-6, sections=None,
                     interleaved=False, out=None, stream=None):
    """A projection's rows q [B, N, Hq, D], k and v [B, N, Hkv, D] (strided
    views; D contiguous) as the attention takes them: RMS norm with weights wq
    and wk (None: no norm), rotation by position (cos, sin [rows, rot / 2]; pos
    int32 [B, N] or [B, N, axes] with ``sections`` pairs per axis; all None: no
    rotation), key and value heads repeated.  Returns three contiguous
    [B, Hq, N, D] tensors (``out``: the same, the caller's)."""
    _of("out", out, 3)
    _on_gpu(q, 4, "[B, N, Hq, D]")
    B, N, Hq, D = q.shape
    dtype, dev, dt = q.dtype, q.get_device(), _dtype_code(q)
    Hkv = k.shape[2] if k.dim() == 4 else 0
    rows, heads = (B, N, Hkv, D), (B, Hq, N, D)
    _rows_of("k", k, rows, dtype, dev, q)
    _rows_of("v", v, rows, dtype, dev, q)
    rope = _rope_of(q, (B, N), pos, cos, sin, wq, wk, eps, sections, interleaved)
    if out is None:
        out = _new(q, (heads,) * 3, stream)
    else:
        for name, t in zip(("out[0]", "out[1]", "out[2]"), out):
            _whole(name, t, heads, dtype, dev, q)
    _run("fastmax_rope_fwd", lib().fastmax_rope_fwd, dev, stream,
         q.data_ptr(), k.data_ptr(), v.data_ptr(),
         _LL9(*q.stride()[:3], *k.stride()[:3], *v.stride()[:3]),
         out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(), B, N, Hq, Hkv, D, rope, dt)
    return tuple(out)


def rope_workspace_bytes(B, N, Hq, Hkv, D, norm) -> int:
    return int(lib().fastmax_rope_workspace_bytes(B, N, Hq, Hkv, D, int(bool(norm))))


def fastmax_rope_bwd(q, k, gq, gk, gv, pos, cos, sin, wq=None, wk=None, eps=1e-6, sections=None,
                     interleaved=False, out=None, workspace=None, stream=None):
    """Backward of fastmax_rope_fwd: gq, gk, gv [B, Hq, N, D] are the gradients
    of its outputs; q and k its inputs (their shapes count; they are read with a
    norm only).  Returns (dq, dk, dv, dwq, dwk), dq [B, N, Hq, D], dk and dv
    [B, N, Hkv, D] (``out``: these three, the caller's, strided as they like),
    dwq and dwk float32 [D] (None without a norm)."""
    _of("out", out, 3)
    _on_gpu(q, 4, "[B, N, Hq, D]")
    B, N, Hq, D = q.shape
    dtype, dev, dt = q.dtype, q.get_device(), _dtype_code(q)
    Hkv = k.shape[2] if k.dim() == 4 else 0
    rows, heads = (B, N, Hkv, D), (B, Hq, N, D)
    _rows_of("k", k, rows, dtype, dev, q)
    _whole("gq", gq, heads, dtype, dev, q)
    _whole("gk", gk, heads, dtype, dev, q)
    _whole("gv", gv, heads, dtype, dev, q)
    rope = _rope_of(q, (B, N), pos, cos, sin, wq, wk, eps, sections, interleaved)
    if out is None:
        out = _new(q, ((B, N, Hq, D), rows, rows), stream)
    else:
        for name, t, shape in zip(("out[0]", "out[1]", "out[2]"), out, (q.shape, rows, rows)):
            _rows_of(name, t, shape, dtype, dev, q)
    dwq = dwk = None
    if wq is not None:
        dwq, dwk = _new(q, ((D,), (D,)), stream, wq.dtype)
    workspace, ws_n = _workspace(
        q, workspace, lambda: rope_workspace_bytes(B, N, Hq, Hkv, D, wq is not None), stream)
    _run("fastmax_rope_bwd", lib().fastmax_rope_bwd, dev, stream,
         q.data_ptr(), k.data_ptr(), _LL6(*q.stride()[:3], *k.stride()[:3]),
         gq.data_ptr(), gk.data_ptr(), gv.data_ptr(),
         out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(),
         _LL9(*(n for t in out for n in t.stride()[:3])),
         _ptr(dwq), _ptr(dwk), B, N, Hq, Hkv, D, rope, dt, _ptr(workspace), ws_n)
    return (*out, dwq, dwk)


def _cache_of(q, k_cache, v_cache, Hkv, dtype=None):
    """(pages, page size, strides) of the caches [pages, Hkv, page, D]; their
    type is q's unless given."""
    shape = k_cache.shape
    if len(shape) != 4:
        raise ValueError(f"k_cache must be [pages, Hkv, page, D], got shape {tuple(shape)}")
    pages, _, page, _ = shape
    dtype, dev = dtype or q.dtype, q.get_device()
    _rows_of("k_cache", k_cache, (pages, Hkv, page, q.shape[-1]), dtype, dev, q)
    _rows_of("v_cache", v_cache, shape, dtype, dev, q)
    st = k_cache.stride()
    if v_cache.stride() != st and any(n > 1 and x != y
                                      for n, x, y in zip(shape, st, v_cache.stride())):
        raise ValueError(f"k_cache and v_cache must have the same strides, got {st} and "
                         f"{v_cache.stride()}")
    return pages, page, _LL3(st[0], st[2], st[1])


def fastmax_cache_append(q, k, v, k_cache, v_cache, slots, pos, cos, sin, wq=None, wk=None,
                         eps=1e-6, sections=None, interleaved=False, q_out=None, stream=None):
    """New tokens q [T, Hq, D], k and v [T, Hkv, D] (strided views; D
    contiguous): norm and rotation as in fastmax_rope_fwd, then the attention's
    standardisation.  k^ and v go to the slots (int64 [T], page * page size +
    place; -1: none) of the caches [pages, Hkv, page, D]; returns q^ [T, Hq, D]."""
    _on_gpu(q, 3, "[T, Hq, D]")
    T, Hq, D = q.shape
    dtype, dev, dt = q.dtype, q.get_device(), _dtype_code(q)
    Hkv = k.shape[1] if k.dim() == 3 else 0
    _rows_of("k", k, (T, Hkv, D), dtype, dev, q)
    _rows_of("v", v, (T, Hkv, D), dtype, dev, q)
    pages, page, cache = _cache_of(q, k_cache, v_cache, Hkv)
    _whole("slots", slots, (T,), _torch().int64, dev, q)
    rope = _rope_of(q, (T,), pos, cos, sin, wq, wk, eps, sections, interleaved)
    if q_out is None:
        q_out, = _new(q, ((T, Hq, D),), stream)
    else:
        _whole("q_out", q_out, (T, Hq, D), dtype, dev, q)
    _run("fastmax_cache_append", lib().fastmax_cache_append, dev, stream,
         q.data_ptr(), k.data_ptr(), v.data_ptr(),
         _LL9(0, *q.stride()[:2], 0, *k.stride()[:2], 0, *v.stride()[:2]),
         q_out.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), cache, slots.data_ptr(),
         T, Hq, Hkv, D, pages, page, rope, dt)
    return q_out


def paged_workspace_bytes(S, T, Hq, Hkv, D, max_q, max_len, window, sinks, dt) -> int:
    return int(lib().fastmax_paged_workspace_bytes(S, T, Hq, Hkv, D, max_q, max_len, window,
                                                   sinks, dt))


def fastmax_paged_fwd(q, k_cache, v_cache, table, lens, q_start=None, max_q=None, max_len=None,
                      p=2, scale=None, window=0, sinks=0, out=None, workspace=None, stream=None):
    """Fastmax attention of new tokens over a paged cache.  q: q^ [T, Hq, D];
    caches [pages, Hkv, page, D]; table int32 [S, cols] of pages; lens int32 [S]
    tokens per sequence, its new ones last; q_start int32 [S + 1] where each
    sequence's rows of q begin (None: one row each).  max_q and max_len: the most
    rows and the most tokens of a sequence (None: T, or what the table holds,
    which costs time where sequences have less).
    window > 0: the last ``window`` keys and the first ``sinks`` only.  Returns
    O [T, Hq, D]."""
    _on_gpu(q, 3, "[T, Hq, D]")
    T, Hq, D = q.shape
    dtype, dev, dt = q.dtype, q.get_device(), _dtype_code(q)
    Hkv = k_cache.shape[1] if k_cache.dim() == 4 else 0
    pages, page, cache = _cache_of(q, k_cache, v_cache, Hkv)
    if table.dim() != 2:
        raise ValueError(f"table must be [S, cols], got shape {tuple(table.shape)}")
    S, cols = table.shape
    int32 = _torch().int32
    _whole("table", table, (S, cols), int32, dev, q)
    _whole("lens", lens, (S,), int32, dev, q)
    if q_start is not None:
        _whole("q_start", q_start, (S + 1,), int32, dev, q)
    if max_q is None:
        max_q = 1 if q_start is None else T
    if max_len is None:
        max_len = cols * page
    if out is None:
        out, = _new(q, ((T, Hq, D),), stream)
    else:
        _whole("out", out, (T, Hq, D), dtype, dev, q)
    workspace, ws_n = _workspace(
        q, workspace,
        lambda: paged_workspace_bytes(S, T, Hq, Hkv, D, max_q, max_len, window, sinks, dt), stream)
    _run("fastmax_paged_fwd", lib().fastmax_paged_fwd, dev, stream,
         q.data_ptr(), _LL3(0, *q.stride()[:2]), k_cache.data_ptr(), v_cache.data_ptr(), cache,
         table.data_ptr(), lens.data_ptr(), _ptr(q_start), out.data_ptr(), S, T, Hq, Hkv, D, pages,
         page, cols, max_q, max_len, p, 1.0 if scale is None else scale, window, sinks, dt,
         _ptr(workspace), ws_n)
    return out


# --- the cache in 8 bits ------------------------------------------------------
def _cache_q8_of(q, k_cache, v_cache, k_scale, v_scale, Hkv):
    """_cache_of 8-bit caches, with their scales float32 [pages, Hkv, page]."""
    torch = _torch()
    pages, page, cache = _cache_of(q, k_cache, v_cache, Hkv, torch.int8)
    _whole("k_scale", k_scale, (pages, Hkv, page), torch.float32, q.get_device(), q)
    _whole("v_scale", v_scale, (pages, Hkv, page), torch.float32, q.get_device(), q)
    return pages, page, cache


def fastmax_cache_append_q8(q, k, v, k_cache, v_cache, k_scale, v_scale, slots, pos, cos, sin,
                            wq=None, wk=None, eps=1e-6, sections=None, interleaved=False,
                            q_out=None, stream=None):
    """fastmax_cache_append into a cache of 8-bit rows: k_cache and v_cache int8
    [pages, Hkv, page, D], k_scale and v_scale float32 [pages, Hkv, page]; a row
    stands for code * scale.  Returns q^ [T, Hq, D]."""
    _on_gpu(q, 3, "[T, Hq, D]")
    T, Hq, D = q.shape
    dtype, dev, dt = q.dtype, q.get_device(), _dtype_code(q)
    Hkv = k.shape[1] if k.dim() == 3 else 0
    _rows_of("k", k, (T, Hkv, D), dtype, dev, q)
    _rows_of("v", v, (T, Hkv, D), dtype, dev, q)
    pages, page, cache = _cache_q8_of(q, k_cache, v_cache, k_scale, v_scale, Hkv)
    _whole("slots", slots, (T,), _torch().int64, dev, q)
    rope = _rope_of(q, (T,), pos, cos, sin, wq, wk, eps, sections, interleaved)
    if q_out is None:
        q_out, = _new(q, ((T, Hq, D),), stream)
    else:
        _whole("q_out", q_out, (T, Hq, D), dtype, dev, q)
    _run("fastmax_cache_append_q8", lib().fastmax_cache_append_q8, dev, stream,
         q.data_ptr(), k.data_ptr(), v.data_ptr(),
         _LL9(0, *q.stride()[:2], 0, *k.stride()[:2], 0, *v.stride()[:2]),
         q_out.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), k_scale.data_ptr(),
         v_scale.data_ptr(), cache, slots.data_ptr(), T, Hq, Hkv, D, pages, page, rope, dt)
    return q_out


def fastmax_cache_read_q8(k_cache, v_cache, k_scale, v_scale, slots, dtype=None, out=None,
                          stream=None):
    """Rows of an 8-bit cache by their slots (int64 [T], page * page size +
    place; one outside the cache: zeros).  Returns k^ and v [T, Hkv, D] of
    ``dtype`` (float32 or bfloat16, the default; ``out``: the same two, the
    caller's)."""
    torch = _torch()
    _of("out", out, 2)
    _on_gpu(k_cache, 4, "[pages, Hkv, page, D]")
    _, Hkv, _, D = k_cache.shape
    dev = k_cache.get_device()
    pages, page, cache = _cache_q8_of(k_cache, k_cache, v_cache, k_scale, v_scale, Hkv)
    if slots.dim() != 1:
        raise ValueError(f"slots must be [T], got shape {tuple(slots.shape)}")
    T = slots.shape[0]
    _whole("slots", slots, (T,), torch.int64, dev, k_cache)
    if out is None:
        dtype = dtype or torch.bfloat16
        out = _new(k_cache, ((T, Hkv, D),) * 2, stream, dtype)
    else:
        dtype = dtype or out[0].dtype
        for name, t in zip(("out[0]", "out[1]"), out):
            _whole(name, t, (T, Hkv, D), dtype, dev, k_cache)
    _run("fastmax_cache_read_q8", lib().fastmax_cache_read_q8, dev, stream,
         k_cache.data_ptr(), v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), cache,
         slots.data_ptr(), out[0].data_ptr(), out[1].data_ptr(), T, Hkv, D, pages, page,
         _dtype_code(out[0]))
    return tuple(out)


def paged_q8_workspace_bytes(S, T, Hq, Hkv, D, max_q, max_len, window, sinks, dt) -> int:
    return int(lib().fastmax_paged_q8_workspace_bytes(S, T, Hq, Hkv, D, max_q, max_len, window,
                                                      sinks, dt))


def fastmax_paged_fwd_q8(q, k_cache, v_cache, k_scale, v_scale, table, lens, q_start=None,
                         max_q=None, max_len=None, p=2, scale=None, window=0, sinks=0, out=None,
                         workspace=None, stream=None):
    """fastmax_paged_fwd over a cache of 8-bit rows (fastmax_cache_append_q8); q
    [T, Hq, D] and O in float32 or bfloat16."""
    _on_gpu(q, 3, "[T, Hq, D]")
    T, Hq, D = q.shape
    dtype, dev, dt = q.dtype, q.get_device(), _dtype_code(q)
    Hkv = k_cache.shape[1] if k_cache.dim() == 4 else 0
    pages, page, cache = _cache_q8_of(q, k_cache, v_cache, k_scale, v_scale, Hkv)
    if table.dim() != 2:
        raise ValueError(f"table must be [S, cols], got shape {tuple(table.shape)}")
    S, cols = table.shape
    int32 = _torch().int32
    _whole("table", table, (S, cols), int32, dev, q)
    _whole("lens", lens, (S,), int32, dev, q)
    if q_start is not None:
        _whole("q_start", q_start, (S + 1,), int32, dev, q)
    if max_q is None:
        max_q = 1 if q_start is None else T
    if max_len is None:
        max_len = cols * page
    if out is None:
        out, = _new(q, ((T, Hq, D),), stream)
    else:
        _whole("out", out, (T, Hq, D), dtype, dev, q)
    workspace, ws_n = _workspace(
        q, workspace,
        lambda: paged_q8_workspace_bytes(S, T, Hq, Hkv, D, max_q, max_len, window, sinks, dt), stream)
    _run("fastmax_paged_fwd_q8", lib().fastmax_paged_fwd_q8, dev, stream,
         q.data_ptr(), _LL3(0, *q.stride()[:2]), k_cache.data_ptr(), v_cache.data_ptr(),
         k_scale.data_ptr(), v_scale.data_ptr(), cache, table.data_ptr(), lens.data_ptr(),
         _ptr(q_start), out.data_ptr(), S, T, Hq, Hkv, D, pages, page, cols, max_q, max_len, p,
         1.0 if scale is None else scale, window, sinks, dt, _ptr(workspace), ws_n)
    return out


# --- packed sequences ---------------------------------------------------------
def packed_workspace_bytes(S, T, Hq, Hkv, D, dt, backward=False) -> int:
    return int(lib().fastmax_packed_workspace_bytes(S, T, Hq, Hkv, D, dt, int(bool(backward))))


def _packed_of(q, k, v, starts):
    """(S, T, Hq, Hkv, D, dtype code, strides) of packed rows, checked."""
    _on_gpu(q, 3, "[T, Hq, D]")
    T, Hq, D = q.shape
    dtype, dev, dt = q.dtype, q.get_device(), _dtype_code(q)
    Hkv = k.shape[1] if k.dim() == 3 else 0
    _rows_of("k", k, (T, Hkv, D), dtype, dev, q)
    _rows_of("v", v, (T, Hkv, D), dtype, dev, q)
    if starts.dim() != 1 or starts.shape[0] < 2:
        raise ValueError(f"starts must be [S + 1], got shape {tuple(starts.shape)}")
    _whole("starts", starts, starts.shape, _torch().int32, dev, q)
    return (starts.shape[0] - 1, T, Hq, Hkv, D, dt,
            _LL9(0, *q.stride()[:2], 0, *k.stride()[:2], 0, *v.stride()[:2]))


def fastmax_packed_fwd(q, k, v, starts, p=2, causal=False, out=None, g=None, want_g=True,
                       workspace=None, stream=None, scale=None):
    """Fastmax attention of packed sequences: q [T, Hq, D], k and v [T, Hkv, D]
    (strided views; D contiguous), starts int32 [S + 1]: sequence s has the tokens
    starts[s] .. starts[s + 1] - 1 and attends to itself.  Returns (O [T, Hq, D],
    G float32 [T, Hq]); rows of no sequence stay as they are."""
    S, T, Hq, Hkv, D, dt, st = _packed_of(q, k, v, starts)
    torch, dev = _torch(), q.get_device()
    if out is None:
        out, = _new(q, ((T, Hq, D),), stream)
    else:
        _whole("out", out, (T, Hq, D), q.dtype, dev, q)
    if g is not None:
        _whole("g", g, (T, Hq), torch.float32, dev, q)
    elif want_g:
        g, = _new(q, ((T, Hq),), stream, torch.float32)
    workspace, ws_n = _workspace(q, workspace,
                                 lambda: packed_workspace_bytes(S, T, Hq, Hkv, D, dt), stream)
    _run("fastmax_packed_fwd", lib().fastmax_packed_fwd, dev, stream,
         q.data_ptr(), k.data_ptr(), v.data_ptr(), st, starts.data_ptr(), out.data_ptr(), _ptr(g),
         S, T, Hq, Hkv, D, p, 1 if causal else 0, 1.0 if scale is None else scale, dt,
         _ptr(workspace), ws_n)
    return out, g


def fastmax_packed_bwd(q, k, v, starts, out, dout, g, p=2, causal=False, grads=None, workspace=None,
                       stream=None, scale=None):
    """Backward of fastmax_packed_fwd from its outputs: (dq [T, Hq, D], dk and dv
    [T, Hkv, D]) of sum(dout * O); ``grads``: the same three, the caller's, strided
    as they like.  Rows of no sequence stay as they are."""
    _of("grads", grads, 3)
    S, T, Hq, Hkv, D, dt, st = _packed_of(q, k, v, starts)
    torch, dtype, dev = _torch(), q.dtype, q.get_device()
    _whole("out", out, (T, Hq, D), dtype, dev, q)
    _whole("dout", dout, (T, Hq, D), dtype, dev, q)
    _whole("g", g, (T, Hq), torch.float32, dev, q)
    shapes = ((T, Hq, D), (T, Hkv, D), (T, Hkv, D))
    if grads is None:
        grads = _new(q, shapes, stream)
    else:
        for i, (t, shape) in enumerate(zip(grads, shapes)):
            _rows_of(f"grads[{i}]", t, shape, dtype, dev, q)
    workspace, ws_n = _workspace(
        q, workspace, lambda: packed_workspace_bytes(S, T, Hq, Hkv, D, dt, True), stream)
    _run("fastmax_packed_bwd", lib().fastmax_packed_bwd, dev, stream,
         q.data_ptr(), k.data_ptr(), v.data_ptr(), st, starts.data_ptr(), out.data_ptr(),
         dout.data_ptr(), g.data_ptr(), grads[0].data_ptr(), grads[1].data_ptr(),
         grads[2].data_ptr(), _LL9(*(n for t in grads for n in (0, *t.stride()[:2]))),
         S, T, Hq, Hkv, D, p, 1 if causal else 0, 1.0 if scale is None else scale, dt,
         _ptr(workspace), ws_n)
    return tuple(grads)
