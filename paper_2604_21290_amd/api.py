"""Thin ctypes binding of libgraphleap.so (include/graphleap.h).

Argument marshalling only: tensors are passed as device pointers, streams as
hipStream_t; every step of the path runs in the library's HIP kernels.  No call
is recorded by autograd: its outputs are detached, also where an input requires
a gradient.  The
binding allocates outputs and workspaces with torch when the caller does not
pass them (PyTorch supplies device memory and streams, nothing else).

The library must have been built (python -m paper_2604_21290_amd.build);
loading raises if it is missing -- there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
import warnings
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgraphleap.so")

GL_F32, GL_BF16 = 0, 1
GL_SCHED_LOOKAHEAD, GL_SCHED_STANDARD, GL_SCHED_LOOKAHEAD_FUSED = 0, 1, 2
GL_TIME_BUILD, GL_TIME_UPDATE, GL_TIME_FUSED, GL_TIME_LINEAR = 0, 1, 2, 3
GL_ACT_NONE, GL_ACT_GELU, GL_ACT_SILU = 0, 1, 2
GL_NORM_LAYER, GL_NORM_RMS = 0, 1
GL_MAX_KD, GL_MAX_M, GL_MAX_K = 64, 4096, 64
GL_MAX_Q8_K = 131071

STATUS = {0: "GL_OK", 1: "GL_ERR_NULL_PTR", 2: "GL_ERR_BAD_SHAPE", 3: "GL_ERR_BAD_K",
          4: "GL_ERR_UNSUPPORTED", 5: "GL_ERR_ALIGNMENT", 6: "GL_ERR_ALIAS", 7: "GL_ERR_HIP",
          8: "GL_ERR_BAD_HANDLE", 9: "GL_ERR_WORKSPACE"}

_vp, _i, _f, _sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
_ll = ctypes.c_longlong

VIG_PARAMS = ("W_in", "b_in", "W_upd", "b_upd", "W_out", "b_out", "W_1", "b_1", "W_2", "b_2")


class VigParams(ctypes.Structure):
    """gl_vig_params: device pointers of one full block's weights (NULL biases allowed)."""
    _fields_ = [(n, ctypes.c_void_p) for n in VIG_PARAMS]

# name -> argtypes (every entry point returns gl_status as int unless noted)
SIGNATURES = {
    "gl_knn_graph": [_vp, _i, _i, _i, _vp, _i, _i, _i, _i, _vp, _vp],
    "gl_pool_keys": [_vp, _i, _i, _i, _i, _i, _i, _vp, _vp],
    "gl_max_pool_nodes": [_vp, _i, _i, _i, _i, _i, _i, _vp, _vp],
    "gl_mrconv_workspace_bytes": [_i, _i, _i, _i, _i, _i],
    "gl_mrconv": [_vp, _i, _i, _i, _vp, _i, _vp, _i, _vp, _vp, _i, _i, _vp, _vp, _sz, _vp],
    "gl_mrconv_noalloc": [_vp, _i, _i, _i, _vp, _i, _vp, _i, _vp, _vp, _i, _i, _vp, _vp],
    "gl_mrconv_heads": [_vp, _i, _i, _i, _vp, _i, _vp, _i, _vp, _vp, _i, _i, _vp, _vp, _sz, _vp],
    "gl_mrconv_heads_workspace_bytes": [_i, _i, _i, _i, _i, _i],
    "gl_lookahead_create": [_vp, _vp, ctypes.POINTER(_vp)],
    "gl_lookahead_destroy": [_vp],
    "gl_lookahead_set_profiling": [_vp, _i],
    "gl_lookahead_kernel_times": [_vp, _i, ctypes.POINTER(_f), _i, ctypes.POINTER(_i)],
    "gl_lookahead_bootstrap": [_vp, _vp, _i, _i, _i, _i, _i, _vp, _i, _i, _i, _vp],
    "gl_graphleap_workspace_bytes": [_i, _i, _i, _i, _i, _i, _i],
    "gl_graphleap_block": [_vp, _vp, _i, _i, _i, _i, _i, _vp, _vp, _i, _vp, _vp, _i, _vp, _vp, _i,
                           _vp, _sz],
    "gl_graphleap_stack": [_vp, _vp, _i, _i, _i, _i, _i, _i, _i, ctypes.POINTER(_i), _vp, _vp, _i,
                           _i, _vp, _vp, _vp, _vp, _vp, _sz],
    "gl_linear": [_vp, _i, _i, _vp, _vp, _i, _i, _i, _vp, _i, _vp, _vp],
    "gl_vig_workspace_bytes": [_i, _i, _i, _i, _i, _i, _i],
    "gl_vig_block": [_vp, _vp, _i, _i, _i, _i, _i, _i, _vp, ctypes.POINTER(VigParams), _i, _vp,
                     _sz, _vp, _vp, _i, _vp],
    "gl_vig_stack": [_vp, _vp, _i, _i, _i, _i, _i, _i, _i, ctypes.POINTER(_i),
                     ctypes.POINTER(VigParams), _i, _i, _vp, _sz, _vp],
    "gl_layer_norm": [_vp, _i, _i, _ll, _vp, _vp, _f, _i, _vp, _vp, _vp, _vp],
    "gl_layer_norm_backward_workspace_bytes": [_i, _i, _i],
    "gl_layer_norm_backward": [_vp, _ll, _vp, _ll, _i, _i, _vp, _vp, _vp, _i, _vp, _vp, _vp, _vp,
                               _sz, _vp],
    "gl_q8_row_bytes": [_i],
    "gl_quantize_rows": [_vp, _i, _i, _ll, _i, _vp, _vp, _vp],
    "gl_layer_norm_q8": [_vp, _i, _i, _ll, _vp, _vp, _f, _i, _vp, _vp, _vp],
    "gl_linear_q8": [_vp, _vp, _i, _i, _vp, _vp, _vp, _i, _i, _vp, _i, _vp, _vp],
    "gl_gated_linear_workspace_bytes": [_i, _i, _i, _i],
    "gl_gated_linear": [_vp, _i, _i, _vp, _vp, _i, _i, _i, _vp, _vp, _vp, _sz, _vp],
    "gl_linear_backward_workspace_bytes": [_i, _i, _i, _i],
    "gl_linear_backward": [_vp, _vp, _i, _i, _vp, _i, _i, _vp, _vp, _vp, _vp, _sz, _vp],
    "gl_gated_linear_backward_workspace_bytes": [_i, _i, _i, _i],
    "gl_gated_linear_backward": [_vp, _vp, _i, _i, _vp, _vp, _i, _i, _i, _vp, _vp, _vp, _vp, _sz, _vp],
    "gl_residual_norm": [_vp, _ll, _vp, _ll, _i, _i, _i, _f, _i, _vp, _vp, _vp, _vp, _i, _vp, _vp, _i,
                         _vp, _vp, _vp, _vp, _vp, _vp, _vp],
    "gl_residual_norm_backward_workspace_bytes": [_i, _i, _i],
    "gl_residual_norm_backward": [_vp, _ll, _vp, _ll, _vp, _ll, _vp, _ll, _i, _i, _i, _i, _vp, _vp, _vp,
                                  _vp, _vp, _vp, _vp, _vp, _i, _vp, _i, _vp, _vp, _vp, _vp, _vp, _vp,
                                  _vp, _vp, _vp, _sz, _vp],
    "gl_status_string": [_i],
    "gl_last_error": [],
    "gl_version": [],
}
RESTYPES = {"gl_status_string": ctypes.c_char_p, "gl_last_error": ctypes.c_char_p,
            "gl_vig_workspace_bytes": ctypes.c_size_t, "gl_mrconv_workspace_bytes": ctypes.c_size_t,
            "gl_mrconv_heads_workspace_bytes": ctypes.c_size_t,
            "gl_layer_norm_backward_workspace_bytes": ctypes.c_size_t,
            "gl_gated_linear_workspace_bytes": ctypes.c_size_t,
            "gl_linear_backward_workspace_bytes": ctypes.c_size_t,
            "gl_gated_linear_backward_workspace_bytes": ctypes.c_size_t,
            "gl_residual_norm_backward_workspace_bytes": ctypes.c_size_t,
            "gl_graphleap_workspace_bytes": ctypes.c_size_t}

_lib = None


class GraphLeapError(RuntimeError):
    def __init__(self, name: str, status: int, detail: str):
        super().__init__(f"{name}: {STATUS.get(status, status)}: {detail}")
        self.status = status


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_2604_21290_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        for name, args in SIGNATURES.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = RESTYPES.get(name, ctypes.c_int)
        _lib = L
    return _lib


_native = None


class _NoCalls:
    """In place of _calls.so where it cannot be loaded: every form is left to the Python path."""
    layer_norm = layer_norm_backward = quantize_rows = layer_norm_q8 = linear_q8 = gated_linear = \
        linear_backward = gated_linear_backward = residual_norm = residual_norm_backward = staticmethod(
            lambda *args: None)


def _calls():
    """The native argument marshalling of the short calls (csrc/calls.cpp).  It saves some
    4 us a call; the Python path makes the same calls of the library without it."""
    global _native
    if _native is None:
        lib()
        try:
            from . import _calls as native
            native.open(LIB_PATH)
        except (ImportError, OSError) as e:
            warnings.warn("_calls.so cannot be loaded, the short calls are marshalled in Python "
                          f"(`python -m paper_2604_21290_amd.build` builds it): {e}", RuntimeWarning, stacklevel=3)
            native = _NoCalls
        _native = native
    return _native


def _check(name: str, status: int):
    if status != 0:
        raise GraphLeapError(name, status, lib().gl_last_error().decode())


def _call(name: str, *args):
    _check(name, getattr(lib(), name)(*args))


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return GL_F32
    if t.dtype == torch.bfloat16:
        return GL_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _p(t):
    if t is None:
        return None
    if isinstance(t, Workspace):
        return ctypes.c_void_p(t.ptr)
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors must be contiguous device tensors")
    return ctypes.c_void_p(t.data_ptr())


def _s(stream) -> ctypes.c_void_p:
    # the current stream's handle without a torch.cuda.Stream around it: 0.2 us, not 2.9
    return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
                           if stream is None else stream.cuda_stream)


# ---------------------------------------------------------------------------
# single calls
# ---------------------------------------------------------------------------
def knn_graph(x: torch.Tensor, k: int, dilation: int = 1, keys: torch.Tensor | None = None,
              out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """idx[B, N, k] int32: dilated kNN of each row of x among keys (or x)."""
    B, N, C = x.shape
    M = N if keys is None else keys.shape[1]
    if out is None:
        out = torch.empty((B, N, k), dtype=torch.int32, device=x.device)
    _call("gl_knn_graph", _p(x), B, N, C, _p(keys), M, k, dilation, _dt(x), _p(out), _s(stream))
    return out


def pool_keys(x: torch.Tensor, H: int, W: int, r: int, out: torch.Tensor | None = None,
              stream=None) -> torch.Tensor:
    B, N, C = x.shape
    if out is None:
        out = torch.empty((B, (H // r) * (W // r), C), dtype=x.dtype, device=x.device)
    _call("gl_pool_keys", _p(x), B, H, W, C, r, _dt(x), _p(out), _s(stream))
    return out


def max_pool_nodes(x: torch.Tensor, H: int, W: int, r: int = 2, out: torch.Tensor | None = None,
                   stream=None) -> torch.Tensor:
    """Node reduction between pyramid stages: r x r max pooling of the H x W grid."""
    B, N, C = x.shape
    if out is None:
        out = torch.empty((B, (H // r) * (W // r), C), dtype=x.dtype, device=x.device)
    _call("gl_max_pool_nodes", _p(x), B, H, W, C, r, _dt(x), _p(out), _s(stream))
    return out


class Workspace:
    """A caller-owned device workspace: a torch uint8 buffer (or none when the
    call needs 0 bytes), passed as pointer and size."""

    def __init__(self, nbytes: int, device):
        self.nbytes = int(nbytes)
        self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=device) if nbytes else None
        self.ptr = self.buf.data_ptr() if nbytes else None

    def record_stream(self, s):
        if self.buf is not None:
            self.buf.record_stream(s)


def mrconv_workspace(B: int, N: int, C: int, k: int, Cout: int, dtype, device) -> Workspace:
    """Workspace of gl_mrconv / gl_mrconv_heads for this layer (empty when the
    fused tile needs none)."""
    dt = GL_BF16 if dtype == torch.bfloat16 else GL_F32
    return Workspace(lib().gl_mrconv_workspace_bytes(B, N, C, k, Cout, dt), device)


def mrconv(x: torch.Tensor, idx: torch.Tensor, W: torch.Tensor, bias: torch.Tensor | None = None,
           keys: torch.Tensor | None = None, out: torch.Tensor | None = None,
           stream=None, ws: Workspace | None = None) -> torch.Tensor:
    """out[B, N, Cout] = [x_i, max_j (keys_j - x_i)] W^T + bias (gl_mrconv).
    ws: the call's workspace (allocated here when not given)."""
    B, N, C = x.shape
    M = N if keys is None else keys.shape[1]
    k = idx.shape[2]
    Cout = W.shape[0]
    if out is None:
        out = torch.empty((B, N, Cout), dtype=x.dtype, device=x.device)
    if ws is None:
        ws = mrconv_workspace(B, N, C, k, Cout, x.dtype, x.device)
    _call("gl_mrconv", _p(x), B, N, C, _p(keys), M, _p(idx), k, _p(W), _p(bias), Cout, _dt(x),
          _p(out), _p(ws), ws.nbytes, _s(stream))
    return out


def mrconv_heads_workspace(B: int, N: int, C: int, k: int, heads: int, dtype, device) -> Workspace:
    """Workspace of gl_mrconv_heads for this layer (empty for the grouped kernel)."""
    dt = GL_BF16 if dtype == torch.bfloat16 else GL_F32
    return Workspace(lib().gl_mrconv_heads_workspace_bytes(B, N, C, k, heads, dt), device)


def mrconv_heads(x: torch.Tensor, idx: torch.Tensor, Wh: torch.Tensor,
                 bias: torch.Tensor | None = None, keys: torch.Tensor | None = None,
                 out: torch.Tensor | None = None, stream=None,
                 ws: Workspace | None = None) -> torch.Tensor:
    """The multi-head update (gl_mrconv_heads): Wh [H, hd, 2hd] holds each head's
    [W_x,h | W_m,h]; out[B, N, C] with C = H * hd."""
    B, N, C = x.shape
    H, hd, two_hd = Wh.shape
    if H * hd != C or two_hd != 2 * hd:
        raise ValueError(f"mrconv_heads: Wh {tuple(Wh.shape)} does not match C={C}")
    M = N if keys is None else keys.shape[1]
    k = idx.shape[2]
    if out is None:
        out = torch.empty((B, N, C), dtype=x.dtype, device=x.device)
    if ws is None:
        ws = mrconv_heads_workspace(B, N, C, k, H, x.dtype, x.device)
    _call("gl_mrconv_heads", _p(x), B, N, C, _p(keys), M, _p(idx), k, _p(Wh), _p(bias), H,
          _dt(x), _p(out), _p(ws), ws.nbytes, _s(stream))
    return out


def mrconv_noalloc(x: torch.Tensor, idx: torch.Tensor, W: torch.Tensor,
                   bias: torch.Tensor | None = None, keys: torch.Tensor | None = None,
                   out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """gl_mrconv_noalloc: the update with the library's own scratch buffer (no
    workspace; calls on one device must not overlap)."""
    B, N, C = x.shape
    M = N if keys is None else keys.shape[1]
    Cout = W.shape[0]
    if out is None:
        out = torch.empty((B, N, Cout), dtype=x.dtype, device=x.device)
    _call("gl_mrconv_noalloc", _p(x), B, N, C, _p(keys), M, _p(idx), idx.shape[2], _p(W), _p(bias),
          Cout, _dt(x), _p(out), _s(stream))
    return out


def linear(x: torch.Tensor, W: torch.Tensor, bias: torch.Tensor | None = None,
           act_in: int = GL_ACT_NONE, act_out: int = GL_ACT_NONE,
           residual: torch.Tensor | None = None, out: torch.Tensor | None = None,
           stream=None) -> torch.Tensor:
    """out[..., Cout] = act_out(act_in(x) W^T + bias) + residual over the last axis."""
    K = x.shape[-1]
    R = x.numel() // K
    Cout = W.shape[0]
    if out is None:
        out = torch.empty(x.shape[:-1] + (Cout,), dtype=x.dtype, device=x.device)
    _call("gl_linear", _p(x), R, K, _p(W), _p(bias), Cout, act_in, act_out, _p(residual), _dt(x),
          _p(out), _s(stream))
    return out


# ---------------------------------------------------------------------------
# layer norm and 8-bit layers: these calls take a few microseconds on the device, so
# their ordinary form (current stream, outputs allocated here) goes through native
# marshalling first, which returns None for anything else.  Like every call of this module
# they are not recorded by autograd: a gradient is asked for by layer_norm_backward
# ---------------------------------------------------------------------------
class Q8Rows:
    """8-bit rows (gl_quantize_rows): q [..., Kp] int8, whose last Kp - K bytes
    are zero, scale [...] float32 and the rows' length K; the values are
    q[..., :K] * scale[..., None]."""
    __slots__ = ("q", "scale", "K")

    def __init__(self, q: torch.Tensor, scale: torch.Tensor, K: int):
        self.q, self.scale, self.K = q, scale, K

    @property
    def shape(self):
        return self.q.shape[:-1] + (self.K,)

    def dequantize(self, dtype=torch.float32) -> torch.Tensor:
        return (self.q[..., : self.K].float() * self.scale[..., None]).to(dtype)


def q8_row_bytes(K: int) -> int:
    """Bytes of one 8-bit row of K values (K rounded up to 16)."""
    n = lib().gl_q8_row_bytes(K)
    if not n:
        raise GraphLeapError("gl_q8_row_bytes", 2, f"K={K} outside [1, {GL_MAX_Q8_K}]")
    return n


def _count(name: str, *ns: int):
    """The library's counts are 32 bits: a larger one is refused here, not passed on cut short."""
    if max(ns) > 0x7fffffff:
        raise GraphLeapError(name, 2, f"counts {ns} past 2^31 - 1")


def _choice(name: str, value: int):
    """An activation or a norm is 32 bits to the library too, which names an unknown one itself."""
    if not -0x80000000 <= value <= 0x7fffffff:
        raise GraphLeapError(name, 4, f"unknown choice {value}")


def _rows(x: torch.Tensor):
    """(R, C, ld) of a device tensor whose leading axes are rows a uniform stride apart."""
    if not x.is_cuda or x.dim() < 1:
        raise ValueError("rows must be a device tensor")
    if x.get_device() != torch.cuda.current_device():
        raise ValueError(f"tensors are on {x.device}, the current device is {torch.cuda.current_device()}")
    if x.is_neg():
        raise ValueError("rows are a negated view: resolve_neg() makes them a plain tensor")
    sh = x.shape
    C = sh[-1]
    R = x.numel() // C if C else 0
    _count("rows", R, C)
    if x.is_contiguous():
        return R, C, C
    st = x.stride()
    if C > 1 and st[-1] != 1:
        raise ValueError("the last axis of rows must be contiguous")
    ld = rows = None
    for n, d in zip(reversed(sh[:-1]), reversed(st[:-1])):
        if n == 1:
            continue
        if ld is None:
            ld, rows = d, n
        elif d == ld * rows:
            rows *= n
        else:
            raise ValueError(f"rows of shape {tuple(sh)} and strides {st} are not a uniform stride apart")
    return R, C, C if ld is None else ld


def _like(name: str, t, shape: tuple, dtype, x: torch.Tensor):
    """An argument that must be contiguous and have this shape and type, on x's device."""
    if t is not None and (t.shape != shape or t.dtype != dtype or t.get_device() != x.get_device()
                          or not t.is_contiguous() or t.is_neg()):
        if t.is_neg():
            raise ValueError(f"{name} is a negated view: resolve_neg() makes it a plain tensor")
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on "
                         f"{x.device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t


def _new(shape, dtype, x: torch.Tensor, stream):
    """A tensor to write on `stream` (the current one if None)."""
    if stream is None:
        return x.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return x.new_empty(shape, dtype=dtype)


def _hold(stream, *ts):
    """Tensors of other streams that `stream` uses are not handed out again before it has."""
    if stream is not None:
        for t in ts:
            if t is not None:
                t.record_stream(stream)


def _ptr(t):
    return None if t is None else t.data_ptr()


def layer_norm(x: torch.Tensor, gamma: torch.Tensor | None = None,
               beta: torch.Tensor | None = None, eps: float = 1e-5, stats: bool = False,
               out: torch.Tensor | None = None, stream=None):
    """(x - mean) * rstd * gamma + beta over the last axis (gl_layer_norm).  x may
    be a slice of wider rows.  stats: return (out, mean, rstd), the row statistics
    in float32 that layer_norm_backward takes.  The outputs are detached: inside an autograd
    graph, call this and layer_norm_backward from a torch.autograd.Function."""
    if stream is None and out is None:
        r = (_native or _calls()).layer_norm(x, gamma, beta, eps, stats)
        if r is not None:
            return r
    R, C, ld = _rows(x)
    _like("gamma", gamma, (C,), x.dtype, x)
    _like("beta", beta, (C,), x.dtype, x)
    if out is None:
        out = _new(x.shape, x.dtype, x, stream)
    else:
        _like("out", out, x.shape, x.dtype, x)
    mean = rstd = None
    if stats:
        mean = _new(x.shape[:-1], torch.float32, x, stream)
        rstd = _new(x.shape[:-1], torch.float32, x, stream)
    _hold(stream, x, gamma, beta, out)
    _call("gl_layer_norm", x.data_ptr(), R, C, ld, _ptr(gamma), _ptr(beta), eps, _dt(x),
          out.data_ptr(), _ptr(mean), _ptr(rstd), _s(stream))
    return (out, mean, rstd) if stats else out


def layer_norm_backward_workspace(x: torch.Tensor) -> Workspace:
    """Workspace of gl_layer_norm_backward for rows shaped like x."""
    R, C, _ = _rows(x)
    return Workspace(lib().gl_layer_norm_backward_workspace_bytes(R, C, _dt(x)), x.device)


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                        gamma: torch.Tensor | None = None, need=(True, True, True),
                        ws: Workspace | None = None, stream=None):
    """(dx, dgamma, dbeta) of layer_norm from its output's gradient dy, its input
    and the row statistics it returned (gl_layer_norm_backward); dgamma and dbeta
    are float32 sums over all rows.  need: which of the three to compute (None
    for the others).  ws: the call's workspace (allocated here when not given)."""
    if stream is None and ws is None and all(need):
        r = (_native or _calls()).layer_norm_backward(dy, x, mean, rstd, gamma)
        if r is not None:
            return r
    R, C, ldx = _rows(x)
    Rd, Cd, lddy = _rows(dy)
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError(f"dy {dy.dtype} {tuple(dy.shape)} does not match x {x.dtype} {tuple(x.shape)}")
    _like("mean", mean, x.shape[:-1], torch.float32, x)
    _like("rstd", rstd, x.shape[:-1], torch.float32, x)
    _like("gamma", gamma, (C,), x.dtype, x)
    dx = _new(x.shape, x.dtype, x, stream) if need[0] else None
    dgamma = _new((C,), torch.float32, x, stream) if need[1] else None
    dbeta = _new((C,), torch.float32, x, stream) if need[2] else None
    wp, wn = None, 0
    if need[1] or need[2]:
        if ws is None:
            wn = lib().gl_layer_norm_backward_workspace_bytes(R, C, _dt(x))
            if wn:
                buf = _new((wn,), torch.uint8, x, stream)
                wp = buf.data_ptr()
        else:
            wp, wn = ws.ptr, ws.nbytes
            if stream is not None:
                ws.record_stream(stream)
    _hold(stream, dy, x, mean, rstd, gamma)
    _call("gl_layer_norm_backward", dy.data_ptr(), lddy, x.data_ptr(), ldx, R, C, mean.data_ptr(),
          rstd.data_ptr(), _ptr(gamma), _dt(x), _ptr(dx), _ptr(dgamma), _ptr(dbeta), wp, wn,
          _s(stream))
    return dx, dgamma, dbeta


def _q8_out(x: torch.Tensor, R: int, K: int, out: Q8Rows | None, stream) -> Q8Rows:
    Kp = (K + 15) // 16 * 16
    if out is None:
        return Q8Rows(_new(x.shape[:-1] + (Kp,), torch.int8, x, stream),
                      _new(x.shape[:-1], torch.float32, x, stream), K)
    if out.K != K:
        raise ValueError(f"out holds rows of {out.K} values, x has {K}")
    _like("out.q", out.q, x.shape[:-1] + (Kp,), torch.int8, x)
    _like("out.scale", out.scale, x.shape[:-1], torch.float32, x)
    _hold(stream, out.q, out.scale)
    return out


def quantize_rows(x: torch.Tensor, out: Q8Rows | None = None, stream=None) -> Q8Rows:
    """x's rows (its last axis) as 8-bit integers with a scale each
    (gl_quantize_rows): activations per token, or a weight per output channel."""
    if stream is None and out is None:
        r = (_native or _calls()).quantize_rows(x)
        if r is not None:
            return Q8Rows(r[0], r[1], x.shape[-1])
    R, K, ld = _rows(x)
    out = _q8_out(x, R, K, out, stream)
    _hold(stream, x)
    _call("gl_quantize_rows", x.data_ptr(), R, K, ld, _dt(x), out.q.data_ptr(), out.scale.data_ptr(),
          _s(stream))
    return out


def layer_norm_q8(x: torch.Tensor, gamma: torch.Tensor | None = None,
                  beta: torch.Tensor | None = None, eps: float = 1e-5, out: Q8Rows | None = None,
                  stream=None) -> Q8Rows:
    """layer_norm and quantize_rows in one pass (gl_layer_norm_q8)."""
    if stream is None and out is None:
        r = (_native or _calls()).layer_norm_q8(x, gamma, beta, eps)
        if r is not None:
            return Q8Rows(r[0], r[1], x.shape[-1])
    R, K, ld = _rows(x)
    _like("gamma", gamma, (K,), x.dtype, x)
    _like("beta", beta, (K,), x.dtype, x)
    out = _q8_out(x, R, K, out, stream)
    _hold(stream, x, gamma, beta)
    _call("gl_layer_norm_q8", x.data_ptr(), R, K, ld, _ptr(gamma), _ptr(beta), eps, _dt(x),
          out.q.data_ptr(), out.scale.data_ptr(), _s(stream))
    return out


def linear_q8(x: Q8Rows, W: Q8Rows, bias: torch.Tensor | None = None, act_out: int = GL_ACT_NONE,
              residual: torch.Tensor | None = None, dtype=torch.bfloat16,
              out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """out[..., Cout] = act_out(x W^T + bias) + residual of 8-bit rows x and weights
    W [Cout, K] (gl_linear_q8); bias, residual and out are in `dtype`.  The output is
    detached; 8-bit rows have no gradient."""
    if stream is None and out is None and (dtype is torch.bfloat16 or dtype is torch.float32):
        r = (_native or _calls()).linear_q8(x.q, x.scale, x.K, W.q, W.scale, W.K, bias, act_out, residual,
                                            dtype is torch.bfloat16)
        if r is not None:
            return r
    R, Kp, _ = _rows(x.q)
    if W.q.dim() != 2 or x.K != W.K:
        raise ValueError(f"linear_q8: rows {tuple(x.shape)} do not match weights {tuple(W.shape)}")
    Cout, lead = W.q.shape[0], x.q.shape[:-1]
    _count("linear_q8", Cout)
    want = (x.K + 15) // 16 * 16
    _like("x.q", x.q, lead + (want,), torch.int8, x.q)
    _like("x.scale", x.scale, lead, torch.float32, x.q)
    _like("W.q", W.q, (Cout, want), torch.int8, x.q)
    _like("W.scale", W.scale, (Cout,), torch.float32, x.q)
    _like("bias", bias, (Cout,), dtype, x.q)
    _like("residual", residual, lead + (Cout,), dtype, x.q)
    if out is None:
        out = _new(lead + (Cout,), dtype, x.q, stream)
    else:
        _like("out", out, lead + (Cout,), dtype, x.q)
    _hold(stream, x.q, x.scale, W.q, W.scale, bias, residual, out)
    _call("gl_linear_q8", x.q.data_ptr(), x.scale.data_ptr(), R, x.K, W.q.data_ptr(),
          W.scale.data_ptr(), _ptr(bias), Cout, act_out, _ptr(residual), _dt(out), out.data_ptr(),
          _s(stream))
    return out


# ---------------------------------------------------------------------------
# training an FFN: the gated layer, the layers' backward passes, and the end of a block with
# its gradients.  Nothing is recorded by autograd here either: a forward pass returns what
# its backward pass takes
# ---------------------------------------------------------------------------
def _matrix(name: str, t: torch.Tensor, shape: tuple | None, x: torch.Tensor) -> torch.Tensor:
    """A contiguous tensor of the layer x -> ...: of this shape, or of any (x itself)."""
    if not t.is_cuda or t.dim() < 1:
        raise ValueError(f"{name} must be a device tensor")
    if t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{name} is on {t.device}, the current device is {torch.cuda.current_device()}")
    return _like(name, t, t.shape if shape is None else shape, x.dtype, x)


def _scratch(nbytes: int, x: torch.Tensor, ws, stream):
    """The pointer and size of a call's workspace, and its buffer if it is allocated here."""
    if ws is not None:
        if stream is not None:
            ws.record_stream(stream)
        return ws.ptr, ws.nbytes, None
    if not nbytes:
        return None, 0, None
    buf = _new((nbytes,), torch.uint8, x, stream)
    return buf.data_ptr(), nbytes, buf


def _layer(name: str, x: torch.Tensor, W: torch.Tensor):
    """(R, K, outputs) of a layer's input rows and weight."""
    _matrix("x", x, None, x)
    K = x.shape[-1]
    if W.dim() != 2 or W.shape[1] != K:
        raise ValueError(f"{name}: W {tuple(W.shape)} does not match rows {tuple(x.shape)}")
    _matrix("W", W, W.shape, x)
    R = x.numel() // K if K else 0
    _count(name, R, K, W.shape[0])
    return R, K, W.shape[0]


def _halves(name: str, W: torch.Tensor) -> int:
    if W.shape[0] % 2:
        raise ValueError(f"{name}: W's rows are the gate's and as many others, got {W.shape[0]}")
    return W.shape[0] // 2


def gated_linear_workspace(x: torch.Tensor, W: torch.Tensor) -> Workspace:
    """Workspace of gl_gated_linear for this layer (empty for many, not for all of whole vectors)."""
    R, K, N = _layer("gated_linear", x, W)
    return Workspace(lib().gl_gated_linear_workspace_bytes(R, K, _halves("gated_linear", W), _dt(x)), x.device)


def gated_linear(x: torch.Tensor, W: torch.Tensor, bias: torch.Tensor | None = None,
                 act: int = GL_ACT_SILU, keep: bool = False, out: torch.Tensor | None = None,
                 ws: Workspace | None = None, stream=None):
    """h[..., F] = act(g) * u with [g | u] = x W^T + bias over the last axis, W [2F, K]
    (gl_gated_linear).  keep: return (h, pre), pre [..., 2F] the products that
    gated_linear_backward takes.  The outputs are detached."""
    if stream is None and out is None and ws is None:
        r = (_native or _calls()).gated_linear(x, W, bias, act, keep)
        if r is not None:
            return r
    R, K, N = _layer("gated_linear", x, W)
    F = _halves("gated_linear", W)
    _choice("gated_linear", act)
    _like("bias", bias, (N,), x.dtype, x)
    lead = x.shape[:-1]
    if out is None:
        out = _new(lead + (F,), x.dtype, x, stream)
    else:
        _like("out", out, lead + (F,), x.dtype, x)
    pre = _new(lead + (N,), x.dtype, x, stream) if keep else None
    dt = _dt(x)
    wp, wn, _buf = _scratch(0 if ws is not None else lib().gl_gated_linear_workspace_bytes(R, K, F, dt), x, ws, stream)
    _hold(stream, x, W, bias, out)
    _call("gl_gated_linear", x.data_ptr(), R, K, W.data_ptr(), _ptr(bias), F, act, dt, out.data_ptr(), _ptr(pre), wp,
          wn, _s(stream))
    return (out, pre) if keep else out


def linear_backward_workspace(x: torch.Tensor, W: torch.Tensor) -> Workspace:
    """Workspace of gl_linear_backward for this layer."""
    R, K, N = _layer("linear_backward", x, W)
    return Workspace(lib().gl_linear_backward_workspace_bytes(R, K, N, _dt(x)), x.device)


def gated_linear_backward_workspace(x: torch.Tensor, W: torch.Tensor) -> Workspace:
    """Workspace of gl_gated_linear_backward for this layer."""
    R, K, N = _layer("gated_linear_backward", x, W)
    return Workspace(lib().gl_gated_linear_backward_workspace_bytes(R, K, _halves("gated_linear_backward", W), _dt(x)),
                     x.device)


def _layer_grads(need, x, W, N, stream):
    if not any(need):
        raise ValueError("no gradient is asked for")
    return (_new(x.shape, x.dtype, x, stream) if need[0] else None,
            _new(W.shape, x.dtype, x, stream) if need[1] else None,
            _new((N,), torch.float32, x, stream) if need[2] else None)


def linear_backward(dy: torch.Tensor, x: torch.Tensor, W: torch.Tensor, need=(True, True, True),
                    ws: Workspace | None = None, stream=None):
    """(dx, dW, dbias) of linear without activations, out = x W^T + bias, from its output's
    gradient dy [..., Cout] (gl_linear_backward); dW in x's type, dbias a float32 sum over
    all rows.  need: which of the three to compute (None for the others).  ws: the call's
    workspace (allocated here when not given)."""
    if stream is None and ws is None and any(need):
        r = (_native or _calls()).linear_backward(dy, x, W, *need)
        if r is not None:
            return r
    R, K, N = _layer("linear_backward", x, W)
    _matrix("dy", dy, x.shape[:-1] + (N,), x)
    dt = _dt(x)
    dx, dW, db = _layer_grads(need, x, W, N, stream)
    wp, wn, _buf = _scratch(0 if ws is not None else lib().gl_linear_backward_workspace_bytes(R, K, N, dt), x, ws, stream)
    _hold(stream, dy, x, W)
    _call("gl_linear_backward", dy.data_ptr(), x.data_ptr(), R, K, W.data_ptr(), N, dt, _ptr(dx), _ptr(dW), _ptr(db), wp,
          wn, _s(stream))
    return dx, dW, db


def gated_linear_backward(dh: torch.Tensor, x: torch.Tensor, W: torch.Tensor, pre: torch.Tensor,
                          act: int = GL_ACT_SILU, need=(True, True, True), ws: Workspace | None = None,
                          stream=None):
    """(dx, dW, dbias) of gated_linear from its output's gradient dh [..., F], its input and
    weight, and the products that it kept (gl_gated_linear_backward); dW in x's type,
    dbias [2F] a float32 sum over all rows.  need and ws as in linear_backward."""
    if stream is None and ws is None and any(need):
        r = (_native or _calls()).gated_linear_backward(dh, x, W, pre, act, *need)
        if r is not None:
            return r
    R, K, N = _layer("gated_linear_backward", x, W)
    F = _halves("gated_linear_backward", W)
    _choice("gated_linear_backward", act)
    _matrix("dh", dh, x.shape[:-1] + (F,), x)
    _matrix("pre", pre, x.shape[:-1] + (N,), x)
    dt = _dt(x)
    dx, dW, db = _layer_grads(need, x, W, N, stream)
    wp, wn, _buf = _scratch(0 if ws is not None else lib().gl_gated_linear_backward_workspace_bytes(R, K, F, dt), x, ws,
                            stream)
    _hold(stream, dh, x, W, pre)
    _call("gl_gated_linear_backward", dh.data_ptr(), x.data_ptr(), R, K, W.data_ptr(), pre.data_ptr(), F, act, dt,
          _ptr(dx), _ptr(dW), _ptr(db), wp, wn, _s(stream))
    return dx, dW, db


class ResidualStats(NamedTuple):
    """The rows' statistics of residual_norm's norms, float32 (None: there is none)."""
    mean_b: torch.Tensor | None
    rstd_b: torch.Tensor | None
    mean_s: torch.Tensor | None
    rstd_s: torch.Tensor | None


class ResidualGrads(NamedTuple):
    """The gradients of residual_norm (None: of an argument that was None).  dpost and dnorm
    are (gamma's, beta's); all but dx and db are float32."""
    dx: torch.Tensor
    db: torch.Tensor
    dgate: torch.Tensor | None
    dscale: torch.Tensor | None
    dpost: tuple | None
    dnorm: tuple | None


def _norm_pair(name: str, w, C: int, x: torch.Tensor):
    if w is None:
        return None, None
    gamma, beta = w
    _like(f"{name}'s gamma", gamma, (C,), x.dtype, x)
    _like(f"{name}'s beta", beta, (C,), x.dtype, x)
    return gamma, beta


def _rows_per_gate(gate, x: torch.Tensor, R: int) -> int:
    """A gate's axes are x's first ones: one for each image, or for each row."""
    if gate is None:
        return 1
    if gate.dim() < 1 or gate.dim() >= x.dim() or not gate.numel():
        raise ValueError(f"gate {tuple(gate.shape)}: its axes must be the first of {tuple(x.shape)}, without the last")
    _like("gate", gate, x.shape[:gate.dim()], torch.float32, x)
    return R // gate.numel()


def residual_norm(x: torch.Tensor, b: torch.Tensor, post=None, scale: torch.Tensor | None = None,
                  gate: torch.Tensor | None = None, norm=None, kind: int = GL_NORM_LAYER, eps: float = 1e-5,
                  stats: bool = False, stream=None):
    """(s, y): s = x + gate * scale * n, y = norm(s) for the next block (gl_residual_norm),
    where n is a block's output b, normalised first if post is given.  post, norm: (gamma,
    beta) of a norm over the last axis, either None for ones and zeros; None for no norm (y
    is None without norm).  scale [C]; gate: float32, of x's first axes (an image's, or a
    row's).  kind: GL_NORM_LAYER or GL_NORM_RMS.  x and b may be slices of wider rows.
    stats: return (s, y, ResidualStats), which residual_norm_backward takes.  The outputs
    are detached."""
    if stream is None:
        r = (_native or _calls()).residual_norm(x, b, post, scale, gate, norm, kind, eps, stats)
        if r is not None:
            return (r[0], r[1], ResidualStats(*r[2])) if stats else r
    R, C, ldx = _rows(x)
    Rb, Cb, ldb = _rows(b)
    _choice("residual_norm", kind)
    if b.shape != x.shape or b.dtype != x.dtype or b.get_device() != x.get_device():
        raise ValueError(f"b {b.dtype} {tuple(b.shape)} does not match x {x.dtype} {tuple(x.shape)}")
    g1, b1 = _norm_pair("post", post, C, x)
    g2, b2 = _norm_pair("norm", norm, C, x)
    _like("scale", scale, (C,), x.dtype, x)
    per = _rows_per_gate(gate, x, R)
    dt = _dt(x)
    s = _new(x.shape, x.dtype, x, stream)
    y = _new(x.shape, x.dtype, x, stream) if norm is not None else None

    def kept(on):
        return _new(x.shape[:-1], torch.float32, x, stream) if stats and on else None
    st = ResidualStats(kept(post is not None and kind == GL_NORM_LAYER), kept(post is not None),
                       kept(norm is not None and kind == GL_NORM_LAYER), kept(norm is not None))
    _hold(stream, x, b, g1, b1, g2, b2, scale, gate)
    _call("gl_residual_norm", x.data_ptr(), ldx, b.data_ptr(), ldb, R, C, kind, eps, post is not None, _ptr(g1),
          _ptr(b1), _ptr(scale), _ptr(gate), per, _ptr(g2), _ptr(b2), dt, s.data_ptr(), _ptr(y), _ptr(st.mean_b),
          _ptr(st.rstd_b), _ptr(st.mean_s), _ptr(st.rstd_s), _s(stream))
    return (s, y, st) if stats else (s, y)


def residual_norm_backward_workspace(b: torch.Tensor) -> Workspace:
    """Workspace of gl_residual_norm_backward for rows shaped like b."""
    R, C, _ = _rows(b)
    return Workspace(lib().gl_residual_norm_backward_workspace_bytes(R, C, _dt(b)), b.device)


def residual_norm_backward(ds: torch.Tensor | None, dy: torch.Tensor | None, b: torch.Tensor,
                           s: torch.Tensor | None, stats, post=None, scale: torch.Tensor | None = None,
                           gate: torch.Tensor | None = None, norm=None, kind: int = GL_NORM_LAYER,
                           ws: Workspace | None = None, stream=None) -> ResidualGrads:
    """The gradients of residual_norm, from those of its outputs (either may be None), what
    it was given and returned, and its ResidualStats (gl_residual_norm_backward).  ws: the
    call's workspace (allocated here when not given)."""
    if stream is None and ws is None:
        r = (_native or _calls()).residual_norm_backward(ds, dy, b, s, stats, post, scale, gate, norm, kind)
        if r is not None:
            return ResidualGrads(*r)
    R, C, ldb = _rows(b)
    _choice("residual_norm_backward", kind)
    if ds is None and dy is None:
        raise ValueError("ds or dy is required")
    if (dy is None) != (norm is None):
        raise ValueError("dy and norm belong together")
    ld = [0, 0, 0]
    for i, (name, t) in enumerate((("ds", ds), ("dy", dy), ("s", s if dy is not None else None))):
        if t is None:
            if name == "s" and dy is not None:
                raise ValueError("s is required with dy")
            continue
        ld[i] = _rows(t)[2]
        if t.shape != b.shape or t.dtype != b.dtype or t.get_device() != b.get_device():
            raise ValueError(f"{name} {t.dtype} {tuple(t.shape)} does not match b {b.dtype} {tuple(b.shape)}")
    g1, b1 = _norm_pair("post", post, C, b)
    g2, b2 = _norm_pair("norm", norm, C, b)
    _like("scale", scale, (C,), b.dtype, b)
    per = _rows_per_gate(gate, b, R)
    mean_b, rstd_b, mean_s, rstd_s = stats
    for name, t, on in (("mean_b", mean_b, post is not None and kind == GL_NORM_LAYER), ("rstd_b", rstd_b, post is not None),
                        ("mean_s", mean_s, norm is not None and kind == GL_NORM_LAYER), ("rstd_s", rstd_s, norm is not None)):
        if on and t is None:
            raise ValueError(f"{name} is required")
        _like(name, t, b.shape[:-1], torch.float32, b)
    dt = _dt(b)

    def vec(on, n=(C,)):
        return _new(n, torch.float32, b, stream) if on else None
    dx, db = _new(b.shape, b.dtype, b, stream), _new(b.shape, b.dtype, b, stream)
    dgate, dscale = vec(gate is not None, () if gate is None else gate.shape), vec(scale is not None)
    dg1, db1, dg2, db2 = (vec(t is not None) for t in (g1, b1, g2, b2))
    want = any(t is not None for t in (dgate, dscale, dg1, db1, dg2, db2))
    need = lib().gl_residual_norm_backward_workspace_bytes(R, C, dt) if want and ws is None else 0
    wp, wn, _buf = _scratch(need, b, ws, stream)
    _hold(stream, ds, dy, b, s, mean_b, rstd_b, mean_s, rstd_s, g1, b1, g2, scale, gate)
    _call("gl_residual_norm_backward", _ptr(ds), ld[0], _ptr(dy), ld[1], b.data_ptr(), ldb,
          None if dy is None else s.data_ptr(), ld[2], R, C, kind, post is not None, _ptr(mean_b), _ptr(rstd_b),
          _ptr(mean_s), _ptr(rstd_s), _ptr(g1), _ptr(b1), _ptr(scale), _ptr(gate), per, _ptr(g2), dt, dx.data_ptr(),
          db.data_ptr(), _ptr(dgate), _ptr(dscale), _ptr(dg1), _ptr(db1), _ptr(dg2), _ptr(db2), wp, wn, _s(stream))
    return ResidualGrads(dx, db, dgate, dscale, None if post is None else (dg1, db1),
                         None if norm is None else (dg2, db2))


def vig_params(p: dict) -> VigParams:
    """gl_vig_params from a dict of device tensors keyed like VIG_PARAMS."""
    return VigParams(*[(p[n].data_ptr() if p.get(n) is not None else None) for n in VIG_PARAMS])


def _grid(N, H, W):
    """The node grid (H, W); a plain N-node set is the N x 1 grid."""
    if H is None:
        return N, 1
    if H * W != N:
        raise GraphLeapError("grid", 2, f"H*W={H * W} != N={N}")
    return H, W


def vig_workspace(x0: torch.Tensor, k: int, H=None, W=None, pool_r: int = 1) -> torch.Tensor:
    B, N, C = x0.shape
    H, W = _grid(N, H, W)
    n = lib().gl_vig_workspace_bytes(B, H, W, C, pool_r, k, _dt(x0))
    if not n:
        raise GraphLeapError("gl_vig_workspace_bytes", 2, "bad shape")
    return torch.empty(n, dtype=torch.uint8, device=x0.device)


# ---------------------------------------------------------------------------
# lookahead
# ---------------------------------------------------------------------------
class Lookahead:
    """Owns a gl_lookahead handle bound to an update stream and a build stream."""

    def __init__(self, s_update=None, s_build=None):
        self.s_update = s_update if s_update is not None else torch.cuda.current_stream()
        self.s_build = s_build if s_build is not None else torch.cuda.Stream()
        h = ctypes.c_void_p()
        _call("gl_lookahead_create", _s(self.s_update), _s(self.s_build), ctypes.byref(h))
        self._h = h

    def close(self):
        if self._h is not None and self._h.value:
            _call("gl_lookahead_destroy", self._h)
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _keep(self, *ts):
        for t in ts:
            if t is not None:
                t.record_stream(self.s_build)

    def set_profiling(self, max_records: int):
        _call("gl_lookahead_set_profiling", self._h, max_records)

    def kernel_times_ms(self, which: int = GL_TIME_BUILD, cap: int = 1 << 16) -> list:
        """Durations (ms) of the profiled builds (GL_TIME_BUILD), updates
        (GL_TIME_UPDATE) or one-launch blocks (GL_TIME_FUSED)."""
        buf = (ctypes.c_float * cap)()
        n = ctypes.c_int()
        _call("gl_lookahead_kernel_times", self._h, which, buf, cap, ctypes.byref(n))
        return list(buf[: n.value])

    def bootstrap(self, x0, H, W, k, dilation0, pool_r=1, keys_ws=None, idx0=None):
        B, N, C = x0.shape
        if idx0 is None:
            idx0 = torch.empty((B, N, k), dtype=torch.int32, device=x0.device)
        self._keep(x0, keys_ws, idx0)
        _call("gl_lookahead_bootstrap", self._h, _p(x0), B, H, W, C, pool_r, _p(keys_ws), k,
              dilation0, _dt(x0), _p(idx0))
        return idx0

    def block(self, x_in, H, W, idx_use, Wt, bias=None, pool_r=1, keys_ws=None, x_out=None,
              idx_next=None, dilation_next=1, ws: Workspace | None = None):
        B, N, C = x_in.shape
        k = idx_use.shape[2]
        if x_out is None:
            x_out = torch.empty_like(x_in)
        if ws is None:
            ws = graphleap_workspace(x_in, H, W, k, pool_r)
        self._keep(x_in, keys_ws, idx_next)
        _call("gl_graphleap_block", self._h, _p(x_in), B, H, W, C, pool_r, _p(keys_ws),
              _p(idx_use), k, _p(Wt), _p(bias), _dt(x_in), _p(x_out), _p(idx_next),
              dilation_next, _p(ws), ws.nbytes)
        return x_out

    def vig_block(self, x_in, idx_use, params: dict, ws, u_out=None, x_out=None, idx_next=None,
                  dilation_next=1, H=None, W=None, pool_r=1):
        """One full ViG block; returns (x_out, u_out).  With pool_r > 1 the
        graphs index U's keys pooled pool_r x pool_r over the H x W grid."""
        B, N, C = x_in.shape
        H, W = _grid(N, H, W)
        k = idx_use.shape[2]
        x_out = torch.empty_like(x_in) if x_out is None else x_out
        u_out = torch.empty_like(x_in) if u_out is None else u_out
        self._keep(x_in, ws, u_out, idx_use, idx_next)
        pp = vig_params(params)
        _call("gl_vig_block", self._h, _p(x_in), B, H, W, C, pool_r, k, _p(idx_use),
              ctypes.byref(pp), _dt(x_in), _p(ws), ws.numel(), _p(u_out), _p(idx_next),
              dilation_next, _p(x_out))
        return x_out, u_out

    def vig_stack(self, x0, params: list, dilations, k, schedule=GL_SCHED_LOOKAHEAD_FUSED,
                  ws=None, x_out=None, H=None, W=None, pool_r=1):
        """len(dilations) full ViG blocks; params: list of dicts of device tensors.
        With pool_r > 1 keys are pooled pool_r x pool_r over the H x W grid."""
        B, N, C = x0.shape
        H, W = _grid(N, H, W)
        L = len(dilations)
        ws = vig_workspace(x0, k, H, W, pool_r) if ws is None else ws
        x_out = torch.empty_like(x0) if x_out is None else x_out
        dil = (ctypes.c_int * L)(*dilations)
        arr = (VigParams * L)(*[vig_params(p) for p in params])
        self._keep(x0, ws)
        _call("gl_vig_stack", self._h, _p(x0), B, H, W, C, pool_r, L, k, dil, arr, _dt(x0),
              schedule, _p(ws), ws.numel(), _p(x_out))
        return x_out

    def stack(self, x0, H, W, Ws, bs, dilations, k, pool_r=1, schedule=GL_SCHED_LOOKAHEAD,
              ws=None, x_out=None):
        """Run len(dilations) blocks; Ws [L, C, 2C], bs [L, C] or None."""
        B, N, C = x0.shape
        L = len(dilations)
        if ws is None:
            ws = make_stack_workspace(x0, H, W, k, pool_r)
        if x_out is None:
            x_out = torch.empty_like(x0)
        dil = (ctypes.c_int * L)(*dilations)
        self._keep(x0, ws["x"], ws["idx"], ws["keys"])
        ws["mr"].record_stream(self.s_build)
        _call("gl_graphleap_stack", self._h, _p(x0), B, H, W, C, pool_r, L, k, dil, _p(Ws),
              _p(bs), _dt(x0), schedule, _p(ws["x"]), _p(ws["idx"]), _p(ws["keys"]), _p(x_out),
              _p(ws["mr"]), ws["mr"].nbytes)
        return x_out


def graphleap_workspace(x0: torch.Tensor, H: int, W: int, k: int, pool_r: int = 1) -> Workspace:
    """The MRConv workspace of gl_graphleap_block / gl_graphleap_stack."""
    B, N, C = x0.shape
    return Workspace(lib().gl_graphleap_workspace_bytes(B, H, W, C, pool_r, k, _dt(x0)), x0.device)


def make_stack_workspace(x0: torch.Tensor, H: int, W: int, k: int, pool_r: int = 1) -> dict:
    B, N, C = x0.shape
    M = (H // pool_r) * (W // pool_r)
    return {
        "x": torch.empty((2, B, N, C), dtype=x0.dtype, device=x0.device),
        "idx": torch.empty((2, B, N, k), dtype=torch.int32, device=x0.device),
        "keys": torch.empty((B, M, C), dtype=x0.dtype, device=x0.device) if pool_r > 1 else None,
        "mr": graphleap_workspace(x0, H, W, k, pool_r),
    }


def version() -> int:
    return lib().gl_version()
