"""Thin ctypes binding of libtoma's C ABI (include/toma.h): same names, argument marshalling only.

Every function takes torch CUDA tensors (device memory and the current stream come from torch),
hands raw pointers to the library and raises TomaError on a non-zero status.  There is no CPU
path: if libtoma.so has not been built, loading it fails.
"""
import ctypes
import functools
import math
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# (a process started with TOMA_SANITIZE=1 loads the host-sanitizer build instead: CPU argument checks only)
LIB_PATH = os.path.join(_HERE, "libtoma_san.so" if os.environ.get("TOMA_SANITIZE", "0") == "1" else "libtoma.so")

TOMA_F32, TOMA_BF16, TOMA_MX8 = 0, 1, 2
ACTIVATIONS = {"none": 0, "gelu": 1, "gelu_tanh": 2, "silu": 3}
TOMA_REUSE_IDX, TOMA_REUSE_A, TOMA_RECOMPUTE_WEIGHTS = 1, 2, 4
EXPORTS = ("toma_workspace_bytes", "toma_status_string", "toma_select", "toma_select_static", "toma_merge", "toma_map_bytes",
           "toma_map_build", "toma_merge_cached", "toma_attend", "toma_cross_attend", "toma_unmerge", "toma_unmerge_pinv", "toma_recompute_cache_bytes", "toma_merge_recompute",
           "toma_unmerge_recompute", "toma_layer", "toma_mlp", "toma_mx_scale_stride", "toma_mx_quantize", "toma_mx_quantize_weight",
           "toma_mx_dequantize", "toma_rmsnorm", "toma_linear_workspace_bytes", "toma_linear", "toma_ffn_workspace_bytes", "toma_ffn",
           "toma_profile_enable",
           "toma_profile_kernel_name", "toma_profile_read", "toma_profile_map_product", "toma_profile_linear", "toma_profile_linear_kernel",
           "toma_profile_greedy_parts")


class TomaError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class toma_desc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("W", ctypes.c_int32), ("C", ctypes.c_int32),
                ("tile_h", ctypes.c_int32), ("tile_w", ctypes.c_int32), ("d_loc", ctypes.c_int32),
                ("merge_regions", ctypes.c_int32), ("tau", ctypes.c_float), ("logit_scale", ctypes.c_float),
                ("dtype", ctypes.c_int32)]

    @property
    def P(self):
        return (self.H // self.tile_h) * (self.W // self.tile_w)

    @property
    def N(self):
        return self.H * self.W

    @property
    def D(self):
        return self.P * self.d_loc


class toma_attn_desc(ctypes.Structure):
    _fields_ = [("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("t_extra", ctypes.c_int32)]


class toma_norm_desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("C", ctypes.c_int32), ("eps", ctypes.c_float), ("x_type", ctypes.c_int32),
                ("y_type", ctypes.c_int32)]


class toma_linear_desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("K", ctypes.c_int32), ("N", ctypes.c_int32), ("x_type", ctypes.c_int32),
                ("y_type", ctypes.c_int32), ("act", ctypes.c_int32)]


class toma_ffn_desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("C", ctypes.c_int32), ("hidden", ctypes.c_int32), ("eps", ctypes.c_float),
                ("x_type", ctypes.c_int32), ("w_type", ctypes.c_int32), ("act", ctypes.c_int32)]


_lib = None


def lib():
    """Load libtoma.so (built by `python -m paper_2509_10918_amd.build`); no fallback exists."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with paper_2509_10918_amd/build.py "
                              "(hipcc, gfx950); there is no CPU fallback")
        L = ctypes.CDLL(LIB_PATH)
        L.toma_workspace_bytes.restype = ctypes.c_size_t
        L.toma_workspace_bytes.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
        L.toma_status_string.restype = ctypes.c_char_p
        L.toma_status_string.argtypes = [ctypes.c_int]
        vp, sz = ctypes.c_void_p, ctypes.c_size_t
        L.toma_select.argtypes = [vp, vp, vp, vp, vp, vp, sz, vp]
        L.toma_select_static.argtypes = [vp, vp, vp, vp, vp, vp]
        L.toma_select_static.restype = ctypes.c_int
        L.toma_merge.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.toma_map_bytes.restype = ctypes.c_size_t
        L.toma_map_bytes.argtypes = [vp]
        L.toma_map_build.argtypes = [vp, vp, vp, vp]
        L.toma_merge_cached.argtypes = [vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.toma_attend.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.toma_cross_attend.argtypes = [vp, vp, vp, vp, ctypes.c_int32, ctypes.c_int32, vp, vp, vp, vp, vp, vp, sz, vp]
        L.toma_cross_attend.restype = ctypes.c_int
        L.toma_unmerge.argtypes = [vp, vp, vp, vp, vp, ctypes.c_int32, vp, vp, sz, vp]
        L.toma_recompute_cache_bytes.restype = ctypes.c_size_t
        L.toma_recompute_cache_bytes.argtypes = [vp]
        L.toma_merge_recompute.argtypes = [vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.toma_merge_recompute.restype = ctypes.c_int
        L.toma_unmerge_recompute.argtypes = [vp, vp, vp, vp, vp, vp, ctypes.c_int32, vp, vp, sz, vp]
        L.toma_unmerge_recompute.restype = ctypes.c_int
        L.toma_unmerge_pinv.argtypes = [vp, vp, vp, vp, ctypes.c_int32, ctypes.c_float, vp, vp, sz, vp]
        L.toma_unmerge_pinv.restype = ctypes.c_int
        L.toma_layer.argtypes = [vp, vp, ctypes.c_uint32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.toma_mlp.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, vp, vp, vp, vp, vp, vp]
        i32 = ctypes.c_int32
        L.toma_mx_scale_stride.restype = sz
        L.toma_mx_scale_stride.argtypes = [i32]
        L.toma_mx_quantize.argtypes = L.toma_mx_quantize_weight.argtypes = L.toma_mx_dequantize.argtypes = [i32, i32, i32, vp, vp, vp, vp]
        L.toma_rmsnorm.argtypes = [vp] * 8
        L.toma_linear_workspace_bytes.restype = L.toma_ffn_workspace_bytes.restype = sz
        L.toma_linear_workspace_bytes.argtypes = L.toma_ffn_workspace_bytes.argtypes = [vp]
        L.toma_linear.argtypes = [vp] * 10 + [sz, vp]
        L.toma_ffn.argtypes = [vp] * 12 + [sz, vp]
        L.toma_profile_linear.argtypes = [vp, ctypes.POINTER(ctypes.c_int32)]
        L.toma_profile_linear_kernel.restype = ctypes.c_char_p
        L.toma_profile_linear_kernel.argtypes = [vp]
        for name in ("toma_profile_linear", "toma_mx_quantize", "toma_mx_quantize_weight", "toma_mx_dequantize", "toma_rmsnorm", "toma_linear", "toma_ffn"):
            getattr(L, name).restype = ctypes.c_int
        for name in ("toma_select", "toma_merge", "toma_map_build", "toma_merge_cached", "toma_attend", "toma_cross_attend", "toma_unmerge", "toma_unmerge_pinv", "toma_recompute_cache_bytes", "toma_merge_recompute",
           "toma_unmerge_recompute",
                     "toma_layer", "toma_mlp"):
            getattr(L, name).restype = ctypes.c_int
        L.toma_profile_enable.argtypes = [ctypes.c_int]
        L.toma_profile_kernel_name.restype = ctypes.c_char_p
        L.toma_profile_kernel_name.argtypes = [ctypes.c_int]
        L.toma_profile_read.argtypes = [ctypes.c_char_p, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_float)]
        L.toma_profile_map_product.argtypes = [vp, ctypes.c_int, ctypes.POINTER(ctypes.c_int32)]
        L.toma_profile_map_product.restype = ctypes.c_int
        L.toma_profile_greedy_parts.argtypes = [vp, vp, vp, vp, vp, sz, vp]
        L.toma_profile_greedy_parts.restype = ctypes.c_int
        _lib = L
    return _lib


def status_string(status):
    return lib().toma_status_string(int(status)).decode()


def make_desc(B, H, W, C, tile_h, tile_w, d_loc, merge_regions, tau, dtype, logit_scale=0.0):
    code = {torch.float32: TOMA_F32, torch.bfloat16: TOMA_BF16, "f32": TOMA_F32, "bf16": TOMA_BF16}[dtype]
    return toma_desc(B, H, W, C, tile_h, tile_w, d_loc, merge_regions, tau, logit_scale, code)


def torch_dtype(desc):
    return torch.bfloat16 if desc.dtype == TOMA_BF16 else torch.float32


def _ref(s):
    return None if s is None else ctypes.addressof(s)


def _ptr(t):
    if t is None:
        return None
    if not (t.is_cuda and t.is_contiguous()):
        raise ValueError("libtoma takes contiguous CUDA tensors")
    return t.data_ptr()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _check(status, where):
    if status != 0:
        raise TomaError(status, where)


def toma_workspace_bytes(desc, attn=None):
    return lib().toma_workspace_bytes(_ref(desc), _ref(attn))


def alloc_workspace(desc, attn=None, device="cuda"):
    n = toma_workspace_bytes(desc, attn)
    if n == 0:
        raise TomaError(2, "toma_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def toma_select(desc, X, idx, gain, gap, ws):
    _check(lib().toma_select(_ref(desc), _ptr(X), _ptr(idx), _ptr(gain), _ptr(gap), _ptr(ws), ws.numel(),
                             _stream()), "toma_select")


def toma_select_static(desc, X, idx, gain, gap):
    _check(lib().toma_select_static(_ref(desc), _ptr(X), _ptr(idx), _ptr(gain), _ptr(gap), _stream()),
           "toma_select_static")


def toma_merge(desc, X, idx, A, Z, amap, Xm, ws):
    _check(lib().toma_merge(_ref(desc), _ptr(X), _ptr(idx), _ptr(A), _ptr(Z), _ptr(amap), _ptr(Xm), _ptr(ws),
                            ws.numel(), _stream()), "toma_merge")


def toma_map_bytes(desc):
    return lib().toma_map_bytes(_ref(desc))


def toma_map_build(desc, A, amap):
    _check(lib().toma_map_build(_ref(desc), _ptr(A), _ptr(amap), _stream()), "toma_map_build")


def toma_merge_cached(desc, X, A, Z, amap, Xm, ws):
    _check(lib().toma_merge_cached(_ref(desc), _ptr(X), _ptr(A), _ptr(Z), _ptr(amap), _ptr(Xm), _ptr(ws),
                                   ws.numel(), _stream()), "toma_merge_cached")


def toma_attend(desc, attn, Xm, X_extra, Wq, Wk, Wv, Wo, O, ws):
    _check(lib().toma_attend(_ref(desc), _ref(attn), _ptr(Xm), _ptr(X_extra), _ptr(Wq), _ptr(Wk), _ptr(Wv),
                             _ptr(Wo), _ptr(O), _ptr(ws), ws.numel(), _stream()), "toma_attend")


def toma_cross_attend(desc, attn, U, Ctx, Wq, Wk, Wv, Wo, O, ws):
    _check(lib().toma_cross_attend(_ref(desc), _ref(attn), _ptr(U), _ptr(Ctx), Ctx.shape[1], Ctx.shape[2], _ptr(Wq),
                                   _ptr(Wk), _ptr(Wv), _ptr(Wo), _ptr(O), _ptr(ws), ws.numel(), _stream()),
           "toma_cross_attend")


def toma_unmerge(desc, A, Z, amap, O, Y, ws):
    _check(lib().toma_unmerge(_ref(desc), _ptr(A), _ptr(Z), _ptr(amap), _ptr(O), O.shape[1], _ptr(Y), _ptr(ws),
                              ws.numel(), _stream()), "toma_unmerge")


def toma_recompute_cache_bytes(desc):
    return lib().toma_recompute_cache_bytes(_ref(desc))


def toma_merge_recompute(desc, X, idx, Z, wcache, Xm, ws):
    _check(lib().toma_merge_recompute(_ref(desc), _ptr(X), _ptr(idx), _ptr(Z), _ptr(wcache), _ptr(Xm), _ptr(ws),
                                      ws.numel(), _stream()), "toma_merge_recompute")


def toma_unmerge_recompute(desc, X, idx, Z, wcache, O, Y, ws):
    _check(lib().toma_unmerge_recompute(_ref(desc), _ptr(X), _ptr(idx), _ptr(Z), _ptr(wcache), _ptr(O), O.shape[1],
                                        _ptr(Y), _ptr(ws), ws.numel(), _stream()), "toma_unmerge_recompute")


def toma_unmerge_pinv(desc, A, Z, O, rcond, Y, ws):
    _check(lib().toma_unmerge_pinv(_ref(desc), _ptr(A), _ptr(Z), _ptr(O), O.shape[1], float(rcond), _ptr(Y), _ptr(ws),
                                   ws.numel(), _stream()), "toma_unmerge_pinv")


def toma_layer(desc, attn, reuse_flags, X, X_extra, idx, A, Z, amap, Wq, Wk, Wv, Wo, Y, Y_extra, ws):
    _check(lib().toma_layer(_ref(desc), _ref(attn), int(reuse_flags), _ptr(X), _ptr(X_extra), _ptr(idx), _ptr(A),
                            _ptr(Z), _ptr(amap), _ptr(Wq), _ptr(Wk), _ptr(Wv), _ptr(Wo), _ptr(Y), _ptr(Y_extra),
                            _ptr(ws), ws.numel(), _stream()), "toma_layer")


def toma_mlp(In, W1, W2, Hbuf, Out):
    """Out = gelu(In W1) W2 on the rows of In ([..., C]); Hbuf is [rows, hidden] scratch."""
    C, hidden = W1.shape
    rows = In.numel() // C
    code = TOMA_BF16 if In.dtype == torch.bfloat16 else TOMA_F32
    _check(lib().toma_mlp(code, rows, C, hidden, _ptr(In), _ptr(W1), _ptr(W2), _ptr(Hbuf), _ptr(Out), _stream()),
           "toma_mlp")


# ---- operators around the core modules --------------------------------------------------------------
# These check shapes, types and the device as well: the C ABI takes bare pointers.

_TYPE = {torch.float32: TOMA_F32, torch.bfloat16: TOMA_BF16, "f32": TOMA_F32, "bf16": TOMA_BF16, "mx8": TOMA_MX8, TOMA_F32: TOMA_F32,
         TOMA_BF16: TOMA_BF16, TOMA_MX8: TOMA_MX8}
_TORCH = {TOMA_F32: torch.float32, TOMA_BF16: torch.bfloat16, TOMA_MX8: torch.uint8}


_ROWS, _WEIGHT, _CODES = range(3)   # what a tensor is


@functools.lru_cache(maxsize=1024)
def _fits(shape, want, kind):
    """Whether a contiguous tensor of this shape holds what one of the shape `want` ((rows, width), (width,)) does.  Weights: any whose last
    dimension is right.  Rows: one after the other, so that the last dimensions are one row, or all of it is flat, or (not of codes) the
    last dimension is several: the norm of single heads."""
    if math.prod(shape) != math.prod(want):
        return False
    width = want[-1]
    if len(want) == 1 or len(shape) == 1 or shape[-1] == width:
        return kind != _WEIGHT or shape[-1] == width
    if kind == _WEIGHT:
        return False
    n = 1
    for s in reversed(shape):
        n *= s
        if n == width:
            return True
    return kind == _ROWS and len(shape) > 0 and shape[-1] % width == 0


def _refuse(what, t, dtype, shape, kind, device):
    """The reason why a tensor is not taken."""
    count, got = math.prod(shape), tuple(t.shape)
    if kind == _WEIGHT and got[-1:] != shape[-1:]:
        raise ValueError(f"{what}: last dimension {shape[-1]} expected, got the shape {got}")
    if t.dtype is not dtype or t.numel() != count:
        raise ValueError(f"{what}: {count} elements of {dtype} expected, got {t.numel()} of {t.dtype}")
    if not _fits(got, shape, kind):
        raise ValueError(f"{what}: rows of {shape[-1]} expected, got the shape {got}")
    if t.get_device() < 0 or not t.is_contiguous():
        raise ValueError(f"{what}: libtoma takes contiguous CUDA tensors")
    raise ValueError(f"{what} lies on {t.device}, the current device is cuda:{device}")


class _Call:
    """Pointers of one call's tensor arguments after their checks, and the current stream.  (A small call's time is the host's: the
    device and the stream are asked for once per call.)"""

    __slots__ = ("device",)

    def __init__(self):
        self.device = torch._C._cuda_getDevice() if torch.cuda.is_initialized() else 0

    def arg(self, what, t, dtype, shape, kind=_ROWS):
        """shape: (rows, width) or (width,)"""
        if t is None:
            return None
        s = t.shape
        if (s != shape and not _fits(s, shape, kind)) or t.dtype is not dtype or t.get_device() != self.device or not t.is_contiguous():
            _refuse(what, t, dtype, shape, kind, self.device)
        return t.data_ptr()

    def codes(self, what, t, rows, width):
        return None if t is None else self.arg(what, t, torch.uint8, (rows, _scale_stride(width)), _CODES)

    def scratch(self, ws):
        """Pointer and bytes of a scratch tensor (None: no scratch)."""
        return (None, 0) if ws is None else (self.arg("ws", ws, torch.uint8, (ws.numel(),)), ws.numel())

    def stream(self):
        return torch._C._cuda_getCurrentRawStream(self.device)


def _scale_stride(K):
    return 4 * ((K + 127) // 128)


def toma_mx_scale_stride(K):
    return lib().toma_mx_scale_stride(K)


def alloc_mx(rows, K, device="cuda"):
    """Elements and scale codes of an 8-bit tensor."""
    stride = toma_mx_scale_stride(K)
    if stride == 0:
        raise TomaError(5, "toma_mx_scale_stride")
    return (torch.empty((rows, K), dtype=torch.uint8, device=device),
            torch.empty((rows, stride), dtype=torch.uint8, device=device))


def _pack_call(name, what, plain, shape, code, lead, rows, K, Q, S):
    c = _Call()
    p = c.arg(what, plain, _TORCH[max(code, 0)], shape)
    q, s = c.arg("Q", Q, torch.uint8, (rows, K)), c.codes("S", S, rows, K)
    args = (q, s, p) if what == "Y" else (p, q, s)
    _check(getattr(lib(), name)(code, *lead, *args, c.stream()), name)


def toma_mx_quantize(X, Q, S):
    """X [..., K] -> Q [rows, K], S [rows, stride] (alloc_mx)."""
    rows, K = Q.shape
    _pack_call("toma_mx_quantize", "X", X, (rows, K), _TYPE.get(X.dtype, -1), (rows, K), rows, K, Q, S)


def toma_mx_quantize_weight(W, Q, S):
    """W [K, N] -> Q [N, K], S [N, stride] (alloc_mx(N, K))."""
    K, N = W.shape
    _pack_call("toma_mx_quantize_weight", "W", W, (K, N), _TYPE.get(W.dtype, -1), (K, N), N, K, Q, S)


def toma_mx_dequantize(Q, S, Y):
    """The values of Q [rows, K], S as Y [..., K] (float32 or bfloat16)."""
    rows, K = Q.shape
    _pack_call("toma_mx_dequantize", "Y", Y, (rows, K), _TYPE.get(Y.dtype, -1), (rows, K), rows, K, Q, S)


def make_norm_desc(rows, C, eps, x_type, y_type=None):
    return toma_norm_desc(rows, C, eps, _TYPE[x_type], _TYPE[x_type if y_type is None else y_type])


def toma_rmsnorm(desc, X, R, gamma, H, Y, Ys=None):
    """X, R, H, Y: rows of C, under any leading dimensions (or several rows in the last: heads)."""
    rows, C, x, y = desc.rows, desc.C, desc.x_type, desc.y_type
    e, n, c = _TORCH.get(x), (rows, C), _Call()
    arg = c.arg
    _check(lib().toma_rmsnorm(_ref(desc), arg("X", X, e, n), arg("R", R, e, n), arg("gamma", gamma, e, (C,)), arg("H", H, e, n),
                              arg("Y", Y, e if y == x else _TORCH.get(y), n), c.codes("Ys", Ys, rows, C), c.stream()),
           "toma_rmsnorm")


def make_linear_desc(rows, K, N, x_type, y_type=None, act="none"):
    return toma_linear_desc(rows, K, N, _TYPE[x_type], _TYPE[x_type if y_type is None else y_type], ACTIVATIONS[act])


def toma_linear_workspace_bytes(desc):
    return lib().toma_linear_workspace_bytes(_ref(desc))


def _alloc_scratch(n, device):
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def alloc_linear_workspace(desc, device="cuda"):
    """Scratch of toma_linear; None when the shape needs none."""
    return _alloc_scratch(toma_linear_workspace_bytes(desc), device)


def toma_linear(desc, X, Xs, W, Ws, bias, R, Y, Ys, ws):
    rows, K, N, x = desc.rows, desc.K, desc.N, desc.x_type
    t, e, n = _TORCH.get(x), torch.float32 if x == TOMA_F32 else torch.bfloat16, (rows, N)   # e: type of bias and residual
    c = _Call()
    arg, codes = c.arg, c.codes
    w = arg("W", W, t, (N, K) if x == TOMA_MX8 else (K, N), _WEIGHT)
    _check(lib().toma_linear(_ref(desc), arg("X", X, t, (rows, K)), codes("Xs", Xs, rows, K), w, codes("Ws", Ws, N, K), arg("bias", bias, e, (N,)),
                             arg("R", R, e, n), arg("Y", Y, _TORCH.get(desc.y_type), n), codes("Ys", Ys, rows, N), *c.scratch(ws), c.stream()),
           "toma_linear")


def make_ffn_desc(rows, C, hidden, eps, x_type, w_type=None, act="gelu"):
    return toma_ffn_desc(rows, C, hidden, eps, _TYPE[x_type], _TYPE[x_type if w_type is None else w_type], ACTIVATIONS[act])


def toma_ffn_workspace_bytes(desc):
    return lib().toma_ffn_workspace_bytes(_ref(desc))


def alloc_ffn_workspace(desc, device="cuda"):
    n = toma_ffn_workspace_bytes(desc)
    if n == 0:
        raise TomaError(5, "toma_ffn_workspace_bytes")
    return _alloc_scratch(n, device)


def toma_ffn(desc, X, R, gamma, W1, W1s, b1, W2, W2s, b2, Y, ws):
    C, hidden, w = desc.C, desc.hidden, desc.w_type
    e, t, n, c = _TORCH.get(desc.x_type), _TORCH.get(w), (desc.rows, C), _Call()
    arg, codes = c.arg, c.codes
    up, down = ((hidden, C), (C, hidden)) if w == TOMA_MX8 else ((C, hidden), (hidden, C))
    w1, w2 = arg("W1", W1, t, up, _WEIGHT), arg("W2", W2, t, down, _WEIGHT)
    _check(lib().toma_ffn(_ref(desc), arg("X", X, e, n), arg("R", R, e, n), arg("gamma", gamma, e, (C,)), w1, codes("W1s", W1s, hidden, C),
                          arg("b1", b1, e, (hidden,)), w2, codes("W2s", W2s, C, hidden), arg("b2", b2, e, (C,)), arg("Y", Y, e, n),
                          *c.scratch(ws), c.stream()),
           "toma_ffn")


def toma_profile_enable(on):
    _check(lib().toma_profile_enable(1 if on else 0), "toma_profile_enable")


def toma_profile_kernel_names():
    names, i = [], 0
    while True:
        n = lib().toma_profile_kernel_name(i)
        if n is None:
            return names
        names.append(n.decode())
        i += 1


def toma_profile_read(kernel):
    """(launches, total milliseconds) of one kernel since the last read; clears them."""
    n, ms = ctypes.c_int32(0), ctypes.c_float(0.0)
    _check(lib().toma_profile_read(kernel.encode(), ctypes.byref(n), ctypes.byref(ms)), "toma_profile_read")
    return n.value, ms.value


def toma_profile_map_product(desc, which):
    """(rows, columns, K split) of the block tile of the merge (0) / unmerge (1) product or of the write
    pass of the two-pass weights (2), or None."""
    out = (ctypes.c_int32 * 3)()
    rc = lib().toma_profile_map_product(_ref(desc), int(which), out)
    return None if rc != 0 else tuple(out)


def toma_profile_linear(desc):
    """(rows, columns, K split) of toma_linear's workgroups for this descriptor."""
    out = (ctypes.c_int32 * 3)()
    _check(lib().toma_profile_linear(_ref(desc), out), "toma_profile_linear")
    return tuple(out)


def toma_profile_linear_kernel(desc):
    """Name of the kernel that toma_linear takes for this descriptor; None for an invalid one."""
    name = lib().toma_profile_linear_kernel(_ref(desc))
    return None if name is None else name.decode()


def toma_profile_greedy_parts(desc, X, idx, parts, ws):
    """toma_select through the greedy kernel that times the parts of its rounds; parts: int64
    [B * P, waves, 8] (waves = 8 for regions of 256 tokens, 2 for regions of 64)."""
    _check(lib().toma_profile_greedy_parts(_ref(desc), _ptr(X), _ptr(idx), _ptr(parts), _ptr(ws), ws.numel(), _stream()),
           "toma_profile_greedy_parts")


def alloc_cache(desc, device="cuda"):
    """Caller-owned pattern cache (idx, A, Z, amap) of one layer; amap is None when the shape uses no
    block map."""
    dt = torch_dtype(desc)
    R = desc.merge_regions
    idx = torch.empty((desc.B, desc.P, desc.d_loc), dtype=torch.int32, device=device)
    A = torch.empty((desc.B, R, desc.D // R, desc.N // R), dtype=dt, device=device)
    Z = torch.empty((desc.B, desc.D), dtype=torch.float32, device=device)
    n = toma_map_bytes(desc)
    amap = torch.empty(n, dtype=torch.uint8, device=device) if n else None
    return idx, A, Z, amap
