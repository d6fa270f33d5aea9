"""ctypes binding of libnystra (include/nystra.h): argument marshalling only.

Every function keeps the name of the C entry point it wraps and forwards
device pointers of torch tensors plus torch's current HIP stream.  No step of
the attention is computed here, and there is no fallback: if libnystra.so is
missing or a call fails, a NystraError is raised.
"""
import ctypes
import functools
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libnystra.so")

F32, BF16 = 0, 1
LM_POOL2D, LM_SEGMENT1D = 0, 1
VARIANT_AUTO, VARIANT_GENERIC, VARIANT_TILED, VARIANT_SPLIT = 0, 1, 2, 3

# Every symbol the header declares.
EXPORTS = (
    "nystra_default_opts", "nystra_attn_forward", "nystra_attn_forward_ex",
    "nystra_exact_attn_forward", "nystra_landmark_pool", "nystra_landmark_map",
    "nystra_select_variant", "nystra_attn_workspace_size", "nystra_attn_forward_ws",
    "nystra_block_workspace_size", "nystra_block_forward", "nystra_attn_forward_noalloc",
    "nystra_block_packed_size", "nystra_block_pack_weights", "nystra_block_forward_packed",
    "nystra_layer_forward", "nystra_status_str", "nystra_last_error",
    "nystra_layer_norm_forward", "nystra_layer_norm_workspace_size", "nystra_layer_norm_backward",
    "nystra_dropout", "nystra_diff_attn_workspace_size", "nystra_diff_attn_forward",
    "nystra_diff_attn_backward",
)
STATIC_SCRATCH_BYTES = 32 << 20   # NYSTRA_STATIC_SCRATCH_BYTES
BLOCK_NYSTROM, BLOCK_EXACT = 0, 1
CAUSAL_NONE, CAUSAL_START, CAUSAL_END = 0, 1, 2
DIFF_SHORT_KEYS = 256             # NYSTRA_DIFF_SHORT_KEYS
NORM_MAX_CHANNELS = 4096
DIFF_MAX_WIDTH = 64               # of queries and keys; of values twice that


class NystraError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        detail = ""
        if _lib is not None:
            detail = _lib.nystra_status_str(status).decode()
            if status == 7:
                detail += ": " + _lib.nystra_last_error().decode()
        super().__init__(f"{where} failed with status {status} ({detail})")


class BlockShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("batch", "height", "width", "channels", "heads",
                                              "window", "shift")]


class LayerParams(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("norm1_w", "norm1_b", "norm2_w", "norm2_b",
                                                "w1", "b1", "w2", "b2")] +
                [("eps1", ctypes.c_float), ("eps2", ctypes.c_float), ("hidden", ctypes.c_int)])


class Opts(ctypes.Structure):
    _fields_ = [("pinv_iters", ctypes.c_int), ("landmark_mode", ctypes.c_int),
                ("scale", ctypes.c_float), ("variant", ctypes.c_int)]


class View(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p)] + [(n, ctypes.c_int64) for n in ("window", "head",
                                                                             "token")]


class DiffShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("n_windows", "heads", "kv_heads", "n_q", "n_k", "d_qk",
                                            "d_v", "causal")] + [("scale", ctypes.c_float)]


_lib = None
_vp = ctypes.c_void_p
_i = ctypes.c_int


def lib():
    """The loaded libnystra.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() or "
                          "python paper_2506_08520_amd/build.py")
    L = ctypes.CDLL(LIB_PATH)
    L.nystra_default_opts.argtypes = [ctypes.POINTER(Opts)]
    L.nystra_attn_forward.argtypes = [_vp] * 4 + [_i] * 6 + [_vp]
    L.nystra_attn_forward_ex.argtypes = [_vp] * 4 + [_i] * 6 + [ctypes.POINTER(Opts), _vp]
    L.nystra_exact_attn_forward.argtypes = [_vp] * 4 + [_i] * 5 + [ctypes.c_float, _vp]
    L.nystra_landmark_pool.argtypes = [_vp] * 5 + [_i] * 7 + [_vp]
    L.nystra_landmark_map.argtypes = [_i, _i, _i, _vp]
    L.nystra_select_variant.argtypes = [_i, _i, _i, _i, ctypes.POINTER(Opts)]
    L.nystra_attn_workspace_size.argtypes = [_i] * 6 + [ctypes.POINTER(Opts),
                                                         ctypes.POINTER(ctypes.c_size_t)]
    L.nystra_attn_forward_ws.argtypes = ([_vp] * 4 + [_i] * 6 +
                                         [ctypes.POINTER(Opts), _vp, ctypes.c_size_t, _vp])
    L.nystra_status_str.argtypes = [_i]
    L.nystra_status_str.restype = ctypes.c_char_p
    L.nystra_last_error.argtypes = []
    L.nystra_last_error.restype = ctypes.c_char_p
    L.nystra_block_workspace_size.argtypes = [ctypes.POINTER(BlockShape), _i, _i,
                                              ctypes.POINTER(Opts), _i,
                                              ctypes.POINTER(ctypes.c_size_t)]
    L.nystra_block_forward.argtypes = ([_vp] * 6 + [ctypes.POINTER(BlockShape), _i, _i,
                                                     ctypes.POINTER(Opts), _i, _vp,
                                                     ctypes.c_size_t, _vp])
    L.nystra_attn_forward_noalloc.argtypes = ([_vp] * 4 + [_i] * 6 +
                                              [ctypes.POINTER(Opts), _vp])
    L.nystra_block_packed_size.argtypes = [_i, _i, ctypes.POINTER(ctypes.c_size_t)]
    L.nystra_block_pack_weights.argtypes = [_vp, _vp, _i, _i, _vp, ctypes.c_size_t, _vp]
    L.nystra_block_forward_packed.argtypes = ([_vp] * 6 + [ctypes.c_size_t, _vp,
                                                           ctypes.POINTER(BlockShape), _i, _i,
                                                           ctypes.POINTER(Opts), _i, _vp,
                                                           ctypes.c_size_t, _vp])
    L.nystra_layer_forward.argtypes = ([_vp] * 6 + [ctypes.c_size_t, ctypes.POINTER(LayerParams),
                                                    _vp, ctypes.POINTER(BlockShape), _i, _i,
                                                    ctypes.POINTER(Opts), _i, _vp,
                                                    ctypes.c_size_t, _vp])
    i64, u64, size = ctypes.c_int64, ctypes.c_uint64, ctypes.c_size_t
    view, dshape = ctypes.POINTER(View), ctypes.POINTER(DiffShape)
    L.nystra_layer_norm_forward.argtypes = ([_vp, i64, _vp, _vp, _vp, i64, _vp, _vp, i64, _i,
                                             ctypes.c_float, _i, _vp])
    L.nystra_layer_norm_workspace_size.argtypes = [i64, _i, ctypes.POINTER(size)]
    L.nystra_layer_norm_backward.argtypes = ([_vp, i64, _vp, i64, _vp, _vp, _vp, _vp, i64, _vp,
                                              _vp, i64, _i, _i, _vp, size, _vp])
    L.nystra_dropout.argtypes = [_vp, _vp, _vp, i64, ctypes.c_float, u64, u64, _vp, _i, _vp]
    L.nystra_diff_attn_workspace_size.argtypes = [dshape, _i, _i, ctypes.POINTER(size)]
    L.nystra_diff_attn_forward.argtypes = ([view] * 3 + [_vp, _vp, view, _vp, _vp, dshape, _i, _vp,
                                                         size, _vp])
    L.nystra_diff_attn_backward.argtypes = ([view] * 4 + [_vp, _vp, view, _vp, _vp] + [view] * 3 +
                                            [_vp, dshape, _i, _vp, size, _vp])
    for name in EXPORTS:
        if name not in ("nystra_status_str", "nystra_last_error"):
            getattr(L, name).restype = ctypes.c_int
    _lib = L
    return L


def _check(rc, where):
    if rc != 0:
        raise NystraError(rc, where)


def _dtype_code(t):
    import torch
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _stream(stream):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def _shape(q, k, v):
    if q.dim() != 4:
        raise ValueError("tensors must be [n_windows, heads, N, d_h]")
    for t in (q, k, v):
        if t.shape != q.shape or t.dtype != q.dtype or not t.is_contiguous() or not t.is_cuda:
            raise ValueError("Q, K, V must be contiguous device tensors of one shape and dtype")
    return tuple(int(x) for x in q.shape)


def nystra_default_opts():
    o = Opts()
    _check(lib().nystra_default_opts(ctypes.byref(o)), "nystra_default_opts")
    return o


def make_opts(pinv_iters=6, landmark_mode=LM_POOL2D, scale=0.0, variant=VARIANT_AUTO):
    return Opts(pinv_iters, landmark_mode, scale, variant)


def nystra_attn_forward(q, k, v, m, out=None, stream=None):
    """PnP-Nystra with default options; returns O (same shape/dtype as q)."""
    import torch
    W, H, N, d = _shape(q, k, v)
    o = torch.empty_like(q) if out is None else out
    rc = lib().nystra_attn_forward(_ptr(q), _ptr(k), _ptr(v), _ptr(o), W, H, N, d, m,
                                   _dtype_code(q), _stream(stream))
    _check(rc, "nystra_attn_forward")
    return o


def nystra_attn_forward_ex(q, k, v, m, opts=None, out=None, stream=None):
    import torch
    W, H, N, d = _shape(q, k, v)
    o = torch.empty_like(q) if out is None else out
    po = ctypes.byref(opts) if opts is not None else None
    rc = lib().nystra_attn_forward_ex(_ptr(q), _ptr(k), _ptr(v), _ptr(o), W, H, N, d, m,
                                      _dtype_code(q), po, _stream(stream))
    _check(rc, "nystra_attn_forward_ex")
    return o


def nystra_attn_workspace_size(n_windows, heads, N, d_h, m, dtype=F32, opts=None):
    """Bytes of device workspace nystra_attn_forward_ws needs (0: none)."""
    n = ctypes.c_size_t(0)
    po = ctypes.byref(opts) if opts is not None else None
    _check(lib().nystra_attn_workspace_size(n_windows, heads, N, d_h, m, dtype, po,
                                            ctypes.byref(n)), "nystra_attn_workspace_size")
    return int(n.value)


def nystra_attn_forward_ws(q, k, v, m, opts=None, workspace=None, out=None, stream=None):
    """PnP-Nystra through the workspace entry point.  `workspace` is a device
    tensor of at least nystra_attn_workspace_size() bytes; when None, one of
    exactly that size is allocated from torch's allocator (256-byte aligned)."""
    import torch
    W, H, N, d = _shape(q, k, v)
    code = _dtype_code(q)
    o = torch.empty_like(q) if out is None else out
    need = nystra_attn_workspace_size(W, H, N, d, m, code, opts)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    nbytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    po = ctypes.byref(opts) if opts is not None else None
    rc = lib().nystra_attn_forward_ws(_ptr(q), _ptr(k), _ptr(v), _ptr(o), W, H, N, d, m, code,
                                      po, _ptr(workspace), nbytes, _stream(stream))
    _check(rc, "nystra_attn_forward_ws")
    return o


def nystra_attn_forward_noalloc(q, k, v, m, opts=None, out=None, stream=None):
    """PnP-Nystra through the allocation-free entry point (the token-split
    workspace is the library's static device array)."""
    import torch
    W, H, N, d = _shape(q, k, v)
    o = torch.empty_like(q) if out is None else out
    po = ctypes.byref(opts) if opts is not None else None
    rc = lib().nystra_attn_forward_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(o), W, H, N, d, m,
                                           _dtype_code(q), po, _stream(stream))
    _check(rc, "nystra_attn_forward_noalloc")
    return o


def nystra_block_workspace_size(shape, m, dtype=F32, opts=None, attention=BLOCK_NYSTROM):
    n = ctypes.c_size_t(0)
    po = ctypes.byref(opts) if opts is not None else None
    _check(lib().nystra_block_workspace_size(ctypes.byref(shape), m, dtype, po, attention,
                                             ctypes.byref(n)), "nystra_block_workspace_size")
    return int(n.value)


def nystra_block_forward(x, w_qkv, b_qkv, w_proj, b_proj, heads, window, shift=0, m=16,
                         opts=None, attention=BLOCK_NYSTROM, workspace=None, out=None,
                         stream=None, packed=None):
    """Window-attention block on x [B, H, W, C] (device, contiguous); returns Y
    of the same shape.  Biases may be None.  The workspace is allocated from
    torch's allocator when not given.  ``packed``: the image from
    nystra_block_pack_weights of these weights (the per-call packing is then
    skipped)."""
    import torch
    if x.dim() != 4 or not x.is_contiguous() or not x.is_cuda:
        raise ValueError("x must be a contiguous device tensor [B, H, W, C]")
    for t in (w_qkv, b_qkv, w_proj, b_proj):
        if t is not None and (t.dtype != x.dtype or not t.is_contiguous() or not t.is_cuda):
            raise ValueError("weights must be contiguous device tensors of x's dtype")
    Bn, H, W, C = (int(v) for v in x.shape)
    shape = BlockShape(Bn, H, W, C, heads, window, shift)
    code = _dtype_code(x)
    need = nystra_block_workspace_size(shape, m, code, opts, attention)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    nbytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    y = torch.empty_like(x) if out is None else out
    po = ctypes.byref(opts) if opts is not None else None
    if packed is None:
        rc = lib().nystra_block_forward(_ptr(x), _ptr(w_qkv), _ptr(b_qkv), _ptr(w_proj),
                                        _ptr(b_proj), _ptr(y), ctypes.byref(shape), m, code, po,
                                        attention, _ptr(workspace), nbytes, _stream(stream))
        _check(rc, "nystra_block_forward")
    else:
        rc = lib().nystra_block_forward_packed(_ptr(x), _ptr(w_qkv), _ptr(b_qkv), _ptr(w_proj),
                                               _ptr(b_proj), _ptr(packed),
                                               packed.numel() * packed.element_size(), _ptr(y),
                                               ctypes.byref(shape), m, code, po, attention,
                                               _ptr(workspace), nbytes, _stream(stream))
        _check(rc, "nystra_block_forward_packed")
    return y


def nystra_layer_forward(x, w_qkv, b_qkv, w_proj, b_proj, packed, norm1, norm2, w1, b1, w2, b2,
                         heads, window, shift=0, m=16, opts=None, attention=BLOCK_NYSTROM,
                         workspace=None, stream=None):
    """Transformer layer on x [B, H, W, C] (bf16, device, contiguous): the block
    between LayerNorm and residual, then LayerNorm, MLP and residual.  ``norm1``
    and ``norm2`` are (weight, bias, eps); ``w1`` [hidden, C] and ``w2``
    [C, hidden] as nn.Linear holds them; ``packed`` from
    nystra_block_pack_weights."""
    import torch
    if x.dim() != 4 or not x.is_contiguous() or not x.is_cuda:
        raise ValueError("x must be a contiguous device tensor [B, H, W, C]")
    C, hidden = int(x.shape[-1]), int(w1.shape[0])
    if tuple(w1.shape) != (hidden, C) or tuple(w2.shape) != (C, hidden):
        raise ValueError("expected w1 [hidden, C] and w2 [C, hidden]")
    sizes = ((w_qkv, 3 * C * C), (b_qkv, 3 * C), (w_proj, C * C), (b_proj, C), (w1, hidden * C),
             (b1, hidden), (w2, hidden * C), (b2, C), (norm1[0], C), (norm1[1], C),
             (norm2[0], C), (norm2[1], C))
    for t, n in sizes:
        if t is not None and (t.dtype != x.dtype or t.numel() != n or not t.is_contiguous() or
                              t.device != x.device):
            raise ValueError("weights must be contiguous tensors of x's dtype and device")
    shape = BlockShape(*(int(v) for v in x.shape), heads, window, shift)
    code = _dtype_code(x)
    need = nystra_block_workspace_size(shape, m, code, opts, attention)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    nbytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    pk = packed.numel() * packed.element_size() if packed is not None else 0
    y = torch.empty_like(x)
    lp = LayerParams(*(_ptr(t) for t in (*norm1[:2], *norm2[:2], w1, b1, w2, b2)),
                     float(norm1[2]), float(norm2[2]), hidden)
    po = ctypes.byref(opts) if opts is not None else None
    rc = lib().nystra_layer_forward(_ptr(x), _ptr(w_qkv), _ptr(b_qkv), _ptr(w_proj), _ptr(b_proj),
                                    _ptr(packed), pk, ctypes.byref(lp), _ptr(y),
                                    ctypes.byref(shape), m, code, po, attention, _ptr(workspace),
                                    nbytes, _stream(stream))
    _check(rc, "nystra_layer_forward")
    return y


def nystra_block_packed_size(channels, dtype=F32):
    """Bytes of the packed W_qkv and W_proj image (0 for channels > 256)."""
    n = ctypes.c_size_t(0)
    _check(lib().nystra_block_packed_size(int(channels), dtype, ctypes.byref(n)),
           "nystra_block_packed_size")
    return n.value


def nystra_block_pack_weights(w_qkv, w_proj, out=None, stream=None):
    """Packs w_qkv [C, 3C] and w_proj [C, C] (device, contiguous, one dtype)
    for nystra_block_forward(..., packed=); returns the uint8 image (None for
    channels > 256, where the block reads the weights as given)."""
    import torch
    C = int(w_proj.shape[0])
    for t in (w_qkv, w_proj):
        if t.dtype != w_proj.dtype or not t.is_contiguous() or not t.is_cuda:
            raise ValueError("weights must be contiguous device tensors of one dtype")
    if tuple(w_qkv.shape) != (C, 3 * C) or tuple(w_proj.shape) != (C, C):
        raise ValueError("expected w_qkv [C, 3C] and w_proj [C, C]")
    code = _dtype_code(w_proj)
    need = nystra_block_packed_size(C, code)
    if need == 0:
        return None
    if out is None:
        out = torch.empty(need, dtype=torch.uint8, device=w_proj.device)
    rc = lib().nystra_block_pack_weights(_ptr(w_qkv), _ptr(w_proj), C, code, _ptr(out),
                                         out.numel(), _stream(stream))
    _check(rc, "nystra_block_pack_weights")
    return out


def nystra_exact_attn_forward(q, k, v, scale=0.0, out=None, stream=None):
    import torch
    W, H, N, d = _shape(q, k, v)
    o = torch.empty_like(q) if out is None else out
    rc = lib().nystra_exact_attn_forward(_ptr(q), _ptr(k), _ptr(v), _ptr(o), W, H, N, d,
                                         _dtype_code(q), float(scale), _stream(stream))
    _check(rc, "nystra_exact_attn_forward")
    return o


def nystra_landmark_pool(q, k, m, mode=LM_POOL2D, with_map=True, stream=None):
    """Step 1 alone: (Qbar, Kbar) fp32 [W, H, m, d] and the int32[N] map."""
    import torch
    W, H, N, d = _shape(q, k, q)
    qb = torch.empty((W, H, m, d), dtype=torch.float32, device=q.device)
    kb = torch.empty_like(qb)
    mp = torch.empty(N, dtype=torch.int32, device=q.device) if with_map else None
    rc = lib().nystra_landmark_pool(_ptr(q), _ptr(k), _ptr(qb), _ptr(kb), _ptr(mp), W, H, N,
                                    d, m, _dtype_code(q), mode, _stream(stream))
    _check(rc, "nystra_landmark_pool")
    return qb, kb, mp


def nystra_landmark_map(N, m, mode=LM_POOL2D):
    out = np.zeros(N, dtype=np.int32)
    _check(lib().nystra_landmark_map(N, m, mode, out.ctypes.data_as(ctypes.c_void_p)),
           "nystra_landmark_map")
    return out


def nystra_select_variant(N, d_h, m, dtype=F32, opts=None):
    po = ctypes.byref(opts) if opts is not None else None
    r = lib().nystra_select_variant(N, d_h, m, dtype, po)
    if r < 0:
        raise NystraError(-r, "nystra_select_variant")
    return r


def nystra_status_str(status):
    return lib().nystra_status_str(status).decode()


# ---- training and serving a layer: LayerNorm, dropout, differential attention ----


def _placed(f):
    """Runs f on its first tensor's device and on `stream` (default: that device's
    current stream).  On a stream that is not the current one everything that f
    allocates belongs to that stream, so that nothing is reused under its kernels."""
    name = f.__code__.co_varnames[0]

    @functools.wraps(f)
    def call(*args, stream=None, **kw):
        import torch
        first = args[0] if args else kw.get(name)
        if not isinstance(first, torch.Tensor) or not first.is_cuda:
            raise ValueError(f"{f.__name__} needs device tensors")
        if stream is None and first.device.index == torch.cuda.current_device():
            return f(*args, **kw)
        with torch.cuda.device(first.device):
            if stream is None:
                return f(*args, **kw)
            if stream.device != first.device:
                raise ValueError("the stream belongs to another device than the tensors")
            with torch.cuda.stream(stream):
                return f(*args, **kw)
    return call


def _raw_stream(t):
    import torch
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _same(first, tensors, dtype=None):
    dtype, index = dtype or first.dtype, first.get_device()
    for t in tensors:
        if t is not None and (t.dtype != dtype or t.get_device() != index):
            raise ValueError(f"expected {dtype} tensors on {first.device}")


def _vector(t, n, what):
    if t is not None and (t.numel() != n or not t.is_contiguous()):
        raise ValueError(f"{what} must be contiguous with {n} elements")


def _rows(t, C):
    """The row stride of [..., C] as a list of rows (raises where there is none)."""
    if t.is_contiguous():
        return C
    if C > 1 and t.stride(-1) != 1:
        raise ValueError("the channels must be contiguous")
    try:
        stride = t.view(-1, C).stride(0)
    except RuntimeError:
        raise ValueError("the rows must lie at one stride") from None
    return stride if t.numel() > C else C


def _addr(t):
    return t.data_ptr() if t is not None else None


def _bytes(t):
    return t.numel() * t.element_size() if t is not None else 0


def _contiguous_like(t):
    import torch
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


@_placed
def nystra_layer_norm_forward(x, weight=None, bias=None, eps=1e-5, with_stats=False, out=None):
    """LayerNorm over the last dimension of x [..., C] (rows at one stride): y, or
    with_stats (y, mean, rstd) for the backward pass (fp32, one value to a row)."""
    import torch
    C = x.shape[-1] if x.dim() else 0
    code = _dtype_code(x)
    _same(x, (weight, bias, out))
    _vector(weight, C, "weight")
    _vector(bias, C, "bias")
    rows = x.numel() // max(C, 1)
    if out is None:
        out = _contiguous_like(x)
    elif out.shape != x.shape:
        raise ValueError("out must have x's shape")
    mean = rstd = None
    if with_stats:
        mean, rstd = torch.empty((2,) + x.shape[:-1], dtype=torch.float32,
                                 device=x.device).unbind(0)
    rc = lib().nystra_layer_norm_forward(x.data_ptr(), _rows(x, C), _addr(weight), _addr(bias),
                                         out.data_ptr(), _rows(out, C), _addr(mean), _addr(rstd),
                                         rows, C, eps, code, _raw_stream(x))
    _check(rc, "nystra_layer_norm_forward")
    return (out, mean, rstd) if with_stats else out


@functools.lru_cache(maxsize=256)
def nystra_layer_norm_workspace_size(rows, channels):
    n = ctypes.c_size_t(0)
    _check(lib().nystra_layer_norm_workspace_size(rows, channels, ctypes.byref(n)),
           "nystra_layer_norm_workspace_size")
    return int(n.value)


@_placed
def nystra_layer_norm_backward(dy, x, weight, mean, rstd, workspace=None):
    """(dx, dweight, dbias) of nystra_layer_norm_forward; weight may be None (ones)."""
    import torch
    C = x.shape[-1] if x.dim() else 0
    code = _dtype_code(x)
    _same(dy, (x, weight))
    _same(dy, (mean, rstd), torch.float32)
    rows = x.numel() // max(C, 1)
    if dy.shape != x.shape:
        raise ValueError("dy must have x's shape")
    _vector(weight, C, "weight")
    _vector(mean, rows, "mean")
    _vector(rstd, rows, "rstd")
    dx = _contiguous_like(x)
    dw, db = x.new_empty((2, C)).unbind(0)
    if workspace is None:
        workspace = torch.empty(nystra_layer_norm_workspace_size(rows, C), dtype=torch.uint8,
                                device=x.device)
    else:
        _same(dy, (workspace,), workspace.dtype)
    rc = lib().nystra_layer_norm_backward(dy.data_ptr(), _rows(dy, C), x.data_ptr(), _rows(x, C),
                                          _addr(weight), mean.data_ptr(), rstd.data_ptr(),
                                          dx.data_ptr(), C, dw.data_ptr(), db.data_ptr(), rows, C,
                                          code, workspace.data_ptr(), _bytes(workspace),
                                          _raw_stream(x))
    _check(rc, "nystra_layer_norm_backward")
    return dx, dw, db


@_placed
def nystra_dropout(x, p, seed=0, offset=0, state=None, residual=None, out=None):
    """residual + dropout(x) of contiguous tensors.  The mask follows from the
    element's index, `seed` and `offset` (non-negative, below 2^64): the same call on the
    gradient, without residual, is the backward pass.  `state`: int64 [2] on the device
    in place of the seed and added to the offset (for recorded graphs)."""
    import torch
    code = _dtype_code(x)
    _same(x, (residual, out))
    for t in (x, residual, out):
        if t is not None and (t.shape != x.shape or not t.is_contiguous()):
            raise ValueError("x, residual and out must be contiguous and of one shape")
    if state is not None:
        _same(x, (state,), torch.int64)
        _vector(state, 2, "state")
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise ValueError("seed and offset must be in [0, 2^64)")
    if out is None:
        out = torch.empty_like(x)
    rc = lib().nystra_dropout(x.data_ptr(), _addr(residual), out.data_ptr(), x.numel(), p, seed,
                              offset, _addr(state), code, _raw_stream(x))
    _check(rc, "nystra_dropout")
    return out


def _view(t):
    s = t.stride()
    if len(s) != 4 or (s[3] != 1 and t.shape[3] > 1):
        raise ValueError("expected [windows, heads, tokens, width] with contiguous rows")
    return View(t.data_ptr(), s[0], s[1], s[2])


def _diff_shape(q, k, v, lam, kv_len, scale, causal):
    import torch
    if q.dim() != 4 or k.dim() != 4 or v.dim() != 4:
        raise ValueError("expected [windows, heads, tokens, width]")
    _same(q, (k, v))
    _same(q, (lam,), torch.float32)
    W, H2, nq, d = q.shape
    Wv, G, nk, dv = v.shape
    if H2 % 2 != 0 or k.shape != (W, 2 * G, nk, d) or Wv != W:
        raise ValueError("expected q [W, 2H, n_q, d], k [W, 2G, n_k, d] and v [W, G, n_k, d_v]")
    _vector(lam, H2 // 2, "lam")
    if kv_len is not None:
        _same(q, (kv_len,), torch.int32)
        _vector(kv_len, W, "kv_len")
    return (W, H2 // 2, G, nq, nk, d, dv, causal, scale)


@functools.lru_cache(maxsize=256)
def _diff_workspace(shape, backward, dtype):
    n = ctypes.c_size_t(0)
    _check(lib().nystra_diff_attn_workspace_size(DiffShape(*shape), int(backward), dtype,
                                                 ctypes.byref(n)),
           "nystra_diff_attn_workspace_size")
    return int(n.value)


def nystra_diff_attn_workspace_size(shape, backward=False, dtype=F32):
    """Bytes of workspace for a DiffShape (forward: 0 unless the keys are split)."""
    return _diff_workspace(tuple(getattr(shape, n) for n, _ in DiffShape._fields_),
                           bool(backward), dtype)


def _diff_buffer(q, workspace, shape, backward, code):
    """(tensor, address, bytes) of the caller's workspace, or of one made for the call."""
    import torch
    if workspace is not None:
        _same(q, (workspace,), workspace.dtype)
        return workspace, workspace.data_ptr(), _bytes(workspace)
    need = _diff_workspace(shape, backward, code)
    if need == 0:
        return None, None, 0
    workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    return workspace, workspace.data_ptr(), need


@_placed
def nystra_diff_attn_forward(q, k, v, lam, scale=0.0, causal=CAUSAL_NONE, kv_len=None,
                             with_saved=False, out=None, workspace=None):
    """Differential attention, O = (softmax(s Q1 K1^T) - lam softmax(s Q2 K2^T)) V, of
    q [W, 2H, n_q, d], k [W, 2G, n_k, d] and v [W, G, n_k, d_v] (heads 2h and 2h + 1 of q
    and k are the two maps of head h; G divides H), lam fp32 [H]; any strides with
    contiguous rows.  kv_len: int32 [W], the keys of each window; causal: CAUSAL_NONE,
    CAUSAL_START or CAUSAL_END.  Returns O [W, H, n_q, d_v] or, with_saved, (O, saved):
    what the backward pass needs besides the inputs."""
    import torch
    shape = _diff_shape(q, k, v, lam, kv_len, scale, causal)
    code = _dtype_code(q)
    W, H, _, nq, nk, _, dv = shape[:7]
    if out is None:
        out = q.new_empty((W, H, nq, dv))
    else:
        _same(q, (out,))
        if out.shape != (W, H, nq, dv):
            raise ValueError(f"out must be {[W, H, nq, dv]}")
    maps = sums = None
    if with_saved:
        sums = torch.empty((W, 2 * H, nq, 2), dtype=torch.float32, device=q.device)
        if code != BF16 or nk > DIFF_SHORT_KEYS:
            # the second map's output, and in bf16, whose output is rounded, the first's
            maps = torch.empty((W, H, nq) + ((2, dv) if code == BF16 else (dv,)),
                               dtype=torch.float32, device=q.device)
    workspace, ws, nbytes = _diff_buffer(q, workspace, shape, False, code)
    rc = lib().nystra_diff_attn_forward(_view(q), _view(k), _view(v), lam.data_ptr(),
                                        _addr(kv_len), _view(out), _addr(maps), _addr(sums),
                                        DiffShape(*shape), code, ws, nbytes, _raw_stream(q))
    _check(rc, "nystra_diff_attn_forward")
    return (out, (maps, sums)) if with_saved else out


@_placed
def nystra_diff_attn_backward(do, q, k, v, lam, o, saved, scale=0.0, causal=CAUSAL_NONE,
                              kv_len=None, grads=None, workspace=None):
    """(dq, dk, dv, dlam) of nystra_diff_attn_forward from its inputs, its output and
    what it saved.  grads: (dq, dk, dv) to write into, strided like the inputs may be."""
    import torch
    shape = _diff_shape(q, k, v, lam, kv_len, scale, causal)
    code = _dtype_code(q)
    W, H, _, nq, nk, _, dv = shape[:7]
    maps, sums = saved
    if do.shape != (W, H, nq, dv) or o.shape != (W, H, nq, dv):
        raise ValueError(f"do and o must be {[W, H, nq, dv]}")
    _same(do, (q, o))
    _same(do, (sums, maps), torch.float32)
    _vector(maps, o.numel() * (2 if code == BF16 else 1), "the saved maps")
    _vector(sums, 4 * W * H * nq, "the saved sums")
    if grads is None:
        grads = tuple(t.new_empty(t.shape) for t in (q, k, v))
    else:
        _same(do, grads)
        if any(t.shape != like.shape for t, like in zip(grads, (q, k, v))):
            raise ValueError("the gradients must have their inputs' shapes")
    dq, dk, dv_ = grads
    dlam = torch.empty_like(lam)
    workspace, ws, nbytes = _diff_buffer(q, workspace, shape, True, code)
    rc = lib().nystra_diff_attn_backward(_view(do), _view(q), _view(k), _view(v), lam.data_ptr(),
                                         _addr(kv_len), _view(o), _addr(maps), _addr(sums),
                                         _view(dq), _view(dk), _view(dv_), dlam.data_ptr(),
                                         DiffShape(*shape), code, ws, nbytes, _raw_stream(q))
    _check(rc, "nystra_diff_attn_backward")
    return dq, dk, dv_, dlam
