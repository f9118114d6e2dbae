"""ctypes binding of libvardrop.so: argument marshalling only.

Every function has the name of the C entry point it calls (include/vardrop.h).  Tensors
are torch tensors on the GPU; torch provides device memory and the current HIP stream,
nothing else.  There is no fallback: if the shared library is missing, loading fails.
"""
import ctypes
import os

import torch

F32 = 0
BF16 = 1
NORM_NONE = 0
NORM_LAYER = 1
NORM_RMS = 2
_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None

_c_int = ctypes.c_int
_c_i64 = ctypes.c_int64
_c_u32 = ctypes.c_uint32
_c_u64 = ctypes.c_uint64
_c_size = ctypes.c_size_t
_c_float = ctypes.c_float
_c_double = ctypes.c_double
_ptr = ctypes.c_void_p

# post, wp, bp, gate, gates, alpha, beta, pre, w, then b, eps, r, h, stats or the gradients and the workspace; stream
_BLOCK_NORM_FWD = [_c_int, _ptr, _ptr, _ptr, _c_int, _c_float, _c_float, _c_int, _ptr] + [_ptr, _c_float] + [_ptr] * 4
_BLOCK_NORM_BWD = [_c_int, _ptr, _ptr, _ptr, _c_int, _c_float, _c_float, _c_int, _ptr] + [_ptr] * 8 + [_c_size, _ptr]

_SIGNATURES = {
    "vardrop_create": (_c_int, [ctypes.POINTER(_ptr), _c_int]),
    "vardrop_destroy": (None, [_ptr]),
    "vardrop_strerror": (ctypes.c_char_p, [_c_int]),
    "vardrop_last_hip_error": (_c_int, [_ptr]),
    "vardrop_hash_strided_workspace_bytes": (ctypes.c_size_t, [_c_int, _c_int, _c_int]),
    "vardrop_hash_default_cutoff": (_c_int, [_c_int]),
    "vardrop_profile_select": (_c_int, [_ptr, _c_int]),
    "vardrop_profile_read": (_c_int, [_ptr, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_c_int)]),
    "vardrop_profile_stride": (_c_int, [_ptr, _c_int]),
    "vardrop_signal_after": (_c_int, [_ptr, _c_int, _ptr]),
    "vardrop_profile_read_all": (_c_int, [_ptr, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_c_int)]),
    "vardrop_kernel_name": (ctypes.c_char_p, [_c_int]),
    "vardrop_hash_workspace_bytes": (_c_size, [_c_int] * 6),
    "vardrop_hash": (_c_int, [_ptr, _ptr, _c_int, _c_int, _c_int, _c_i64, _c_i64, _c_i64, _c_int, _c_int, _c_int,
                              _ptr, _ptr, _ptr, _ptr, _c_size, _ptr]),
    "vardrop_sample_workspace_bytes": (_c_size, [_c_int]),
    "vardrop_sample": (_c_int, [_ptr, _ptr, _c_int, _c_u32, _c_u32, _c_u32, _c_u64, _c_u64,
                                _ptr, _ptr, _ptr, _ptr, _ptr, _c_size, _ptr]),
    "vardrop_sample_dev": (_c_int, [_ptr, _ptr, _c_int, _c_u32, _c_u32, _c_u32, _c_u64, _ptr, _c_int,
                                    _ptr, _ptr, _ptr, _ptr, _c_size, _ptr]),
    "vardrop_sample_nearest_workspace_bytes": (_c_size, [_c_int, _c_int]),
    "vardrop_sample_nearest": (_c_int, [_ptr, _ptr, _ptr, _c_int, _c_int, _c_u32, _c_u32, _c_u32,
                                        _ptr, _ptr, _ptr, _ptr, _ptr, _c_size, _ptr]),
    "vardrop_sample_nearest_noalloc": (_c_int, [_ptr, _ptr, _ptr, _c_int, _c_int, _c_u32, _c_u32, _c_u32,
                                                _ptr, _ptr, _ptr, _ptr]),
    "vardrop_gather": (_c_int, [_ptr, _ptr, _c_int, _c_int, _c_int, _c_int, _ptr, _c_int, _ptr, _ptr]),
    "vardrop_scatter": (_c_int, [_ptr, _ptr, _c_int, _c_int, _c_int, _c_int, _ptr, _c_int, _ptr, _ptr]),
    "vardrop_gather_dev": (_c_int, [_ptr, _ptr, _c_int, _c_int, _c_int, _c_int, _ptr, _ptr, _c_int, _ptr, _ptr, _ptr]),
    "vardrop_scatter_dev": (_c_int, [_ptr, _ptr, _c_int, _c_int, _c_int, _c_int, _ptr, _ptr, _c_int, _ptr, _ptr, _ptr]),
    "vardrop_embed_saved_bytes": (_c_size, [_c_int] * 4),
    "vardrop_embed_workspace_bytes": (_c_size, [_c_int] * 5),
    "vardrop_embed_fwd": (_c_int, [_ptr, _ptr, _c_int, _c_int, _c_int, _c_i64, _c_i64, _ptr, _c_int, _c_int,
                                   _ptr, _ptr, _c_int, _c_int, _ptr, _ptr, _ptr]),
    "vardrop_embed_bwd": (_c_int, [_ptr, _ptr, _c_int, _c_int, _c_int, _c_int, _c_int, _ptr, _ptr, _ptr,
                                   _ptr, _c_size, _ptr]),
    "vardrop_embed_fwd_dev": (_c_int, [_ptr, _ptr, _c_int, _c_int, _c_int, _c_i64, _c_i64, _ptr, _ptr, _c_int, _ptr, _c_int,
                                       _ptr, _ptr, _c_int, _c_int, _ptr, _ptr, _ptr]),
    "vardrop_embed_bwd_dev": (_c_int, [_ptr, _ptr, _c_int, _ptr, _c_int, _c_int, _c_int, _c_int, _ptr, _ptr, _ptr,
                                       _ptr, _c_size, _ptr]),
    "vardrop_attn_fwd_dev": (_c_int, [_ptr, _ptr, _c_int, _ptr, _c_int, _ptr, _c_int, _c_int, _c_int] + [_ptr] * 8 +
                             [_ptr, _ptr, _ptr, _c_size, _ptr]),
    "vardrop_attn_saved_bytes": (_c_size, [_c_int] * 5),
    "vardrop_attn_workspace_bytes": (_c_size, [_c_int] * 5),
    "vardrop_attn_fwd": (_c_int, [_ptr, _ptr, _c_int, _c_int, _c_int, _c_int, _c_int] + [_ptr] * 8 +
                         [_ptr, _ptr, _ptr, _c_size, _ptr]),
    "vardrop_gather_attn_fwd": (_c_int, [_ptr, _ptr, _c_int, _c_int, _ptr, _c_int, _c_int, _c_int, _c_int] + [_ptr] * 8 +
                                [_ptr, _ptr, _ptr, _ptr, _c_size, _ptr]),
    "vardrop_attn_bwd": (_c_int, [_ptr, _ptr, _ptr, _c_int, _c_int, _c_int, _c_int, _c_int] + [_ptr] * 4 +
                         [_ptr] + [_ptr] * 9 + [_ptr, _c_size, _ptr]),
    "vardrop_gather_attn_fwd_dev": (_c_int, [_ptr, _ptr, _c_int, _c_int, _ptr, _ptr, _c_int, _ptr, _c_int, _c_int, _c_int] +
                                    [_ptr] * 8 + [_ptr, _ptr, _ptr, _ptr, _c_size, _ptr]),
    "vardrop_attn_bwd_dev": (_c_int, [_ptr, _ptr, _ptr, _c_int, _ptr, _c_int, _ptr, _c_int, _c_int, _c_int] + [_ptr] * 4 +
                             [_ptr] + [_ptr] * 9 + [_ptr, _c_size, _ptr]),
    "vardrop_block_norm_workspace_bytes": (_c_size, [_c_int] * 4),
    "vardrop_block_norm_fwd": (_c_int, [_ptr, _ptr, _ptr, _c_int, _c_int, _c_int, _c_int, _c_int] + _BLOCK_NORM_FWD),
    "vardrop_block_norm_fwd_dev": (_c_int, [_ptr, _ptr, _ptr, _c_int, _ptr, _c_int, _ptr, _c_int, _c_int, _c_int] + _BLOCK_NORM_FWD),
    "vardrop_block_norm_bwd": (_c_int, [_ptr] * 6 + [_c_int, _c_int, _c_int, _c_int, _c_int] + _BLOCK_NORM_BWD),
    "vardrop_block_norm_bwd_dev": (_c_int, [_ptr] * 6 + [_c_int, _ptr, _c_int, _ptr, _c_int, _c_int, _c_int] + _BLOCK_NORM_BWD),
    "vardrop_tensor_list_bytes": (_c_size, [_c_int, _ptr]),
    "vardrop_tensor_list_build": (_c_int, [_ptr, _c_int] + [_ptr] * 10 + [_ptr, _c_size, _ptr, _ptr]),
    "vardrop_grad_norm": (_c_int, [_ptr, _ptr, _ptr, _ptr]),
    "vardrop_clip_grads": (_c_int, [_ptr, _ptr, _ptr, _c_float, _ptr, _ptr]),
    "vardrop_adamw": (_c_int, [_ptr, _ptr, _c_double, _c_double, _c_double, _c_double, _c_i64, _ptr, _c_float, _ptr, _ptr]),
    "vardrop_adamw_dev": (_c_int, [_ptr, _ptr, _ptr, _c_double, _c_double, _c_double, _ptr, _c_int, _ptr, _c_float, _ptr, _ptr]),
}


class VarDropError(RuntimeError):
    def __init__(self, code, where, detail=""):
        self.code = code
        super().__init__("%s failed: %s (%d)%s" % (where, _strerror(code), code, detail))


def library_path():
    return os.path.join(_HERE, "libvardrop.so")


def load_library():
    """Loads libvardrop.so (built by paper_2501_14183_amd/build.py) and declares its signatures."""
    global _LIB
    if _LIB is None:
        path = library_path()
        if not os.path.exists(path):
            raise ImportError("libvardrop.so is not built: run `python -m paper_2501_14183_amd.build` "
                              "(there is no fallback implementation)")
        lib = ctypes.CDLL(path)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _LIB = lib
    return _LIB


def _strerror(code):
    return load_library().vardrop_strerror(code).decode()


def _p(t):
    return None if t is None else t.data_ptr()


def _scalar(name, t, dtype, device):
    """Address of a number that the library reads or writes in the memory of `device` (None: not given)."""
    if t is None:
        return None
    if t.dtype is dtype and t.get_device() == device and t.numel() > 0:
        return t.data_ptr()
    raise TypeError("%s must hold a %s on device %d: got %s %s on %s" % (name, dtype, device, t.dtype, list(t.shape), t.device))


# torch's own short cut to the current stream's handle: 0.1 us where the stream object takes 2 us, a third of a short call.
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _device_stream(device, stream=None):
    """Raw hipStream_t: `stream` (an integer handle, e.g. torch.cuda.Stream.cuda_stream) or torch's current one on `device`."""
    if device < 0:
        raise TypeError("the tensors must be on the GPU")
    if stream is not None:
        return stream
    if _current_raw_stream is not None:
        return _current_raw_stream(device)
    return torch.cuda.current_stream(device).cuda_stream


def _stream(t, stream=None):
    """_device_stream of a tensor's device."""
    return stream if stream is not None else _device_stream(t.get_device())


def _own_buffers(stream, what, **bufs):
    """Temporaries come from torch's allocator, which hands freed memory to work on torch's current stream: with a
    raw `stream` handle the caller has to own every buffer the call uses."""
    if stream is not None:
        missing = [k for k, v in bufs.items() if v is None]
        if missing:
            raise TypeError("%s on a raw stream needs caller-owned %s" % (what, ", ".join(missing)))


def _dtype_code(t):
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError("tokens and weights must be float32 or bfloat16")


class Context:
    """Owns a vardrop_ctx on one device."""

    def __init__(self, device=0):
        self._lib = load_library()
        self.device = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
        h = ctypes.c_void_p()
        rc = self._lib.vardrop_create(ctypes.byref(h), self.device.index or 0)
        if rc != 0:
            raise VarDropError(rc, "vardrop_create")
        self.handle = h

    def check(self, rc, where):
        if rc != 0:
            detail = ""
            if rc == -3:
                detail = " hipError=%d" % self._lib.vardrop_last_hip_error(self.handle)
            raise VarDropError(rc, where, detail)

    def close(self):
        if getattr(self, "handle", None):
            self._lib.vardrop_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def vardrop_kernel_name(kid):
    name = load_library().vardrop_kernel_name(kid)
    return None if name is None else name.decode()


def vardrop_profile_select(ctx, kid):
    """Brackets every launch of kernel `kid` with HIP events (-1: off)."""
    ctx.check(ctx._lib.vardrop_profile_select(ctx.handle, kid), "vardrop_profile_select")


def vardrop_profile_stride(ctx, stride):
    """Bracket only every `stride`-th launch of the selected kernel (takes effect at the next select)."""
    ctx.check(ctx._lib.vardrop_profile_stride(ctx.handle, stride), "vardrop_profile_stride")


def vardrop_signal_after(ctx, kid, event):
    """The next launch of kernel `kid` carries `event` (a raw hipEvent_t handle, e.g. torch.cuda.Event.cuda_event of
    an event that has been recorded once; None cancels) as the completion event of its own dispatch."""
    ctx.check(ctx._lib.vardrop_signal_after(ctx.handle, kid, ctypes.c_void_p(event) if event else None), "vardrop_signal_after")


def vardrop_profile_read(ctx):
    """-> (summed duration in ms, number of launches) since the last read or select."""
    ms = ctypes.c_double()
    n = _c_int()
    ctx.check(ctx._lib.vardrop_profile_read(ctx.handle, ctypes.byref(ms), ctypes.byref(n)), "vardrop_profile_read")
    return ms.value, n.value


K_ALL = -2          # vardrop_profile_select: every kernel


def vardrop_profile_read_all(ctx):
    """-> {kernel name: (summed duration in ms, launches)} since the last read or select, for the kernels that ran."""
    n = 0
    while load_library().vardrop_kernel_name(n) is not None:
        n += 1
    ms = (ctypes.c_double * n)()
    cnt = (_c_int * n)()
    ctx.check(ctx._lib.vardrop_profile_read_all(ctx.handle, ms, cnt), "vardrop_profile_read_all")
    return {vardrop_kernel_name(k): (ms[k], cnt[k]) for k in range(n) if cnt[k]}


def vardrop_hash(ctx, x, k, f_min=1, f_max=None, want_abar=False, out=None, stream=None, ws=None):
    """x float32 [B, N, L] (any strides) -> (topk int32 [N, k], hash int64 [N] (the uint64 bits), abar or None).

    out: optional (topk, hash) tensors to write into instead of allocating.
    ws:  optional uint8 workspace for inputs whose time stride is not 1 (allocated when missing)."""
    if x.dtype != torch.float32 or x.dim() != 3:
        raise TypeError("x must be float32 [B, N, L]")
    B, N, L = x.shape
    if f_max is None:
        f_max = ctx._lib.vardrop_hash_default_cutoff(L)      # the paper's default cut-off (the library's rule)
    if out is not None:
        topk, hsh = out
    else:
        topk = torch.empty((N, k), dtype=torch.int32, device=x.device)
        hsh = torch.empty((N,), dtype=torch.int64, device=x.device)
    abar = torch.empty((N, f_max - f_min + 1), dtype=torch.float32, device=x.device) if want_abar else None
    sb, sn, st = x.stride()
    if st != 1:
        _own_buffers(stream, "vardrop_hash of a strided batch", ws=ws)
    if st != 1 and ws is None:
        ws = torch.empty(ctx._lib.vardrop_hash_strided_workspace_bytes(B, N, L), dtype=torch.uint8, device=x.device)
    rc = ctx._lib.vardrop_hash(ctx.handle, _p(x), B, N, L, sb, sn, st, k, f_min, f_max,
                               _p(topk), _p(hsh), _p(abar), _p(ws), 0 if ws is None else ws.numel(),
                               _stream(x, stream))
    ctx.check(rc, "vardrop_hash")
    return topk, hsh, abar


def vardrop_sample(ctx, hsh, gs, ratio_num, ratio_den, seed, step, counts_host=None, out=None, stream=None):
    """hash int64 [N] -> (group_id int32 [N], sel int32 [N] (first N' valid), counts int32 [2] = {N', G}).

    counts_host: optional pinned int32 [2] CPU tensor that receives the counts asynchronously.
    out: optional (group_id, sel, counts) tensors to write into instead of allocating.
    """
    N = hsh.shape[0]
    if out is not None:
        gid, sel, counts = out
    else:
        gid = torch.empty((N,), dtype=torch.int32, device=hsh.device)
        sel = torch.empty((N,), dtype=torch.int32, device=hsh.device)
        counts = torch.empty((2,), dtype=torch.int32, device=hsh.device)
    rc = ctx._lib.vardrop_sample(ctx.handle, _p(hsh), N, gs, ratio_num, ratio_den, seed, step,
                                 _p(gid), _p(sel), _p(counts), _p(counts_host), None, 0, _stream(hsh, stream))
    ctx.check(rc, "vardrop_sample")
    return gid, sel, counts


def vardrop_gather(ctx, tokens, sel, n_sel, out=None, stream=None):
    """tokens [B, N, d], sel int32 -> [B, n_sel, d] (written into `out` when given)."""
    B, N, d = tokens.shape
    if out is None:
        out = torch.empty((B, n_sel, d), dtype=tokens.dtype, device=tokens.device)
    rc = ctx._lib.vardrop_gather(ctx.handle, _p(tokens), B, N, d, _dtype_code(tokens), _p(sel), n_sel, _p(out),
                                 _stream(tokens, stream))
    ctx.check(rc, "vardrop_gather")
    return out


def vardrop_scatter(ctx, dxs, sel, n_sel, N, stream=None):
    """dxs [B, n_sel, d] -> dtokens [B, N, d] with zeros at dropped variates."""
    B, _, d = dxs.shape
    out = torch.empty((B, N, d), dtype=dxs.dtype, device=dxs.device)
    rc = ctx._lib.vardrop_scatter(ctx.handle, _p(dxs), B, N, d, _dtype_code(dxs), _p(sel), n_sel, _p(out),
                                  _stream(dxs, stream))
    ctx.check(rc, "vardrop_scatter")
    return out


def vardrop_attn_fwd(ctx, xs, Wq, Wk, Wv, Wo, H, bq=None, bk=None, bv=None, bo=None, saved=None, out=None, stream=None):
    """xs [B, n, d] -> (y [B, n, d], saved uint8 buffer for the backward); y is written into `out` when given."""
    B, n, d = xs.shape
    code = _dtype_code(xs)
    nbytes = ctx._lib.vardrop_attn_saved_bytes(B, n, d, H, code)
    if saved is None or saved.numel() < nbytes:
        saved = torch.empty((max(nbytes, 256),), dtype=torch.uint8, device=xs.device)
    y = torch.empty_like(xs) if out is None else out
    rc = ctx._lib.vardrop_attn_fwd(ctx.handle, _p(xs), B, n, d, H, code, _p(Wq), _p(Wk), _p(Wv), _p(Wo),
                                   _p(bq), _p(bk), _p(bv), _p(bo), _p(y), _p(saved), None, 0, _stream(xs, stream))
    ctx.check(rc, "vardrop_attn_fwd")
    return y, saved


def vardrop_gather_attn_fwd(ctx, tokens, sel, n_sel, Wq, Wk, Wv, Wo, H, bq=None, bk=None, bv=None, bo=None,
                            saved=None, out=None, stream=None):
    """tokens [B, N, d], sel int32 (first n_sel entries: the kept rows) -> (xs [B, n_sel, d], y [B, n_sel, d], saved):
    the gather and the attention forward in one call.  `out`, when given, is the pair (xs, y) to write into."""
    B, N, d = tokens.shape
    code = _dtype_code(tokens)
    nbytes = ctx._lib.vardrop_attn_saved_bytes(B, n_sel, d, H, code)
    if saved is None or saved.numel() < nbytes:
        saved = torch.empty((max(nbytes, 256),), dtype=torch.uint8, device=tokens.device)
    if out is not None:
        xs, y = out
    else:
        xs = torch.empty((B, n_sel, d), dtype=tokens.dtype, device=tokens.device)
        y = torch.empty_like(xs)
    rc = ctx._lib.vardrop_gather_attn_fwd(ctx.handle, _p(tokens), B, N, _p(sel), n_sel, d, H, code,
                                          _p(Wq), _p(Wk), _p(Wv), _p(Wo), _p(bq), _p(bk), _p(bv), _p(bo),
                                          _p(xs), _p(y), _p(saved), None, 0, _stream(tokens, stream))
    ctx.check(rc, "vardrop_gather_attn_fwd")
    return xs, y, saved


def vardrop_attn_bwd(ctx, dy, xs, Wq, Wk, Wv, Wo, H, saved, bias_grads=False, ws=None, out=None, stream=None):
    """-> (dxs, dWq, dWk, dWv, dWo) or, with bias_grads, (..., dbq, dbk, dbv, dbo); weight grads are float32.
    `out`, when given, is that tuple of preallocated tensors."""
    B, n, d = xs.shape
    code = _dtype_code(xs)
    nbytes = ctx._lib.vardrop_attn_workspace_bytes(B, n, d, H, code)
    _own_buffers(stream, "vardrop_attn_bwd", ws=ws, out=out)
    if ws is None or ws.numel() < nbytes:
        ws = torch.empty((max(nbytes, 256),), dtype=torch.uint8, device=xs.device)
    if out is not None:
        dxs, dW = out[0], list(out[1:5])
        db = list(out[5:9]) if bias_grads else [None] * 4
    else:
        dxs = torch.empty_like(xs)
        dW = [torch.empty((d, d), dtype=torch.float32, device=xs.device) for _ in range(4)]
        db = [torch.empty((d,), dtype=torch.float32, device=xs.device) if bias_grads else None for _ in range(4)]
    rc = ctx._lib.vardrop_attn_bwd(ctx.handle, _p(dy), _p(xs), B, n, d, H, code, _p(Wq), _p(Wk), _p(Wv), _p(Wo),
                                   _p(saved), _p(dxs), *[_p(t) for t in dW], *[_p(t) for t in db],
                                   _p(ws), ws.numel(), _stream(xs, stream))
    ctx.check(rc, "vardrop_attn_bwd")
    return (dxs, *dW, *db) if bias_grads else (dxs, *dW)


def vardrop_embed_fwd(ctx, x, sel, n_sel, We, be=None, standardise=True, saved=None, out=None, stream=None):
    """x float32 [B, N, L] (time contiguous), sel int32, We [L, d] -> (xs [B, n_sel, d] in We's dtype, saved)."""
    if x.dtype != torch.float32 or x.dim() != 3 or x.stride(2) != 1:
        raise TypeError("x must be float32 [B, N, L] with contiguous time")
    B, N, L = x.shape
    d = We.shape[1]
    dt = _dtype_code(We)
    if saved is None:
        saved = torch.empty(ctx._lib.vardrop_embed_saved_bytes(B, n_sel, L, dt), dtype=torch.uint8, device=x.device)
    xs = out if out is not None else torch.empty((B, n_sel, d), dtype=We.dtype, device=x.device)
    rc = ctx._lib.vardrop_embed_fwd(ctx.handle, _p(x), B, N, L, x.stride(0), x.stride(1), _p(sel), n_sel,
                                    1 if standardise else 0, _p(We), _p(be), d, dt, _p(xs), _p(saved),
                                    _stream(x, stream))
    ctx.check(rc, "vardrop_embed_fwd")
    return xs, saved


def vardrop_embed_bwd(ctx, dxs, L, saved, want_bias=True, ws=None, out=None, stream=None):
    """dxs [B, n_sel, d], saved from vardrop_embed_fwd -> (dWe float32 [L, d], dbe float32 [d] or None).
    `out`, when given, is that pair of preallocated tensors."""
    B, n_sel, d = dxs.shape
    dt = _dtype_code(dxs)
    _own_buffers(stream, "vardrop_embed_bwd", ws=ws, out=out)
    if ws is None:
        ws = torch.empty(max(ctx._lib.vardrop_embed_workspace_bytes(B, n_sel, L, d, dt), 256), dtype=torch.uint8,
                         device=dxs.device)
    if out is not None:
        dWe, dbe = out
    else:
        dWe = torch.empty((L, d), dtype=torch.float32, device=dxs.device)
        dbe = torch.empty((d,), dtype=torch.float32, device=dxs.device) if want_bias else None
    rc = ctx._lib.vardrop_embed_bwd(ctx.handle, _p(dxs), B, n_sel, L, d, dt, _p(saved), _p(dWe), _p(dbe),
                                    _p(ws), ws.numel(), _stream(dxs, stream))
    ctx.check(rc, "vardrop_embed_bwd")
    return dWe, dbe


def vardrop_sample_nearest(ctx, hsh, abar, gs, ratio_num, ratio_den, stream=None):
    """hash int64 [N], abar float32 [N, F] -> (group_id int32 [N], sel int32 [N] (first N' valid), counts int32 [2]):
    every group keeps the members closest to its mean spectrum."""
    N, F = abar.shape
    dev = hsh.device
    if stream is not None:
        raise TypeError("vardrop_sample_nearest allocates its workspace: call it on torch's current stream")
    gid = torch.empty((N,), dtype=torch.int32, device=dev)
    sel = torch.empty((N,), dtype=torch.int32, device=dev)
    counts = torch.empty((2,), dtype=torch.int32, device=dev)
    ws = torch.empty(max(ctx._lib.vardrop_sample_nearest_workspace_bytes(N, F), 256), dtype=torch.uint8, device=dev)
    rc = ctx._lib.vardrop_sample_nearest(ctx.handle, _p(hsh), _p(abar), N, F, gs, ratio_num, ratio_den,
                                         _p(gid), _p(sel), _p(counts), None, _p(ws), ws.numel(), _stream(hsh, stream))
    ctx.check(rc, "vardrop_sample_nearest")
    return gid, sel, counts



# ---------------------------------------------------------------- device-side token count
def _count(t, n_dev, status):
    """Device of the tensor t, and the addresses of the count and of the status word there."""
    device = t.get_device()
    return device, _scalar("n_dev", n_dev, torch.int32, device), _scalar("status", status, torch.int32, device)


def vardrop_sample_dev(ctx, hsh, gs, ratio_num, ratio_den, seed, step_dev, advance, out, stream=None):
    """vardrop_sample with the step counter in device memory (step_dev: int64 [1]); out = (group_id, sel, counts)."""
    N = hsh.shape[0]
    gid, sel, counts = out
    device = hsh.get_device()
    rc = ctx._lib.vardrop_sample_dev(ctx.handle, _p(hsh), N, gs, ratio_num, ratio_den, seed,
                                     _scalar("step_dev", step_dev, torch.int64, device), 1 if advance else 0,
                                     _p(gid), _p(sel), _p(counts), None, 0, _device_stream(device, stream))
    ctx.check(rc, "vardrop_sample_dev")
    return gid, sel, counts


def vardrop_gather_dev(ctx, tokens, sel, n_dev, n_max, out, status=None, stream=None):
    """tokens [B, N, d], sel int32, n_dev int32 [1] on the device -> out (>= B * n_max * d elements), packed [B, N', d]."""
    B, N, d = tokens.shape
    device, p_n, p_status = _count(tokens, n_dev, status)
    rc = ctx._lib.vardrop_gather_dev(ctx.handle, _p(tokens), B, N, d, _dtype_code(tokens), _p(sel), p_n, n_max,
                                     p_status, _p(out), _device_stream(device, stream))
    ctx.check(rc, "vardrop_gather_dev")
    return out


def vardrop_scatter_dev(ctx, dxs, sel, n_dev, n_max, out, status=None, stream=None):
    """dxs packed [B, N', d] -> out [B, N, d] with zeros at dropped variates; N' read from n_dev on the device."""
    B, N, d = out.shape
    device, p_n, p_status = _count(out, n_dev, status)
    rc = ctx._lib.vardrop_scatter_dev(ctx.handle, _p(dxs), B, N, d, _dtype_code(out), _p(sel), p_n, n_max,
                                      p_status, _p(out), _device_stream(device, stream))
    ctx.check(rc, "vardrop_scatter_dev")
    return out


def vardrop_gather_attn_fwd_dev(ctx, tokens, sel, n_dev, n_max, Wq, Wk, Wv, Wo, H, xs, y, saved,
                                bq=None, bk=None, bv=None, bo=None, status=None, stream=None):
    """Gather + attention forward with N' read on the device from n_dev (int32 [1]); xs, y hold >= B * n_max * d
    elements and receive [B, N', d] packed; saved holds vardrop_attn_saved_bytes(B, n_max, d, H) bytes."""
    B, N, d = tokens.shape
    device, p_n, p_status = _count(tokens, n_dev, status)
    rc = ctx._lib.vardrop_gather_attn_fwd_dev(ctx.handle, _p(tokens), B, N, _p(sel), p_n, n_max, p_status, d, H,
                                              _dtype_code(tokens), _p(Wq), _p(Wk), _p(Wv), _p(Wo),
                                              _p(bq), _p(bk), _p(bv), _p(bo), _p(xs), _p(y), _p(saved), None, 0,
                                              _device_stream(device, stream))
    ctx.check(rc, "vardrop_gather_attn_fwd_dev")
    return xs, y, saved


def vardrop_attn_bwd_dev(ctx, dy, xs, n_dev, n_max, Wq, Wk, Wv, Wo, H, saved, ws, out, status=None, stream=None):
    """Attention backward with N' read on the device; out = (dxs, dWq, dWk, dWv, dWo[, dbq, dbk, dbv, dbo]);
    B is taken from the weights' caller: dy, xs, dxs are flat or [B, n_max, d] buffers, so B = out[0].shape[0]."""
    B = out[0].shape[0]
    d = Wq.shape[0]
    dxs, dW = out[0], list(out[1:5])
    db = list(out[5:9]) if len(out) >= 9 else [None] * 4
    device, p_n, p_status = _count(Wq, n_dev, status)
    rc = ctx._lib.vardrop_attn_bwd_dev(ctx.handle, _p(dy), _p(xs), B, p_n, n_max, p_status, d, H, _dtype_code(Wq),
                                       _p(Wq), _p(Wk), _p(Wv), _p(Wo), _p(saved), _p(dxs), *[_p(t) for t in dW],
                                       *[_p(t) for t in db], _p(ws), ws.numel(), _device_stream(device, stream))
    ctx.check(rc, "vardrop_attn_bwd_dev")
    return out


def vardrop_sample_nearest_noalloc(ctx, hsh, abar, gs, ratio_num, ratio_den, out, stream=None):
    """vardrop_sample_nearest on the library's static scratch (allocates nothing); out = (group_id, sel, counts)."""
    N, F = abar.shape
    gid, sel, counts = out
    rc = ctx._lib.vardrop_sample_nearest_noalloc(ctx.handle, _p(hsh), _p(abar), N, F, gs, ratio_num, ratio_den,
                                                 _p(gid), _p(sel), _p(counts), _stream(hsh, stream))
    ctx.check(rc, "vardrop_sample_nearest_noalloc")
    return gid, sel, counts


def vardrop_attn_fwd_dev(ctx, xs, n_dev, n_max, Wq, Wk, Wv, Wo, H, y, saved, bq=None, bk=None, bv=None, bo=None,
                         status=None, stream=None):
    """Attention forward on packed tokens xs ([B, n_max, d] buffer holding [B, N', d]) with N' read on the device."""
    B, d = xs.shape[0], Wq.shape[0]
    device, p_n, p_status = _count(xs, n_dev, status)
    rc = ctx._lib.vardrop_attn_fwd_dev(ctx.handle, _p(xs), B, p_n, n_max, p_status, d, H, _dtype_code(Wq),
                                       _p(Wq), _p(Wk), _p(Wv), _p(Wo), _p(bq), _p(bk), _p(bv), _p(bo),
                                       _p(y), _p(saved), None, 0, _device_stream(device, stream))
    ctx.check(rc, "vardrop_attn_fwd_dev")
    return y, saved


def vardrop_embed_fwd_dev(ctx, x, sel, n_dev, n_max, We, be, xs, saved, standardise=True, status=None, stream=None):
    """Embedding of the kept windows with their count read on the device; xs: [B, n_max, d] buffer, packed [B, N', d]."""
    B, N, L = x.shape
    device, p_n, p_status = _count(x, n_dev, status)
    rc = ctx._lib.vardrop_embed_fwd_dev(ctx.handle, _p(x), B, N, L, x.stride(0), x.stride(1), _p(sel), p_n, n_max,
                                        p_status, 1 if standardise else 0, _p(We), _p(be), We.shape[1], _dtype_code(We),
                                        _p(xs), _p(saved), _device_stream(device, stream))
    ctx.check(rc, "vardrop_embed_fwd_dev")
    return xs, saved


def vardrop_embed_bwd_dev(ctx, dxs, n_dev, n_max, L, saved, ws, out, stream=None):
    """Weight gradients of the embedding with the count read on the device; out = (dWe, dbe or None)."""
    B, d = dxs.shape[0], dxs.shape[-1]
    dWe, dbe = out
    device, p_n, _ = _count(dxs, n_dev, None)
    rc = ctx._lib.vardrop_embed_bwd_dev(ctx.handle, _p(dxs), B, p_n, n_max, L, d, _dtype_code(dxs), _p(saved),
                                        _p(dWe), _p(dbe), _p(ws), ws.numel(), _device_stream(device, stream))
    ctx.check(rc, "vardrop_embed_bwd_dev")
    return dWe, dbe


# ---------------------------------------------------------------- norms before and after a block
# These calls are made twice a block and take a few microseconds on the GPU, less than a call of a checking function for every
# tensor costs: the checks stand in line (host time of a call with everything given, beside the library's own: forward 3.4 us, backward
# 5.1; a call for every tensor had added 1.4 and 2.0).
_CODES = {torch.float32: F32, torch.bfloat16: BF16}


def _refuse(name, t, numel, dtype):
    raise TypeError("%s must be contiguous, %s, of %d elements, on the device of the call's first tensor: got %s %s on %s"
                    % (name, dtype, numel, t.dtype, list(t.shape), t.device))


def _block_type(res, *others):
    """Element type of a block's tensors (the first one given, results included), that of the residual stream where there is none."""
    for t in others:
        if t is not None:
            return t.dtype
    return res.dtype


def _gate_rows(gate, B, d):
    k = gate.numel()
    if gate.shape[-1] != d or (k != d and k != B * d):
        raise TypeError("gate must be [d], [1, d] or [B, d]")
    return 1 if k == d else B


def vardrop_block_norm_workspace_bytes(B, n, d, gates):
    """Bytes of the workspace of vardrop_block_norm_bwd; gates: rows of the gate (0 = none)."""
    return max(load_library().vardrop_block_norm_workspace_bytes(B, n, d, gates), 256)


def vardrop_block_norm_fwd(ctx, x, f=None, pre=NORM_LAYER, w=None, b=None, post=NORM_NONE, wp=None, bp=None, gate=None,
                           alpha=1.0, beta=1.0, eps=1e-5, want_r=True, want_stats=True, out=None, stream=None,
                           n_dev=None, status=None):
    """r = alpha x + beta gate * post(f), h = pre(r): x [B, n, d] the residual stream, f the block's output (None: none).

    -> (r, h, stats): r in x's type, h in the block's, stats float32 [B*n, 4] for the backward.  `out`, when given, is that
    triple of preallocated tensors; entries that are None are not written (h is None exactly when pre is NORM_NONE).
    n_dev (int32 [1] on the device): the tensors are buffers for x.shape[1] tokens that hold [B, N', d] packed."""
    B, n, d = x.shape
    res, fp32 = x.dtype, torch.float32
    r, h, stats = (None, None, None) if out is None else out
    dt = f.dtype if f is not None else _block_type(x, h, w, b, wp, bp, gate)
    if out is None:
        _own_buffers(stream, "vardrop_block_norm_fwd", out=out)
        r = torch.empty_like(x) if want_r or pre == NORM_NONE else None
        h = torch.empty((B, n, d), dtype=dt, device=x.device) if pre != NORM_NONE else None
        stats = torch.empty((B * n, 4), dtype=torch.float32, device=x.device) if want_stats else None
    dev = x.get_device()                       # and all others on the same
    rows = B * n
    k = rows * d
    gates = 0 if gate is None else _gate_rows(gate, B, d)
    p_x = x.data_ptr() if x.dtype is res and x.numel() == k and x.is_contiguous() else _refuse("x", x, k, res)
    p_f = None if f is None else (f.data_ptr() if f.dtype is dt and f.numel() == k and f.is_contiguous() and f.get_device() == dev
                                  else _refuse("f", f, k, dt))
    p_r = None if r is None else (r.data_ptr() if r.dtype is res and r.numel() == k and r.is_contiguous() and r.get_device() == dev
                                  else _refuse("r", r, k, res))
    p_h = None if h is None else (h.data_ptr() if h.dtype is dt and h.numel() == k and h.is_contiguous() and h.get_device() == dev
                                  else _refuse("h", h, k, dt))
    p_w = None if w is None else (w.data_ptr() if w.dtype is dt and w.numel() == d and w.is_contiguous() and w.get_device() == dev
                                  else _refuse("w", w, d, dt))
    p_b = None if b is None else (b.data_ptr() if b.dtype is dt and b.numel() == d and b.is_contiguous() and b.get_device() == dev
                                  else _refuse("b", b, d, dt))
    p_wp = None if wp is None else (wp.data_ptr() if wp.dtype is dt and wp.numel() == d and wp.is_contiguous()
                                    and wp.get_device() == dev else _refuse("wp", wp, d, dt))
    p_bp = None if bp is None else (bp.data_ptr() if bp.dtype is dt and bp.numel() == d and bp.is_contiguous()
                                    and bp.get_device() == dev else _refuse("bp", bp, d, dt))
    p_gate = None if gate is None else (gate.data_ptr() if gate.dtype is dt and gate.numel() == gates * d and gate.is_contiguous()
                                        and gate.get_device() == dev else _refuse("gate", gate, gates * d, dt))
    p_stats = None if stats is None else (stats.data_ptr() if stats.dtype is fp32 and stats.numel() == 4 * rows and stats.is_contiguous()
                                          and stats.get_device() == dev else _refuse("stats", stats, 4 * rows, fp32))
    on = _device_stream(dev, stream)
    if n_dev is None:
        rc = ctx._lib.vardrop_block_norm_fwd(ctx.handle, p_x, p_f, B, n, d, _CODES.get(res, -1), _CODES.get(dt, -1), post, p_wp, p_bp, p_gate,
                                             gates, alpha, beta, pre, p_w, p_b, eps, p_r, p_h, p_stats, on)
    else:
        rc = ctx._lib.vardrop_block_norm_fwd_dev(ctx.handle, p_x, p_f, B, _scalar("n_dev", n_dev, torch.int32, dev), n,
                                                 _scalar("status", status, torch.int32, dev), d, _CODES.get(res, -1), _CODES.get(dt, -1), post,
                                                 p_wp, p_bp, p_gate, gates, alpha, beta, pre, p_w, p_b, eps, p_r, p_h, p_stats, on)
    if rc:
        ctx.check(rc, "vardrop_block_norm_fwd")
    return r, h, stats


def vardrop_block_norm_bwd(ctx, dr, dh, r, f, stats, pre=NORM_LAYER, w=None, post=NORM_NONE, wp=None, bp=None, gate=None,
                           alpha=1.0, beta=1.0, bias_grads=False, ws=None, out=None, stream=None, n_dev=None, status=None):
    """Gradients of vardrop_block_norm_fwd from dr and dh, those of r and h (dr may be None; dh is None exactly when pre
    is NORM_NONE); r, f, stats as the forward had them.

    -> (dx, df, dw, db, dwp, dbp, dgate): dx in the residual's type, df in the block's, the rest float32.  Without `out`, df is
    made when f is given, the vectors' gradients for the vectors given (db, dbp with bias_grads).  `out`, when given, is that
    tuple of preallocated tensors; entries that are None are skipped."""
    like = dr if dr is not None else r
    if like is None:
        raise TypeError("one of dr and r has to be given")
    B, n, d = like.shape
    res, fp32 = like.dtype, torch.float32
    dx, df, dw, db, dwp, dbp, dgate = (None,) * 7 if out is None else out
    dt = dh.dtype if dh is not None else _block_type(like, f, df, w, wp, bp, gate)
    if out is None:
        _own_buffers(stream, "vardrop_block_norm_bwd", out=out)

        def vector(wanted, *shape):
            return torch.empty(shape, dtype=fp32, device=like.device) if wanted else None

        dx = torch.empty_like(like)
        df = None if f is None else torch.empty_like(f)
        dw, db = vector(w is not None, d), vector(bias_grads and pre != NORM_NONE, d)
        dwp, dbp = vector(wp is not None, d), vector(bias_grads and post != NORM_NONE, d)
        dgate = None if gate is None else vector(True, *gate.shape)
    dev = like.get_device()                    # and all others on the same
    rows = B * n
    k = rows * d
    gates = 0 if gate is None else _gate_rows(gate, B, d)
    p_dr = None if dr is None else (dr.data_ptr() if dr.dtype is res and dr.numel() == k and dr.is_contiguous()
                                    else _refuse("dr", dr, k, res))
    p_dh = None if dh is None else (dh.data_ptr() if dh.dtype is dt and dh.numel() == k and dh.is_contiguous()
                                    and dh.get_device() == dev else _refuse("dh", dh, k, dt))
    p_r = None if r is None else (r.data_ptr() if r.dtype is res and r.numel() == k and r.is_contiguous() and r.get_device() == dev
                                  else _refuse("r", r, k, res))
    p_f = None if f is None else (f.data_ptr() if f.dtype is dt and f.numel() == k and f.is_contiguous() and f.get_device() == dev
                                  else _refuse("f", f, k, dt))
    p_dx = None if dx is None else (dx.data_ptr() if dx.dtype is res and dx.numel() == k and dx.is_contiguous()
                                    and dx.get_device() == dev else _refuse("dx", dx, k, res))
    p_df = None if df is None else (df.data_ptr() if df.dtype is dt and df.numel() == k and df.is_contiguous()
                                    and df.get_device() == dev else _refuse("df", df, k, dt))
    p_w = None if w is None else (w.data_ptr() if w.dtype is dt and w.numel() == d and w.is_contiguous() and w.get_device() == dev
                                  else _refuse("w", w, d, dt))
    p_wp = None if wp is None else (wp.data_ptr() if wp.dtype is dt and wp.numel() == d and wp.is_contiguous()
                                    and wp.get_device() == dev else _refuse("wp", wp, d, dt))
    p_bp = None if bp is None else (bp.data_ptr() if bp.dtype is dt and bp.numel() == d and bp.is_contiguous()
                                    and bp.get_device() == dev else _refuse("bp", bp, d, dt))
    p_gate = None if gate is None else (gate.data_ptr() if gate.dtype is dt and gate.numel() == gates * d and gate.is_contiguous()
                                        and gate.get_device() == dev else _refuse("gate", gate, gates * d, dt))
    p_stats = None if stats is None else (stats.data_ptr() if stats.dtype is fp32 and stats.numel() == 4 * rows and stats.is_contiguous()
                                          and stats.get_device() == dev else _refuse("stats", stats, 4 * rows, fp32))
    p_dw = None if dw is None else (dw.data_ptr() if dw.dtype is fp32 and dw.numel() == d and dw.is_contiguous()
                                    and dw.get_device() == dev else _refuse("dw", dw, d, fp32))
    p_db = None if db is None else (db.data_ptr() if db.dtype is fp32 and db.numel() == d and db.is_contiguous()
                                    and db.get_device() == dev else _refuse("db", db, d, fp32))
    p_dwp = None if dwp is None else (dwp.data_ptr() if dwp.dtype is fp32 and dwp.numel() == d and dwp.is_contiguous()
                                      and dwp.get_device() == dev else _refuse("dwp", dwp, d, fp32))
    p_dbp = None if dbp is None else (dbp.data_ptr() if dbp.dtype is fp32 and dbp.numel() == d and dbp.is_contiguous()
                                      and dbp.get_device() == dev else _refuse("dbp", dbp, d, fp32))
    p_dgate = None if dgate is None else (dgate.data_ptr() if dgate.dtype is fp32 and dgate.numel() == gates * d and dgate.is_contiguous()
                                          and dgate.get_device() == dev else _refuse("dgate", dgate, gates * d, fp32))
    if ws is None and (dw is not None or db is not None or dwp is not None or dbp is not None or dgate is not None):
        _own_buffers(stream, "vardrop_block_norm_bwd", ws=ws)
        ws = torch.empty(vardrop_block_norm_workspace_bytes(B, n, d, gates), dtype=torch.uint8, device=like.device)
    if ws is not None and not (ws.is_contiguous() and ws.get_device() == dev):
        raise TypeError("ws must be contiguous, on device %d" % dev)
    p_ws, room, on = _p(ws), 0 if ws is None else ws.numel(), _device_stream(dev, stream)
    if n_dev is None:
        rc = ctx._lib.vardrop_block_norm_bwd(ctx.handle, p_dr, p_dh, p_r, p_f, p_stats, B, n, d, _CODES.get(res, -1), _CODES.get(dt, -1), post,
                                             p_wp, p_bp, p_gate, gates, alpha, beta, pre, p_w, p_dx, p_df, p_dw, p_db, p_dwp, p_dbp, p_dgate,
                                             p_ws, room, on)
    else:
        rc = ctx._lib.vardrop_block_norm_bwd_dev(ctx.handle, p_dr, p_dh, p_r, p_f, p_stats, B, _scalar("n_dev", n_dev, torch.int32, dev), n,
                                                 _scalar("status", status, torch.int32, dev), d, _CODES.get(res, -1), _CODES.get(dt, -1), post,
                                                 p_wp, p_bp, p_gate, gates, alpha, beta, pre, p_w, p_dx, p_df, p_dw, p_db, p_dwp, p_dbp, p_dgate,
                                                 p_ws, room, on)
    if rc:
        ctx.check(rc, "vardrop_block_norm_bwd")
    return dx, df, dw, db, dwp, dbp, dgate


# ---------------------------------------------------------------- tensor lists: gradient norm, clipping, AdamW
class _TensorListStruct(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("table_bytes", ctypes.c_size_t), ("numel", ctypes.c_int64),
                ("tensors", ctypes.c_int32), ("chunks", ctypes.c_int32), ("has", ctypes.c_uint32), ("built", ctypes.c_uint32)]


class TensorList:
    """A vardrop_tensor_list with its table and the tensors it names, which it keeps alive.

    grads: float32 or bfloat16 tensors on one device, contiguous; clipped: where vardrop_clip_grads writes (None: in place);
    params, exp_avg, exp_avg_sq: float32, for vardrop_adamw; weights: bfloat16 copies of the weights, entries may be None;
    decay: weight decay of each tensor.  Building it enqueues work on torch's current stream and costs the host 1.5 us for each
    tensor and more: it is made once and used every step, so the tensors have to stay where they are."""

    def __init__(self, ctx, grads, clipped=None, params=None, exp_avg=None, exp_avg_sq=None, weights=None, decay=None):
        grads = list(grads)
        count = len(grads)
        numel = [t.numel() for t in grads]
        device = ctx.device.index or 0
        room = max(count, 1)

        def addresses(what, tensors, dtypes, may_miss=False):
            """The list of tensors and a C array of their addresses."""
            if tensors is None:
                return None, None
            tensors = list(tensors)
            if len(tensors) != count:
                raise TypeError("%s: %d tensors for %d gradients" % (what, len(tensors), count))
            for t, k in zip(tensors, numel):
                if t is None and may_miss:
                    continue
                if t is None or t.numel() != k or t.dtype not in dtypes or not t.is_contiguous() or t.get_device() != device:
                    raise TypeError("%s: contiguous tensors of the gradients' sizes on %s wanted, in %s"
                                    % (what, ctx.device, " or ".join(str(d) for d in dtypes)))
            return tensors, (ctypes.c_void_p * room)(*[None if t is None else t.data_ptr() for t in tensors])

        both, fp32 = (torch.float32, torch.bfloat16), (torch.float32,)

        def codes(tensors):
            """C array of the element types; None where all are float32, which the library takes for that."""
            if tensors is None or all(t.dtype is torch.float32 for t in tensors):
                return None
            return (ctypes.c_int32 * room)(*[_CODES[t.dtype] for t in tensors])

        grads, g = addresses("grads", grads, both)
        clipped, c = addresses("clipped", clipped, both)
        params, p = addresses("params", params, fp32)
        exp_avg, m = addresses("exp_avg", exp_avg, fp32)
        exp_avg_sq, v = addresses("exp_avg_sq", exp_avg_sq, fp32)
        weights, w = addresses("weights", weights, (torch.bfloat16,), may_miss=True)
        if decay is not None and len(decay) != count:
            raise TypeError("decay: %d values for %d gradients" % (len(decay), count))
        rates = None if decay is None else (ctypes.c_float * room)(*decay)
        sizes = (ctypes.c_int64 * room)(*numel)
        self.tensors = (grads, clipped, params, exp_avg, exp_avg_sq, weights)
        self.device = device
        nbytes = ctx._lib.vardrop_tensor_list_bytes(count, sizes)
        if nbytes == 0:
            raise VarDropError(-1, "vardrop_tensor_list_bytes")
        self.table = torch.empty(nbytes, dtype=torch.uint8, device=ctx.device)
        self.struct = _TensorListStruct()
        self.pointer = ctypes.addressof(self.struct)
        rc = ctx._lib.vardrop_tensor_list_build(ctx.handle, count, sizes, g, codes(grads), c, codes(clipped), p, m, v, w, rates,
                                                self.table.data_ptr(), nbytes, self.pointer, _stream(self.table, None))
        ctx.check(rc, "vardrop_tensor_list_build")


def _clip_norm(max_norm, where):
    """max_norm, 0 for no clipping, as the library gets it: one that only rounds to 0 is none."""
    if 0.0 < max_norm <= 2.0 ** -150:
        raise VarDropError(-1, where)
    return max_norm


def vardrop_grad_norm(ctx, tensors, out=None, stream=None):
    """Global norm of a TensorList's gradients -> float32 [1] on the device (`out` when given)."""
    if out is None:
        _own_buffers(stream, "vardrop_grad_norm", out=out)
        out = torch.empty(1, dtype=torch.float32, device=ctx.device)
    rc = ctx._lib.vardrop_grad_norm(ctx.handle, tensors.pointer, _scalar("out", out, torch.float32, tensors.device),
                                    _device_stream(tensors.device, stream))
    if rc:
        ctx.check(rc, "vardrop_grad_norm")
    return out


def vardrop_clip_grads(ctx, tensors, norm, max_norm, status=None, stream=None):
    """Gradients times min(1, max_norm / (norm + 1e-6)) into the list's `clipped` tensors (in place without them)."""
    rc = ctx._lib.vardrop_clip_grads(ctx.handle, tensors.pointer, _scalar("norm", norm, torch.float32, tensors.device), max_norm,
                                     _scalar("status", status, torch.int32, tensors.device), _device_stream(tensors.device, stream))
    if rc:
        ctx.check(rc, "vardrop_clip_grads")


def vardrop_adamw(ctx, tensors, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, norm=None, max_norm=0.0, status=None, stream=None):
    """AdamW step number `step` (from 1) of a TensorList with params; with `norm` and max_norm the gradients are clipped in it."""
    rc = ctx._lib.vardrop_adamw(ctx.handle, tensors.pointer, lr, beta1, beta2, eps, step, _scalar("norm", norm, torch.float32, tensors.device),
                                _clip_norm(max_norm, "vardrop_adamw"), _scalar("status", status, torch.int32, tensors.device),
                                _device_stream(tensors.device, stream))
    if rc:
        ctx.check(rc, "vardrop_adamw")


def vardrop_adamw_dev(ctx, tensors, lr_dev, step_dev, beta1=0.9, beta2=0.999, eps=1e-8, norm=None, max_norm=0.0, advance=True,
                      status=None, stream=None):
    """vardrop_adamw with the rate (float32 [1]) and the number of steps done (int64 [1], advanced) in device memory."""
    rc = ctx._lib.vardrop_adamw_dev(ctx.handle, tensors.pointer, _scalar("lr_dev", lr_dev, torch.float32, tensors.device), beta1, beta2, eps,
                                    _scalar("step_dev", step_dev, torch.int64, tensors.device), 1 if advance else 0,
                                    _scalar("norm", norm, torch.float32, tensors.device), _clip_norm(max_norm, "vardrop_adamw_dev"),
                                    _scalar("status", status, torch.int32, tensors.device), _device_stream(tensors.device, stream))
    if rc:
        ctx.check(rc, "vardrop_adamw_dev")
