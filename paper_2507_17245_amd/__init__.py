"""Python binding of libdistr_attn.so (DistrAttention forward for MI355X / gfx950).

Argument marshalling only: every step of the path runs in the library's HIP kernels.
Tensors are torch tensors on the GPU (torch provides device memory and streams, nothing
else); names mirror the C entry points declared in include/distr_attn.h. There is no
fallback: a missing library or a failing call raises.
"""
import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdistr_attn.so")

DA_OK, DA_ERR_INVALID_ARG, DA_ERR_UNSUPPORTED, DA_ERR_WORKSPACE, DA_ERR_HIP = 0, -1, -2, -3, -4
DA_BF16, DA_F32 = 0, 1

EXPORTS = (
    "distr_attn_fwd", "distr_attn_exact_fwd", "distr_attn_fwd_ex", "distr_attn_exact_fwd_ex",
    "distr_attn_fwd_noalloc", "distr_attn_noalloc_max_bytes",
    "distr_attn_bwd_ex", "distr_attn_exact_bwd_ex",
    "distr_attn_lsh_group", "distr_attn_key_prepass", "distr_attn_kt_bytes",
    "distr_attn_workspace_bytes", "distr_attn_bwd_workspace_bytes", "distr_attn_hyperplanes",
    "distr_attn_qk_norm_rope", "distr_attn_qk_norm_rope_bwd", "distr_attn_qk_bwd_workspace_bytes",
    "distr_attn_cache_append", "distr_attn_paged_fwd", "distr_attn_paged_workspace_bytes",
    "distr_attn_cache4_append", "distr_attn_cache4_read", "distr_attn_paged4_fwd", "distr_attn_paged4_workspace_bytes",
    "distr_attn_set_stream", "distr_attn_release", "distr_attn_last_error", "distr_attn_version",
)


class DaParams(ctypes.Structure):
    """Mirror of da_params."""
    _fields_ = [
        ("B", ctypes.c_int), ("H", ctypes.c_int), ("Hkv", ctypes.c_int), ("N", ctypes.c_int),
        ("d", ctypes.c_int), ("Br", ctypes.c_int), ("Bc", ctypes.c_int), ("n_groups", ctypes.c_int),
        ("causal", ctypes.c_int), ("lsh_seed", ctypes.c_uint64), ("dtype", ctypes.c_int),
        ("n_planes", ctypes.c_int), ("softmax_scale", ctypes.c_float), ("gray_mode", ctypes.c_int),
        ("stream", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_size_t), ("perm_out", ctypes.c_void_p),
        ("hash_out", ctypes.c_void_p), ("perm_in", ctypes.c_void_p), ("kt_in", ctypes.c_void_p),
        ("Nk", ctypes.c_int), ("side", ctypes.c_int), ("lse_out", ctypes.c_void_p),
    ]


class DaRotary(ctypes.Structure):
    """Mirror of da_rotary."""
    _fields_ = [
        ("norm", ctypes.c_int), ("eps", ctypes.c_float), ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p),
        ("weight_dtype", ctypes.c_int), ("weight_heads", ctypes.c_int), ("rope", ctypes.c_int), ("rot_dim", ctypes.c_int),
        ("n_pos", ctypes.c_int), ("cos_table", ctypes.c_void_p), ("sin_table", ctypes.c_void_p),
    ]


class DaQk(ctypes.Structure):
    """Mirror of da_qk."""
    _fields_ = [
        ("B", ctypes.c_int), ("H", ctypes.c_int), ("Hkv", ctypes.c_int), ("N", ctypes.c_int), ("d", ctypes.c_int),
        ("dtype", ctypes.c_int), ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3),
        ("q_out_stride", ctypes.c_int64 * 3), ("k_out_stride", ctypes.c_int64 * 3), ("rotary", DaRotary),
        ("positions", ctypes.c_void_p), ("stream", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_size_t),
    ]


class DaPaged(ctypes.Structure):
    """Mirror of da_paged."""
    _fields_ = [
        ("H", ctypes.c_int), ("Hkv", ctypes.c_int), ("d", ctypes.c_int), ("dtype", ctypes.c_int),
        ("n_seq", ctypes.c_int), ("n_tokens", ctypes.c_int), ("n_pages", ctypes.c_int), ("page_size", ctypes.c_int),
        ("max_pages", ctypes.c_int), ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
        ("row_stride", ctypes.c_int64), ("page_table", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
        ("q_start", ctypes.c_void_p), ("q_stride", ctypes.c_int64 * 2), ("k_stride", ctypes.c_int64 * 2),
        ("v_stride", ctypes.c_int64 * 2), ("rotary", DaRotary), ("positions", ctypes.c_void_p), ("causal", ctypes.c_int),
        ("softmax_scale", ctypes.c_float), ("lse_out", ctypes.c_void_p), ("stream", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
    ]


class DaCache4(ctypes.Structure):
    """Mirror of da_cache4."""
    _fields_ = [
        ("k_codes", ctypes.c_void_p), ("k_scales", ctypes.c_void_p), ("v_codes", ctypes.c_void_p), ("v_scales", ctypes.c_void_p),
        ("code_stride", ctypes.c_int64 * 3), ("scale_stride", ctypes.c_int64 * 3),
    ]


class DistrAttnError(RuntimeError):
    def __init__(self, code, message):
        super().__init__(f"distr_attn error {code}: {message}")
        self.code = code


_lib = None


def lib():
    """The loaded C library. Raises if it has not been built (python -m paper_2507_17245_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with `python paper_2507_17245_amd/build.py`")
        L = ctypes.CDLL(LIB_PATH)
        vp, ci, u64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_uint64
        L.distr_attn_fwd.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, ci, u64, ci]
        L.distr_attn_exact_fwd.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, ci]
        L.distr_attn_noalloc_max_bytes.restype = ctypes.c_size_t
        for name in ("distr_attn_fwd_ex", "distr_attn_exact_fwd_ex", "distr_attn_fwd_noalloc"):
            getattr(L, name).argtypes = [vp, vp, vp, vp, ctypes.POINTER(DaParams)]
        for name in ("distr_attn_bwd_ex", "distr_attn_exact_bwd_ex"):
            getattr(L, name).argtypes = [vp] * 9 + [ctypes.POINTER(DaParams)]
        L.distr_attn_lsh_group.argtypes = [vp, ctypes.POINTER(DaParams)]
        L.distr_attn_key_prepass.argtypes = [vp, vp, ctypes.POINTER(DaParams)]
        for name in ("distr_attn_workspace_bytes", "distr_attn_bwd_workspace_bytes", "distr_attn_kt_bytes"):
            getattr(L, name).argtypes = [ctypes.POINTER(DaParams)]
            getattr(L, name).restype = ctypes.c_size_t
        L.distr_attn_qk_norm_rope.argtypes = [vp] * 4 + [ctypes.POINTER(DaQk)]
        L.distr_attn_qk_norm_rope_bwd.argtypes = [vp] * 8 + [ctypes.POINTER(DaQk)]
        for name in ("distr_attn_cache_append", "distr_attn_paged_fwd"):
            getattr(L, name).argtypes = [vp] * 4 + [ctypes.POINTER(DaPaged)]
        for name in ("distr_attn_cache4_append", "distr_attn_cache4_read", "distr_attn_paged4_fwd"):
            getattr(L, name).argtypes = [vp, vp, ctypes.POINTER(DaCache4), ctypes.POINTER(DaPaged)]
        for name, params in (("distr_attn_qk_bwd_workspace_bytes", DaQk), ("distr_attn_paged_workspace_bytes", DaPaged),
                             ("distr_attn_paged4_workspace_bytes", DaPaged)):
            getattr(L, name).argtypes = [ctypes.POINTER(params)]
            getattr(L, name).restype = ctypes.c_size_t
        L.distr_attn_hyperplanes.argtypes = [u64, ci, ci, ctypes.POINTER(ctypes.c_float)]
        L.distr_attn_set_stream.argtypes = [vp]
        L.distr_attn_last_error.restype = ctypes.c_char_p
        L.distr_attn_version.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _check(rc):
    if rc != DA_OK:
        raise DistrAttnError(rc, lib().distr_attn_last_error().decode())


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def _current_stream():
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dtype_code(t):
    import torch
    if t.dtype == torch.bfloat16:
        return DA_BF16
    if t.dtype == torch.float32:
        return DA_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _shapes(q, k, v):
    if q.dim() != 4 or k.dim() != 4 or tuple(v.shape) != tuple(k.shape):
        raise ValueError("q must be [B,H,N,d]; k, v must be [B,Hkv,Nk,d]")
    B, H, N, d = q.shape
    if k.shape[0] != B or k.shape[3] != d:
        raise ValueError("k, v do not match q")
    for t in (q, k, v):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("tensors must be contiguous and on the GPU")
    if not (q.dtype == k.dtype == v.dtype):
        raise TypeError("q, k, v must share a dtype")
    return B, H, k.shape[1], N, d


def _check_out(q, o):
    """o is written by the kernels with q's shape and element type: anything else would be
    written out of bounds on the device."""
    if tuple(o.shape) != tuple(q.shape) or o.dtype != q.dtype:
        raise ValueError("o must have the shape and dtype of q")
    if not o.is_cuda or not o.is_contiguous():
        raise ValueError("o must be contiguous and on the GPU")


def _check_buffer(t, name, min_bytes):
    """An optional device buffer the library reads or writes `min_bytes` of."""
    if t is None:
        return
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous and on the GPU")
    have = t.numel() * t.element_size()
    if have < min_bytes:
        raise ValueError(f"{name} holds {have} bytes, {min_bytes} needed")


def make_params(q, k, v, Br, Bc=64, n_groups=None, causal=False, lsh_seed=0, n_planes=0,
                softmax_scale=0.0, gray_mode=0, workspace=None, perm_out=None, hash_out=None,
                perm_in=None, kt_in=None, side=0, lse_out=None):
    """side=1: the mirrored form (sample K, fuse Q, one grouping per K block of Bc rows); the
    tables are then [B, Hkv, ceil(Nk/Bc), d]. Nk is taken from k's shape. lse_out: float32
    [B, H, N] that receives the rows' log-sum-exp (what a backward pass needs)."""
    B, H, Hkv, N, d = _shapes(q, k, v)
    Nk = k.shape[2]
    p = DaParams()
    p.B, p.H, p.Hkv, p.N, p.d, p.Br, p.Bc = B, H, Hkv, N, d, Br, Bc
    p.Nk = Nk
    p.side = side
    p.n_groups = d if n_groups is None else n_groups
    p.causal = int(bool(causal))
    p.lsh_seed = lsh_seed
    p.dtype = _dtype_code(q)
    p.n_planes = n_planes
    p.softmax_scale = softmax_scale
    p.gray_mode = gray_mode
    p.stream = _current_stream().value
    if side == 1:
        n_table = B * Hkv * ((Nk + Bc - 1) // Bc) * d if Bc > 0 else 0
    else:
        n_table = B * H * ((N + Br - 1) // Br) * d if Br > 0 else 0
    _check_buffer(workspace, "workspace", 0)
    _check_buffer(perm_out, "perm_out", n_table)
    _check_buffer(hash_out, "hash_out", 4 * n_table)
    _check_buffer(perm_in, "perm_in", n_table)
    if workspace is not None:
        p.workspace = workspace.data_ptr()
        p.workspace_bytes = workspace.numel() * workspace.element_size()
    p.perm_out = perm_out.data_ptr() if perm_out is not None else None
    p.hash_out = hash_out.data_ptr() if hash_out is not None else None
    p.perm_in = perm_in.data_ptr() if perm_in is not None else None
    p.kt_in = kt_in.data_ptr() if kt_in is not None else None
    if kt_in is not None:
        _check_buffer(kt_in, "kt_in", distr_attn_kt_bytes(p))
    if lse_out is not None:
        import torch
        if lse_out.dtype != torch.float32:
            raise TypeError("lse_out must be float32")
        _check_buffer(lse_out, "lse_out", 4 * B * H * N)
        p.lse_out = lse_out.data_ptr()
    return p


def distr_attn_fwd(q, k, v, o, Br, Bc, n_groups, lsh_seed=0, causal=False):
    """Short form: bf16, 16 projections, scale 1/sqrt(d), on torch's current stream."""
    B, H, Hkv, N, d = _shapes(q, k, v)
    if _dtype_code(q) != DA_BF16:
        raise TypeError("the short form takes bf16 tensors; use distr_attn_fwd_ex for float")
    _check_out(q, o)
    lib().distr_attn_set_stream(_current_stream())
    if k.shape[2] != N:
        raise ValueError("the short form takes N keys; use distr_attn_fwd_ex for Nk != N")
    _check(lib().distr_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), B, H, Hkv, N, d, Br, Bc,
                                n_groups, lsh_seed, int(bool(causal))))
    return o


def distr_attn_exact_fwd(q, k, v, o, Br, Bc, causal=False):
    B, H, Hkv, N, d = _shapes(q, k, v)
    if _dtype_code(q) != DA_BF16:
        raise TypeError("the short form takes bf16 tensors; use distr_attn_exact_fwd_ex for float")
    _check_out(q, o)
    lib().distr_attn_set_stream(_current_stream())
    if k.shape[2] != N:
        raise ValueError("the short form takes N keys; use distr_attn_exact_fwd_ex for Nk != N")
    _check(lib().distr_attn_exact_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), B, H, Hkv, N, d, Br, Bc,
                                      int(bool(causal))))
    return o


def _check_ex(q, k, v, o, params):
    B, H, Hkv, N, d = _shapes(q, k, v)
    _check_out(q, o)
    if (params.B, params.H, params.Hkv, params.N, params.d, params.dtype, params.Nk or N) != \
            (B, H, Hkv, N, d, _dtype_code(q), k.shape[2]):
        raise ValueError("params were made for tensors of another shape or dtype")


def distr_attn_fwd_ex(q, k, v, o, params):
    _check_ex(q, k, v, o, params)
    _check(lib().distr_attn_fwd_ex(_ptr(q), _ptr(k), _ptr(v), _ptr(o), ctypes.byref(params)))
    return o


def distr_attn_fwd_noalloc(q, k, v, o, params):
    """distr_attn_fwd_ex on the library's fixed scratch array: allocates nothing."""
    _check_ex(q, k, v, o, params)
    _check(lib().distr_attn_fwd_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(o), ctypes.byref(params)))
    return o


def distr_attn_noalloc_max_bytes():
    return int(lib().distr_attn_noalloc_max_bytes())


def distr_attn_exact_fwd_ex(q, k, v, o, params):
    _check_ex(q, k, v, o, params)
    _check(lib().distr_attn_exact_fwd_ex(_ptr(q), _ptr(k), _ptr(v), _ptr(o), ctypes.byref(params)))
    return o


def _bwd(name, q, k, v, o, dout, lse, dq, dk, dv, params):
    import torch
    _check_ex(q, k, v, o, params)
    _check_out(q, dout)
    _check_out(q, dq)
    _check_out(k, dk)
    _check_out(k, dv)
    if lse.dtype != torch.float32:
        raise TypeError("lse must be float32")
    _check_buffer(lse, "lse", 4 * params.B * params.H * params.N)
    _check(getattr(lib(), name)(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(dout), _ptr(lse), _ptr(dq), _ptr(dk),
                                _ptr(dv), ctypes.byref(params)))
    return dq, dk, dv


def distr_attn_bwd_ex(q, k, v, o, dout, lse, dq, dk, dv, params):
    """Backward of distr_attn_fwd_ex (bf16 tensors: matrix-core kernels; float tensors: float
    arithmetic): fills dq, dk, dv. o and lse are the forward's output and lse_out."""
    return _bwd("distr_attn_bwd_ex", q, k, v, o, dout, lse, dq, dk, dv, params)


def distr_attn_exact_bwd_ex(q, k, v, o, dout, lse, dq, dk, dv, params):
    return _bwd("distr_attn_exact_bwd_ex", q, k, v, o, dout, lse, dq, dk, dv, params)


def distr_attn_lsh_group(q, params):
    _check(lib().distr_attn_lsh_group(_ptr(q), ctypes.byref(params)))


def distr_attn_key_prepass(k, kt_out, params):
    if not k.is_cuda or not k.is_contiguous():
        raise ValueError("k must be contiguous and on the GPU")
    _check_buffer(kt_out, "kt_out", distr_attn_kt_bytes(params))
    _check(lib().distr_attn_key_prepass(_ptr(k), _ptr(kt_out), ctypes.byref(params)))
    return kt_out


def distr_attn_kt_bytes(params):
    return int(lib().distr_attn_kt_bytes(ctypes.byref(params)))


def distr_attn_workspace_bytes(params):
    return int(lib().distr_attn_workspace_bytes(ctypes.byref(params)))


def distr_attn_bwd_workspace_bytes(params):
    return int(lib().distr_attn_bwd_workspace_bytes(ctypes.byref(params)))


def distr_attn_hyperplanes(seed, n_planes, Br):
    """-> numpy float32 [n_planes, Br] (host): the projection matrix the kernels generate."""
    import numpy as np
    out = np.empty((n_planes, Br), dtype=np.float32)
    _check(lib().distr_attn_hyperplanes(seed, n_planes, Br,
                                        out.ctypes.data_as(ctypes.POINTER(ctypes.c_float))))
    return out


def distr_attn_release():
    _check(lib().distr_attn_release())


def distr_attn_version():
    return lib().distr_attn_version().decode()


# ---- around attention: norms and rotation of queries and keys, a cache in pages --------------------------

ROPE = {"none": 0, "halves": 1, "neighbours": 2}
NULL_STREAM = 1   # hipStreamLegacy: the null stream itself, not what a short form or a program has set for calls without one


def _at(t):
    return None if t is None else t.data_ptr()


def _strides(t, what):
    """Strides of all dimensions but the last, which has to be contiguous; those of a single entry do not matter."""
    if t.stride(-1) != 1:
        raise ValueError(f"the channels of {what} must be contiguous")
    return [s if n > 1 else 0 for n, s in zip(t.shape[:-1], t.stride()[:-1])]


def _layout(t):
    return (t.shape, t.stride(), t.dtype, t.device)


def _check_layout(t, like, what):
    if _layout(t) != like:
        raise ValueError(f"params were made for a {what} of another shape, stride, dtype or device")


def _check_device(device, *tensors):
    """All on `device`, the current one (whose stream the call takes)."""
    import torch
    if device.type != "cuda":
        raise ValueError("tensors must be on the GPU")
    if device.index != torch.cuda.current_device():
        raise ValueError(f"tensors are on {device}, the current device is cuda:{torch.cuda.current_device()}")
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError("tensors must be on one device")


def _check_index(t, shape, what):
    import torch
    if t.dtype != torch.int32 or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous int32 of shape {tuple(shape)}")


def _fill_rotary(r, d, heads, norm, eps, weights, rope, cos, sin):
    """weights: (of the queries, of the keys), for `heads` of them."""
    import torch
    if rope not in ROPE:
        raise ValueError(f"rope must be one of {sorted(ROPE)}")
    r.norm, r.eps = int(bool(norm)), eps
    given = [(w, h, n) for w, h, n in zip(weights, heads, ("q_weight", "k_weight")) if w is not None]
    if given and not norm:
        raise ValueError("weights without norm")
    if len({(w.dtype, w.dim()) for w, _, _ in given}) > 1:
        raise ValueError("q_weight and k_weight must share dtype and form")
    for w, h, name in given:
        if tuple(w.shape) not in ((d,), (h, d)) or not w.is_contiguous():
            raise ValueError(f"{name} must be contiguous, [{d}] or [{h}, {d}]")
        r.weight_dtype, r.weight_heads = _dtype_code(w), int(w.dim() == 2)
    r.q_weight, r.k_weight = (w.data_ptr() if w is not None else None for w in weights)
    r.rope = ROPE[rope]
    if r.rope:
        for t, name in ((cos, "cos"), (sin, "sin")):
            if t is None or t.dim() != 2 or t.dtype != torch.float32 or not t.is_contiguous() or t.shape != cos.shape:
                raise ValueError(f"{name} must be contiguous float32 [positions, rotated channels / 2]")
        r.n_pos, r.rot_dim = cos.shape[0], 2 * cos.shape[1]
        r.cos_table, r.sin_table = cos.data_ptr(), sin.data_ptr()


def _fill_workspace(p, workspace, device):
    _check_buffer(workspace, "workspace", 0)
    if workspace is not None:
        p.workspace, p.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    p.stream = _current_stream().value or NULL_STREAM
    import torch
    p.device, p.current_device = device.index, torch.cuda.current_device


def make_qk_params(q, k, q_out, k_out, norm=False, eps=1e-6, q_weight=None, k_weight=None, rope="none", cos=None, sin=None,
                   positions=None, workspace=None):
    """Parameters of distr_attn_qk_norm_rope and its backward for tensors of these layouts: q, q_out [B, H, N, d], k, k_out
    [B, Hkv, N, d] (None: queries alone), any strides with contiguous channels (views of one projection, [B, N, heads, d]
    transposed, outputs in place). norm: RMS norm of each row with eps and the weights ([d], or [heads, d]; None: ones). rope: "none",
    "halves" (pairs of channels j and j + rotated / 2) or "neighbours" (2 j and 2 j + 1), cos and sin float32
    [positions, rotated channels / 2]; positions int32 [B, N], None: 0 .. N - 1 in every batch. workspace: scratch of the
    backward's weight gradients (None: the library's)."""
    if q.dim() != 4 or q_out.shape != q.shape:
        raise ValueError("q and q_out must be [B, H, N, d]")
    if (k is None) != (k_out is None):
        raise ValueError("k and k_out go together")
    B, H, N, d = q.shape
    if k is not None and (k.dim() != 4 or k_out.shape != k.shape or (k.shape[0], k.shape[2], k.shape[3]) != (B, N, d)):
        raise ValueError("k and k_out must be [B, Hkv, N, d]")
    if any(t is not None and t.dtype != q.dtype for t in (q_out, k, k_out)):
        raise TypeError("q, k, q_out, k_out must share a dtype")
    _check_device(q.device, q_out, k, k_out, q_weight, k_weight, cos, sin, positions, workspace)
    p = DaQk()
    p.B, p.H, p.Hkv, p.N, p.d, p.dtype = B, H, 0 if k is None else k.shape[1], N, d, _dtype_code(q)
    p.q_stride[:], p.q_out_stride[:] = _strides(q, "q"), _strides(q_out, "q_out")
    if k is not None:
        p.k_stride[:], p.k_out_stride[:] = _strides(k, "k"), _strides(k_out, "k_out")
    _fill_rotary(p.rotary, d, (H, p.Hkv), norm, eps, (q_weight, k_weight), rope, cos, sin)
    if positions is not None:
        _check_index(positions, (B, N), "positions")
        p.positions = positions.data_ptr()
    _fill_workspace(p, workspace, q.device)
    p.layouts = {"q": _layout(q), "q_out": _layout(q_out), "k": k if k is None else _layout(k), "k_out": k if k is None else _layout(k_out)}
    p.weights = {"q": q_weight, "k": k_weight}
    p.held = (cos, sin, positions, workspace)
    return p


def _run(name, params, *args):
    """The call, on the stream and the device that params were made for."""
    if params.current_device() != params.device:
        raise ValueError(f"params were made for cuda:{params.device}, the current device is cuda:{params.current_device()}")
    _check(getattr(_lib or lib(), name)(*args, ctypes.byref(params)))


def _check_qk(params, tensors):
    for t, name in tensors:
        if params.layouts[name] is None or t is None:
            if params.layouts[name] is not t:
                raise ValueError("params were made with keys, or without")
            continue
        _check_layout(t, params.layouts[name], name)


def distr_attn_qk_norm_rope(q, k, q_out, k_out, params):
    """q_out, k_out = rotation(norm(q)), rotation(norm(k)), in one launch. -> (q_out, k_out)"""
    _check_qk(params, ((q, "q"), (k, "k"), (q_out, "q_out"), (k_out, "k_out")))
    _run("distr_attn_qk_norm_rope", params, _at(q), _at(k), _at(q_out), _at(k_out))
    return q_out, k_out


def distr_attn_qk_norm_rope_bwd(q, k, dq_out, dk_out, dq, dk, params, dq_weight=None, dk_weight=None):
    """Gradient of distr_attn_qk_norm_rope: dq, dk (laid out like q, k) from dq_out, dk_out (like q_out, k_out) and the forward's
    inputs; dq_weight, dk_weight float32 in the weights' shapes ([d] where there is none), or None. -> (dq, dk)"""
    _check_qk(params, ((q, "q"), (k, "k"), (dq_out, "q_out"), (dk_out, "k_out"), (dq, "q"), (dk, "k")))
    for t, of in ((dq_weight, "q"), (dk_weight, "k")):
        if t is None:
            continue
        if of == "k" and params.Hkv == 0:
            raise ValueError("dk_weight without keys")
        w = params.weights[of]
        shape = (params.H if of == "q" else params.Hkv, params.d) if params.rotary.weight_heads else (params.d,)
        if _dtype_code(t) != DA_F32 or tuple(t.shape) != (tuple(w.shape) if w is not None else shape) or not t.is_contiguous() or t.device != dq.device:
            raise ValueError(f"d{of}_weight must be contiguous float32 of the weight's shape")
    _run("distr_attn_qk_norm_rope_bwd", params, _at(q), _at(k), _at(dq_out), _at(dk_out), _at(dq), _at(dk), _at(dq_weight), _at(dk_weight))
    return dq, dk


def distr_attn_qk_bwd_workspace_bytes(params):
    return int(lib().distr_attn_qk_bwd_workspace_bytes(ctypes.byref(params)))


def make_paged_params(k_pages, v_pages, page_table, kv_len, q_start, q=None, k=None, v=None, causal=True, softmax_scale=0.0,
                      lse_out=None, norm=False, eps=1e-6, k_weight=None, rope="none", cos=None, sin=None, positions=None, workspace=None):
    """Parameters of distr_attn_cache_append (k, v given) and distr_attn_paged_fwd (q given) for a batch of sequences in one
    cache. k_pages, v_pages: [pages, Hkv, page size, d], any strides with contiguous channels (a transposed view where
    the tokens lie outside the heads). page_table int32 [sequences, pages of the longest], kv_len int32 [sequences]: tokens with the new
    ones, q_start int32 [sequences + 1]: the new tokens of sequence s are rows q_start[s] .. q_start[s + 1] - 1 of q
    [tokens, H, d] and of k, v [tokens, Hkv, d]. The three are read on the device by each call: a program writes
    the next step's into them and calls again. norm, rope and the rest: of the keys on their way into the cache, as in make_qk_params (positions
    int32 [tokens]; None: a token's place in its sequence). lse_out: float32 [tokens, H]. workspace: of
    distr_attn_paged_workspace_bytes, which a captured call needs for the keys of a row to be dealt out to several workgroups."""
    if k_pages.dim() != 4 or k_pages.shape != v_pages.shape or _strides(k_pages, "k_pages") != _strides(v_pages, "v_pages"):
        raise ValueError("k_pages and v_pages must be [pages, Hkv, page size, d] of the same strides")
    if any(t is not None and t.dtype != k_pages.dtype for t in (v_pages, q, k, v)):
        raise TypeError("q, k, v and the pages must share a dtype")
    p = _paged_params(k_pages.shape, (k_pages, v_pages), page_table, kv_len, q_start, q, k, v, causal, softmax_scale, lse_out, norm, eps, k_weight,
                      rope, cos, sin, positions, workspace)
    p.page_stride, p.head_stride, p.row_stride = _strides(k_pages, "k_pages")
    p.layouts["pages"] = _layout(k_pages)
    return p


def _paged_params(shape, cache, page_table, kv_len, q_start, q, k, v, causal, softmax_scale, lse_out, norm, eps, k_weight, rope, cos, sin, positions,
                  workspace):
    """What calls over pages of `shape` [pages, Hkv, page size, d] share: all but the pages' strides. cache: its tensors."""
    import torch
    n_pages, Hkv, page_size, d = shape
    new = [t for t in (q, k, v) if t is not None]
    if not new or (k is None) != (v is None):
        raise ValueError("q, or k and v, must be given")
    if any(t.dim() != 3 or t.shape[2] != d or t.shape[0] != new[0].shape[0] for t in new) or any(t.shape[1] != Hkv for t in (k, v) if t is not None):
        raise ValueError("q must be [tokens, H, d]; k, v [tokens, Hkv, d]")
    if any(t.dtype != new[0].dtype for t in new):
        raise TypeError("q, k, v must share a dtype")
    if page_table.dim() != 2 or kv_len.dim() != 1:
        raise ValueError("page_table must be [sequences, pages], kv_len [sequences]")
    _check_device(cache[0].device, *cache[1:], page_table, kv_len, q_start, *new, lse_out, k_weight, cos, sin, positions, workspace)
    n_seq, n_tokens = kv_len.shape[0], new[0].shape[0]
    _check_index(page_table, (n_seq, page_table.shape[1]), "page_table")
    _check_index(kv_len, (n_seq,), "kv_len")
    _check_index(q_start, (n_seq + 1,), "q_start")
    p = DaPaged()
    p.H, p.Hkv, p.d, p.dtype = q.shape[1] if q is not None else Hkv, Hkv, d, _dtype_code(new[0])
    p.n_seq, p.n_tokens = n_seq, n_tokens
    p.n_pages, p.page_size, p.max_pages = n_pages, page_size, page_table.shape[1]
    p.page_table, p.kv_len, p.q_start = page_table.data_ptr(), kv_len.data_ptr(), q_start.data_ptr()
    for t, field in ((q, p.q_stride), (k, p.k_stride), (v, p.v_stride)):
        if t is not None:
            field[:] = _strides(t, "q, k, v")
    _fill_rotary(p.rotary, d, (p.H, Hkv), norm, eps, (None, k_weight), rope, cos, sin)
    if positions is not None:
        _check_index(positions, (n_tokens,), "positions")
        p.positions = positions.data_ptr()
    p.causal, p.softmax_scale = int(bool(causal)), softmax_scale
    if lse_out is not None:
        if lse_out.dtype != torch.float32 or q is None or tuple(lse_out.shape) != tuple(q.shape[:2]) or not lse_out.is_contiguous():
            raise ValueError("lse_out must be contiguous float32 [tokens, H]")
        p.lse_out = lse_out.data_ptr()
    _fill_workspace(p, workspace, cache[0].device)
    p.layouts = {"q": q if q is None else _layout(q), "k": k if k is None else _layout(k), "v": v if v is None else _layout(v)}
    p.held = (page_table, kv_len, q_start, lse_out, k_weight, cos, sin, positions, workspace)
    return p


def _check_pages(k_pages, v_pages, params):
    like = params.layouts.get("pages")   # (none: made for a cache in 4 bits)
    if _layout(k_pages) != like or _layout(v_pages) != like:
        raise ValueError("params were made for pages of another shape, stride, dtype or device")


def distr_attn_cache_append(k, v, k_pages, v_pages, params):
    """The new tokens' keys (normed and rotated on the way if params say so) and values into the cache. -> (k_pages, v_pages)"""
    if params.layouts["k"] is None:
        raise ValueError("params were made without k and v")
    _check_layout(k, params.layouts["k"], "k")
    _check_layout(v, params.layouts["v"], "v")
    _check_pages(k_pages, v_pages, params)
    _run("distr_attn_cache_append", params, _at(k), _at(v), _at(k_pages), _at(v_pages))
    return k_pages, v_pages


def distr_attn_paged_fwd(q, k_pages, v_pages, o, params):
    """Exact attention of the new tokens over the cache, their own keys in it: o [tokens, H, d], contiguous."""
    if params.layouts["q"] is None:
        raise ValueError("params were made without q")
    _check_layout(q, params.layouts["q"], "q")
    if o.shape != q.shape or o.dtype != q.dtype or o.device != q.device or not o.is_contiguous():
        raise ValueError("o must be contiguous, of q's shape and dtype, on its device")
    _check_pages(k_pages, v_pages, params)
    _run("distr_attn_paged_fwd", params, _at(q), _at(k_pages), _at(v_pages), _at(o))
    return o


def distr_attn_paged_workspace_bytes(params):
    return int(lib().distr_attn_paged_workspace_bytes(ctypes.byref(params)))


def make_paged4_params(cache, page_table, kv_len, q_start, q=None, k=None, v=None, causal=True, softmax_scale=0.0, lse_out=None, norm=False,
                       eps=1e-6, k_weight=None, rope="none", cos=None, sin=None, positions=None, workspace=None):
    """Parameters of distr_attn_cache4_append and distr_attn_cache4_read (k, v given) and distr_attn_paged4_fwd (q given) for a batch of
    sequences in one cache held in 4 bits: cache = (k_codes, k_scales, v_codes, v_scales), uint8, codes [pages, Hkv, page size, d / 2] with channel
    2 j in the low bits of byte j, scales [pages, Hkv, page size, d / 32]: 2^(byte - 127) for 32 channels. Any strides with contiguous
    rows, the same for keys and values. page_table: no wider than the batch can need, its width decides how the attention is dealt out. The rest as in make_paged_params; workspace of distr_attn_paged4_workspace_bytes."""
    import torch
    k_codes, k_scales, v_codes, v_scales = cache
    for a, b, what in ((k_codes, v_codes, "codes"), (k_scales, v_scales, "scales")):
        if a.dim() != 4 or a.shape != b.shape or _strides(a, what) != _strides(b, what):
            raise ValueError(f"{what} of keys and values must be [pages, Hkv, page size, channels] of the same strides")
        if a.dtype != torch.uint8 or b.dtype != torch.uint8:
            raise TypeError(f"{what} must be uint8")
    d = 2 * k_codes.shape[3]
    if d % 32 != 0 or k_scales.shape != (*k_codes.shape[:3], d // 32):
        raise ValueError("scales must be [pages, Hkv, page size, d / 32]")
    p = _paged_params((*k_codes.shape[:3], d), cache, page_table, kv_len, q_start, q, k, v, causal, softmax_scale, lse_out, norm, eps, k_weight,
                      rope, cos, sin, positions, workspace)
    p.layouts["cache"] = _cache_layout(*cache)
    p.strides = tuple((ctypes.c_int64 * 3)(*_strides(t, what)) for t, what in ((k_codes, "codes"), (k_scales, "scales")))
    return p


def _cache_layout(a, b, c, d):
    """As _layout, of the four tensors at once (a call is 0.7 us shorter than by one after the other)."""
    return (a.shape, a.stride(), a.dtype, a.device, b.shape, b.stride(), b.dtype, b.device,
            c.shape, c.stride(), c.dtype, c.device, d.shape, d.stride(), d.dtype, d.device)


def _cache4(cache, params):
    """The cache as the library takes it: its tensors are those of the call, the layout is that of params."""
    k_codes, k_scales, v_codes, v_scales = cache
    if _cache_layout(k_codes, k_scales, v_codes, v_scales) != params.layouts.get("cache"):   # (none: made for pages of keys and values)
        raise ValueError("params were made for a cache of another shape, stride or device")
    return DaCache4(k_codes.data_ptr(), k_scales.data_ptr(), v_codes.data_ptr(), v_scales.data_ptr(), *params.strides)


def _run_cache4(name, params, k, v, cache):
    if params.layouts["k"] is None:
        raise ValueError("params were made without k and v")
    _check_layout(k, params.layouts["k"], "k")
    _check_layout(v, params.layouts["v"], "v")
    _run(name, params, _at(k), _at(v), ctypes.byref(_cache4(cache, params)))


def distr_attn_cache4_append(k, v, cache, params):
    """The new tokens' keys (normed and rotated on the way if params say so) and values into the cache, in 4 bits. -> cache"""
    _run_cache4("distr_attn_cache4_append", params, k, v, cache)
    return cache


def distr_attn_cache4_read(k, v, cache, params):
    """What the cache holds of the sequences' last tokens, q_start[s + 1] - q_start[s] of sequence s, into k and v [tokens, Hkv, d]. -> (k, v)"""
    _run_cache4("distr_attn_cache4_read", params, k, v, cache)
    return k, v


def distr_attn_paged4_fwd(q, cache, o, params):
    """Exact attention of the new tokens over the cache, their own keys in it: o [tokens, H, d], contiguous."""
    if params.layouts["q"] is None:
        raise ValueError("params were made without q")
    _check_layout(q, params.layouts["q"], "q")
    if o.shape != q.shape or o.dtype != q.dtype or o.device != q.device or not o.is_contiguous():
        raise ValueError("o must be contiguous, of q's shape and dtype, on its device")
    _run("distr_attn_paged4_fwd", params, _at(q), _at(o), ctypes.byref(_cache4(cache, params)))
    return o


def distr_attn_paged4_workspace_bytes(params):
    return int(lib().distr_attn_paged4_workspace_bytes(ctypes.byref(params)))
