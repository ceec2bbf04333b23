"""ctypes binding with the same names as the C entry points (argument marshalling only)."""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Tuple

HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_NAME = "libdynamicrad.so"

MODE_STATIC, MODE_DYNAMIC, MODE_ZSCORE, MODE_UNIFORM = 0, 1, 2, 3
CLASS_NONE, CLASS_NEAR, CLASS_FAR, CLASS_FORCED = 0, 1, 2, 3
ROPE_HALF, ROPE_INTERLEAVED = 0, 1
_STATUS = {0: "DR_OK", 1: "DR_ERR_INVALID_ARG", 2: "DR_ERR_UNSUPPORTED", 3: "DR_ERR_CAPACITY", 4: "DR_ERR_HIP",
           5: "DR_ERR_NOMEM"}


class DRError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"{_STATUS.get(status, status)}: {text}")
        self.status = status
        self.status_name = _STATUS.get(status, str(status))


class Shape(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("N", C.c_int32), ("d", C.c_int32),
                ("Nf", C.c_int32), ("Hg", C.c_int32), ("Wg", C.c_int32), ("Bs", C.c_int32),
                ("dtype", C.c_int32), ("reserved0", C.c_int32),
                ("stride_b", C.c_int64), ("stride_h", C.c_int64), ("stride_n", C.c_int64)]

    @property
    def Sb(self) -> int:
        return -(-self.N // self.Bs)


class MaskParams(C.Structure):
    _fields_ = [("gamma", C.c_double), ("theta_c", C.c_double), ("theta_m", C.c_double),
                ("ratio_far", C.c_double), ("head_fuse", C.c_int32), ("has_tau_far", C.c_int32),
                ("tau_far", C.c_double), ("seed", C.c_uint32), ("reserved", C.c_int32 * 3)]

    def __init__(self, gamma=1.0, theta_c=0.15, theta_m=0.60, ratio_far=-1.0, head_fuse=2, tau_far=None, seed=0):
        super().__init__(gamma, theta_c, theta_m, ratio_far, head_fuse, 0 if tau_far is None else 1,
                         0.0 if tau_far is None else tau_far, seed)


class RopeParams(C.Structure):
    """Rotary positions of the first `dim` channels; `axis_pairs`: pairs of each position axis (one axis by default)."""
    _fields_ = [("theta", C.c_double), ("factor", C.c_double), ("original_len", C.c_double), ("ramp_low", C.c_double),
                ("ramp_high", C.c_double), ("mscale", C.c_double), ("dim", C.c_int32), ("layout", C.c_int32), ("axes", C.c_int32),
                ("axis_pairs", C.c_int32 * 3), ("reserved", C.c_int32 * 2)]

    def __init__(self, dim, layout=ROPE_HALF, axis_pairs=None, theta=10000.0, factor=1.0, original_len=0.0, ramp_low=1.0, ramp_high=32.0,
                 mscale=1.0):
        pairs = [dim // 2] if axis_pairs is None else [int(n) for n in axis_pairs]
        super().__init__(theta, factor, original_len, ramp_low, ramp_high, mscale, dim, layout, len(pairs),
                         (C.c_int32 * 3)(*(pairs + [0, 0, 0])[:3]))


class RopeShape(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("N", C.c_int32), ("d", C.c_int32), ("dtype", C.c_int32), ("reserved0", C.c_int32),
                ("stride_b", C.c_int64), ("stride_h", C.c_int64), ("stride_n", C.c_int64), ("out_stride_b", C.c_int64),
                ("out_stride_h", C.c_int64), ("out_stride_n", C.c_int64)]


class _Cache(C.Structure):
    _fields_ = [("pages", C.c_int32), ("heads", C.c_int32), ("page_tokens", C.c_int32), ("d", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p),
                ("k_scale", C.c_void_p), ("v_scale", C.c_void_p)]


class _Batch(C.Structure):
    _fields_ = [("sequences", C.c_int32), ("tokens", C.c_int32), ("max_pages", C.c_int32), ("reserved0", C.c_int32), ("cu", C.c_void_p),
                ("lens", C.c_void_p), ("page_table", C.c_void_p), ("table_stride", C.c_int64)]


class _TokenStrides(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("reserved0", C.c_int32), ("a_stride_t", C.c_int64), ("a_stride_h", C.c_int64), ("b_stride_t", C.c_int64),
                ("b_stride_h", C.c_int64)]


def lib_path() -> str:
    return os.path.join(HERE, _LIB_NAME)


_lib = None


def load_library():
    """Load the built library; raises with the build command if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise ImportError(f"{path} is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
                          "(or `python paper_2604_20470_amd/build.py`) first; there is no CPU fallback")
    lib = C.CDLL(path)
    vp, i32, i64, f64 = C.c_void_p, C.c_int32, C.c_int64, C.c_double
    shp, mpp = C.POINTER(Shape), C.POINTER(MaskParams)
    lib.dr_version.restype = C.c_char_p
    lib.dr_create.argtypes = [C.POINTER(vp), C.c_int]
    lib.dr_destroy.argtypes = [vp]
    lib.dr_destroy.restype = None
    lib.dr_last_error.argtypes = [vp]
    lib.dr_last_error.restype = C.c_char_p
    lib.dr_class_map.argtypes = [vp, shp, f64, mpp, vp, vp]
    lib.dr_mask_capacity.argtypes = [vp, shp, f64, mpp, C.POINTER(i64), C.POINTER(i32)]
    lib.dr_static_ratio_for_sparsity.argtypes = [vp, shp, f64, mpp, f64, C.POINTER(f64), C.POINTER(f64)]
    lib.dr_block_scores.argtypes = [vp, shp, vp, vp, i32, vp, vp]
    lib.dr_build_mask.argtypes = [vp, shp, i32, f64, f64, mpp, vp, vp, vp, i64, vp, vp]
    lib.dr_sparse_attn_fwd.argtypes = [vp, shp, vp, vp, vp, vp, vp, i32, i64, vp, vp, vp]
    lib.dr_sparse_attn_fwd_static.argtypes = [vp, shp, vp, vp, vp, vp, vp, i32, i64, vp, vp, vp]
    lib.dr_token_scores.argtypes = [vp, shp, vp, vp, i32, vp, vp]
    lib.dr_build_mask_tokens.argtypes = [vp, shp, f64, f64, mpp, vp, vp, vp, i64, vp, vp, vp]
    lib.dr_proxy_loss.argtypes = [vp, vp, vp, i32, i32, i32, vp, i32, i32, f64, f64, vp, vp]
    lib.dr_proxy_objective.argtypes = [vp, shp, vp, vp, vp, vp, i32, i64, vp, f64, f64, vp, vp]
    rsp, rpp, cap, bap, tsp = C.POINTER(RopeShape), C.POINTER(RopeParams), C.POINTER(_Cache), C.POINTER(_Batch), C.POINTER(_TokenStrides)
    lib.dr_rope_fwd.argtypes = [vp, rsp, rpp, vp, vp, i64, i64, vp, vp]
    lib.dr_rope_bwd.argtypes = [vp, rsp, rpp, vp, vp, i64, i64, vp, vp]
    lib.dr_cache_append.argtypes = [vp, cap, bap, tsp, vp, vp, rpp, vp, i64, vp]
    lib.dr_cache_attn_fwd.argtypes = [vp, cap, bap, tsp, i32, vp, vp, i32, vp, vp]
    lib.dr_clock_probe.argtypes = [vp, C.c_uint64, vp, vp]
    lib.dr_mfma_probe.argtypes = [vp, i32, i32, i32, i32, vp, C.POINTER(f64), vp]
    lib.dr_mfma_mix_probe.argtypes = [vp, i32, i32, vp, C.POINTER(f64), vp]
    for name in ("dr_rope_fwd", "dr_rope_bwd", "dr_cache_append", "dr_cache_attn_fwd", "dr_token_scores", "dr_build_mask_tokens", "dr_proxy_loss", "dr_proxy_objective", "dr_static_ratio_for_sparsity", "dr_clock_probe", "dr_mfma_probe", "dr_mfma_mix_probe", "dr_create", "dr_class_map", "dr_mask_capacity", "dr_block_scores", "dr_build_mask",
                 "dr_sparse_attn_fwd", "dr_sparse_attn_fwd_static"):
        getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def version() -> str:
    return load_library().dr_version().decode()


class Context:
    """Owns a dr_ctx (scratch + cached candidate geometry) on one device."""

    def __init__(self, device: int = 0):
        self._lib = load_library()
        self._h = C.c_void_p()
        st = self._lib.dr_create(C.byref(self._h), int(device))
        if st != 0:
            raise DRError(st, f"dr_create(device={device}) failed")
        self.device = device

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            self._lib.dr_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def check(self, st: int):
        if st != 0:
            raise DRError(st, self._lib.dr_last_error(self._h).decode())


def shape_of(t, Nf: int, Hg: int, Wg: int, Bs: int) -> Shape:
    """Shape descriptor of a [B, H, N, d] torch tensor (Q; K, V, O must share its strides)."""
    import torch
    assert t.dim() == 4 and t.stride(3) == 1, "expected [B, H, N, d] with contiguous d"
    dt = {torch.float32: 0, torch.bfloat16: 1}[t.dtype]
    B, H, N, d = t.shape
    return Shape(B, H, N, d, Nf, Hg, Wg, Bs, dt, 0, t.stride(0), t.stride(1), t.stride(2))


def _ptr(t) -> C.c_void_p:
    return C.c_void_p(0 if t is None else t.data_ptr())


def _stream(stream) -> C.c_void_p:
    if stream is None:
        # the handle of torch.cuda.current_stream() without the Stream object around it: that object is 3 us of a call of 8
        import torch
        return C.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))
    return C.c_void_p(getattr(stream, "cuda_stream", stream))


def _pp(params: Optional[MaskParams]):
    return C.byref(params) if params is not None else None


def dr_class_map(ctx: Context, shape: Shape, lam: float, params: Optional[MaskParams], class_map, stream=None):
    ctx.check(ctx._lib.dr_class_map(ctx._h, C.byref(shape), float(lam), _pp(params), _ptr(class_map), _stream(stream)))


def dr_mask_capacity(ctx: Context, shape: Shape, lam: float, params: Optional[MaskParams] = None) -> Tuple[int, int]:
    cand, msel = C.c_int64(0), C.c_int32(0)
    ctx.check(ctx._lib.dr_mask_capacity(ctx._h, C.byref(shape), float(lam), _pp(params), C.byref(cand), C.byref(msel)))
    return cand.value, msel.value


def dr_static_ratio_for_sparsity(ctx: Context, shape: Shape, lam: float, params: Optional[MaskParams],
                                 target: float) -> Tuple[float, float]:
    """(rho, achieved effective sparsity): the largest static ratio on a 1e-3 grid whose mask reaches `target`."""
    rho, got = C.c_double(0.0), C.c_double(0.0)
    ctx.check(ctx._lib.dr_static_ratio_for_sparsity(ctx._h, C.byref(shape), float(lam), _pp(params), float(target),
                                                    C.byref(rho), C.byref(got)))
    return rho.value, got.value


def dr_block_scores(ctx: Context, shape: Shape, Q, K, head_fuse: int, scores, stream=None):
    ctx.check(ctx._lib.dr_block_scores(ctx._h, C.byref(shape), _ptr(Q), _ptr(K), int(head_fuse), _ptr(scores),
                                       _stream(stream)))


def dr_build_mask(ctx: Context, shape: Shape, mode: int, ratio_or_tau: float, lam: float,
                  params: Optional[MaskParams], scores, rowptr, colidx, colidx_capacity: int, nnz, stream=None):
    ctx.check(ctx._lib.dr_build_mask(ctx._h, C.byref(shape), int(mode), float(ratio_or_tau), float(lam), _pp(params),
                                     _ptr(scores), _ptr(rowptr), _ptr(colidx), int(colidx_capacity), _ptr(nnz),
                                     _stream(stream)))


def dr_sparse_attn_fwd(ctx: Context, shape: Shape, Q, K, V, rowptr, colidx, mask_heads: int, colidx_stride: int,
                       O, lse=None, stream=None):
    ctx.check(ctx._lib.dr_sparse_attn_fwd(ctx._h, C.byref(shape), _ptr(Q), _ptr(K), _ptr(V), _ptr(rowptr),
                                          _ptr(colidx), int(mask_heads), int(colidx_stride), _ptr(O), _ptr(lse),
                                          _stream(stream)))


def dr_sparse_attn_fwd_static(ctx: Context, shape: Shape, Q, K, V, rowptr, colidx, mask_heads: int, colidx_stride: int,
                              O, lse=None, stream=None):
    ctx.check(ctx._lib.dr_sparse_attn_fwd_static(ctx._h, C.byref(shape), _ptr(Q), _ptr(K), _ptr(V), _ptr(rowptr),
                                                 _ptr(colidx), int(mask_heads), int(colidx_stride), _ptr(O), _ptr(lse),
                                                 _stream(stream)))


def dr_token_scores(ctx: Context, shape: Shape, Q, K, head_fuse: int, scores, stream=None):
    ctx.check(ctx._lib.dr_token_scores(ctx._h, C.byref(shape), _ptr(Q), _ptr(K), int(head_fuse), _ptr(scores),
                                       _stream(stream)))


def dr_build_mask_tokens(ctx: Context, shape: Shape, tau_near: float, lam: float, params: Optional[MaskParams],
                         token_scores, rowptr, colidx, colidx_capacity: int, nnz, links=None, stream=None):
    ctx.check(ctx._lib.dr_build_mask_tokens(ctx._h, C.byref(shape), float(tau_near), float(lam), _pp(params),
                                            _ptr(token_scores), _ptr(rowptr), _ptr(colidx), int(colidx_capacity),
                                            _ptr(nnz), _ptr(links), _stream(stream)))


def dr_proxy_loss(ctx: Context, A_dense, A_sparse, nnz, Sb: int, target: float, alpha: float, out, stream=None):
    """Enqueue the proxy objective: A_dense, A_sparse float32 [B, H, N, N]; nnz int64 [B, masks]; out float64 [3]."""
    B, H, N, _ = A_dense.shape
    ctx.check(ctx._lib.dr_proxy_loss(ctx._h, _ptr(A_dense), _ptr(A_sparse), int(B), int(H), int(N), _ptr(nnz),
                                     int(nnz.shape[1]), int(Sb), float(target), float(alpha), _ptr(out), _stream(stream)))


def dr_proxy_objective(ctx: Context, shape: Shape, Q, K, rowptr, colidx, mask_heads: int, colidx_stride: int, nnz,
                       target: float, alpha: float, out, stream=None):
    """Enqueue the proxy objective of float32 Q, K under the block CSR; nnz int64 [B, mask_heads]; out float64 [3]."""
    ctx.check(ctx._lib.dr_proxy_objective(ctx._h, C.byref(shape), _ptr(Q), _ptr(K), _ptr(rowptr), _ptr(colidx), int(mask_heads),
                                          int(colidx_stride), _ptr(nnz), float(target), float(alpha), _ptr(out), _stream(stream)))


# ---- streaming: rotary positions, paged cache, attention over it --------------------------------------------

_INVALID = 1


def _refuse(text: str):
    raise DRError(_INVALID, text)


def _need(ok: bool, text: str):
    if not ok:
        _refuse(text)


_DTYPES = None


def _dtype_code(t) -> int:
    global _DTYPES
    if _DTYPES is None:
        import torch
        _DTYPES = {torch.float32: 0, torch.bfloat16: 1}
    code = _DTYPES.get(t.dtype)
    if code is None:
        _refuse(f"dtype {t.dtype}: float32 or bfloat16")
    return code


def _ints(t, name: str, dims: int, device):
    import torch
    if not (t.dtype == torch.int32 and t.dim() == dims and t.device == device and (t.numel() == 0 or t.stride(-1) == 1)):
        _refuse(f"{name}: an int32 tensor of {dims} dimension(s) on {device}, its last one contiguous")


# What a call of these does in Python is of the order of what a launch takes: pointers go through the argument types as plain numbers, devices
# are compared by their numbers (-1: not a GPU), and the text of a refusal is put together only for one.
_raw_stream = None


def _ctx_stream(ctx: Context, stream):
    """The current stream of the context's device (not of the current device, which may be another)."""
    if stream is None:
        global _raw_stream
        if _raw_stream is None:
            import torch
            _raw_stream = torch._C._cuda_getCurrentRawStream
        return _raw_stream(ctx.device)
    return getattr(stream, "cuda_stream", stream)


class PagedCache:
    """Pages of keys and values in e4m3: k [pages, heads, page_tokens, d], v [pages, heads, d, page_tokens], scales [pages, heads].

    A page needs no clearing before it is used (again): the first append to its first slot sets its scale.
    """

    def __init__(self, pages: int, heads: int, page_tokens: int, d: int, device="cuda"):
        import torch
        dev = torch.device(device)
        k = torch.zeros((pages, heads, page_tokens, d), dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)
        v = torch.zeros((pages, heads, d, page_tokens), dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)
        self._set(k, v, *(torch.ones((pages, heads), dtype=torch.float32, device=dev) for _ in range(2)))

    @classmethod
    def of(cls, k, v, k_scale, v_scale) -> "PagedCache":
        """A cache over tensors that the caller has (kept alive by it).  Scales are positive powers of two; one that is none counts as the next
        lower one wherever it is read."""
        self = cls.__new__(cls)
        self._set(k, v, k_scale, v_scale)
        return self

    def _set(self, k, v, k_scale, v_scale):
        import torch
        _need(k.dim() == 4 and v.dim() == 4 and all(t.dtype in (torch.float8_e4m3fn, torch.uint8) and t.is_contiguous() for t in (k, v)),
              "k, v: contiguous float8_e4m3fn (or uint8) tensors of four dimensions")
        pages, heads, page_tokens, d = k.shape
        _need(tuple(v.shape) == (pages, heads, d, page_tokens), f"v must be [pages, heads, d, page_tokens] = {(pages, heads, d, page_tokens)}")
        _need(all(tuple(t.shape) == (pages, heads) and t.dtype == torch.float32 and t.is_contiguous() for t in (k_scale, v_scale)),
              "scales: contiguous float32 [pages, heads]")
        _need(k.device == v.device == k_scale.device == v_scale.device, "the tensors of a cache lie on one device")
        self.k, self.v, self.k_scale, self.v_scale, self.device = k, v, k_scale, v_scale, k.device
        self.pages, self.heads, self.page_tokens, self.d = pages, heads, page_tokens, d
        self.struct = _Cache(pages, heads, page_tokens, d, k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr())

    @staticmethod
    def _powers(scale):
        import torch
        return (scale.view(torch.int32) & 0x7f800000).view(torch.float32)[:, :, None, None]

    def keys(self):
        """float32 [pages, heads, page_tokens, d]: what the codes stand for."""
        import torch
        return self.k.view(torch.float8_e4m3fn).float() * self._powers(self.k_scale)

    def values(self):
        """float32 [pages, heads, page_tokens, d]."""
        import torch
        return (self.v.view(torch.float8_e4m3fn).float() * self._powers(self.v_scale)).transpose(2, 3)


class CacheBatch:
    """A ragged batch: cu int32 [sequences + 1], lens int32 [sequences] (tokens in the cache with the new ones), page_table int32
    [sequences, max_pages]; `tokens`: rows of the tensors that go with it.  The arrays may change between calls (and replays)."""

    def __init__(self, cu, lens, page_table, tokens: int):
        dev = cu.device
        _ints(cu, "cu", 1, dev)
        _ints(lens, "lens", 1, dev)
        _ints(page_table, "page_table", 2, dev)
        n = lens.shape[0]
        _need(cu.shape[0] == n + 1 and page_table.shape[0] == n, "cu, lens and page_table disagree on the number of sequences")
        self.cu, self.lens, self.page_table, self.tokens, self.device = cu, lens, page_table, int(tokens), dev
        # a table of one row may have any row stride
        stride = max(page_table.stride(0), page_table.shape[1]) if n == 1 else page_table.stride(0)
        self.struct = _Batch(n, self.tokens, page_table.shape[1], 0, cu.data_ptr(), lens.data_ptr(), page_table.data_ptr(), stride)


def _rope(ctx: Context, call, rope: RopeParams, X, positions, Y, stream):
    if not (X.dim() == 4 and Y.shape == X.shape and Y.dtype == X.dtype):
        _refuse("X and Y: tensors [B, H, N, d] of one shape and type")
    xs, ys, (B, H, N, d) = X.stride(), Y.stride(), X.shape
    if not (xs[3] == 1 and ys[3] == 1 or X.numel() == 0):
        _refuse("the channels of X and Y must be contiguous")
    if not (X.get_device() == ctx.device and Y.get_device() == ctx.device):
        _refuse(f"X and Y must lie on the context's device {ctx.device}")
    ps_b = ps_a = 0
    if positions is not None:
        dims = positions.dim()
        if dims not in (2, 3):
            _refuse("positions: [axes, N] or [B, axes, N]")
        _ints(positions, "positions", dims, X.device)
        if not (positions.shape[-2] == rope.axes and positions.shape[-1] == N and (dims == 2 or positions.shape[0] == B)):
            _refuse(f"positions: [{rope.axes}, {N}] or [{B}, {rope.axes}, {N}]")
        ps_a = positions.stride(-2)
        ps_b = positions.stride(0) if dims == 3 else 0
    shape = RopeShape(B, H, N, d, _dtype_code(X), 0, xs[0], xs[1], xs[2], ys[0], ys[1], ys[2])
    ctx.check(call(ctx._h, C.byref(shape), C.byref(rope), X.data_ptr(), None if positions is None else positions.data_ptr(), ps_b, ps_a,
                   Y.data_ptr(), _ctx_stream(ctx, stream)))


def dr_rope_fwd(ctx: Context, rope: RopeParams, X, positions, Y, stream=None):
    """Y = R X: X, Y [B, H, N, d] (Y may be X); positions int32 [axes, N] or [B, axes, N]."""
    _rope(ctx, ctx._lib.dr_rope_fwd, rope, X, positions, Y, stream)


def dr_rope_bwd(ctx: Context, rope: RopeParams, dY, positions, dX, stream=None):
    """dX = R^T dY: the gradient of dr_rope_fwd's X (dX may be dY)."""
    _rope(ctx, ctx._lib.dr_rope_bwd, rope, dY, positions, dX, stream)


def _token_strides(ctx: Context, cache: PagedCache, batch: CacheBatch, a, b, heads_of: str):
    if not (a.dim() == 3 and b.shape == a.shape and b.dtype == a.dtype and a.shape[0] == batch.tokens and a.shape[2] == cache.d):
        _refuse(f"{heads_of}: tensors [{batch.tokens}, heads, {cache.d}] of one shape and type")
    s, t = a.stride(), b.stride()
    if not (s[2] == 1 and t[2] == 1 or a.numel() == 0):
        _refuse(f"the channels of {heads_of} must be contiguous")
    if not (a.get_device() == b.get_device() == cache.k.get_device() == batch.cu.get_device() == ctx.device):
        _refuse(f"all tensors must lie on the context's device {ctx.device}")
    return _TokenStrides(_dtype_code(a), 0, s[0], s[1], t[0], t[1])


def dr_cache_append(ctx: Context, cache: PagedCache, batch: CacheBatch, K, V, rope: Optional[RopeParams] = None, positions=None, stream=None):
    """Keys (rotated) and values [tokens, heads, d] into the batch's pages; positions int32 [axes, tokens], or None: places in the sequence."""
    strides = _token_strides(ctx, cache, batch, K, V, "K, V")
    if K.shape[1] != cache.heads:
        _refuse(f"K, V have {K.shape[1]} heads, the cache {cache.heads}")
    ps_a, at = 0, None
    if positions is not None:
        _ints(positions, "positions", 2, K.device)
        if not (rope is not None and tuple(positions.shape) == (rope.axes, batch.tokens)):
            _refuse("positions: [axes, tokens], with a rope")
        ps_a, at = positions.stride(0), positions.data_ptr()
    ctx.check(ctx._lib.dr_cache_append(ctx._h, C.byref(cache.struct), C.byref(batch.struct), C.byref(strides), K.data_ptr(), V.data_ptr(),
                                       C.byref(rope) if rope is not None else None, at, ps_a, _ctx_stream(ctx, stream)))


def dr_cache_attn_fwd(ctx: Context, cache: PagedCache, batch: CacheBatch, Q, O, causal: bool = True, lse=None, stream=None):
    """Attention of the new tokens' queries [tokens, heads, d] over the cache; lse: optional float32 [heads, tokens]."""
    strides, heads, at = _token_strides(ctx, cache, batch, Q, O, "Q, O"), Q.shape[1], None
    if lse is not None:
        import torch
        if not (lse.dtype == torch.float32 and tuple(lse.shape) == (heads, batch.tokens) and lse.is_contiguous() and lse.get_device() == ctx.device):
            _refuse("lse: contiguous float32 [heads, tokens] beside Q")
        at = lse.data_ptr()
    ctx.check(ctx._lib.dr_cache_attn_fwd(ctx._h, C.byref(cache.struct), C.byref(batch.struct), C.byref(strides), heads, Q.data_ptr(), O.data_ptr(),
                                         1 if causal else 0, at, _ctx_stream(ctx, stream)))


def dr_clock_probe(ctx: Context, window_us: int, out, stream=None):
    """Enqueue the clock probe: `out` is a device int64 tensor of two entries (shader ticks, 100 MHz ticks)."""
    ctx.check(ctx._lib.dr_clock_probe(ctx._h, int(window_us), _ptr(out), _stream(stream)))


def dr_mfma_probe(ctx: Context, shape: int, workgroups: int, iters: int, random_operands: bool, sink,
                  stream=None) -> float:
    """Enqueue the MFMA-only loop (shape 32: 32x32x16, 16: 16x16x32); returns the flop count of the launch."""
    flop = C.c_double(0.0)
    ctx.check(ctx._lib.dr_mfma_probe(ctx._h, int(shape), int(workgroups), int(iters), 1 if random_operands else 0,
                                     _ptr(sink), C.byref(flop), _stream(stream)))
    return flop.value


def dr_mfma_mix_probe(ctx: Context, workgroups: int, iters: int, sink, stream=None) -> float:
    """Enqueue the loop of one 32x32x16 matrix instruction + one exponential + two fp32 instructions per slot."""
    flop = C.c_double(0.0)
    ctx.check(ctx._lib.dr_mfma_mix_probe(ctx._h, int(workgroups), int(iters), _ptr(sink), C.byref(flop), _stream(stream)))
    return flop.value
