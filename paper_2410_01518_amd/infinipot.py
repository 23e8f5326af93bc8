"""ctypes binding of libinfinipot (include/infinipot.h).

Argument marshalling only: every step of the path runs in the library's HIP kernels.  Tensors are
torch CUDA tensors (torch owns device memory and streams); bf16 caches may be passed as torch.bfloat16
or as int16/uint16 bit patterns.  There is no CPU fallback: if the shared library is missing the import
of any entry point raises.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libinfinipot.so")

CCD_OK, CCD_NOOP = 0, 1
CCD_EINVAL, CCD_EUNSUPPORTED, CCD_EALIGN, CCD_EWORKSPACE, CCD_ELAUNCH = -1, -2, -3, -4, -5
CCD_FP32, CCD_BF16 = 0, 1
CCD_POOL_NONE, CCD_POOL_MAX, CCD_POOL_AVG = 0, 1, 2
CCD_PATH_AUTO, CCD_PATH_VALU, CCD_PATH_MFMA_SLICES, CCD_PATH_MFMA_UNIT = 0, 1, 2, 3
CCD_ROPE_HALF, CCD_ROPE_PAIRS = 0, 1
CCD_ROPE_PLAIN, CCD_ROPE_LINEAR, CCD_ROPE_NTK, CCD_ROPE_PARTS = 0, 1, 2, 3
CCD_INT8, CCD_E4M3 = 0, 1

EXPORTS = ("ccd_workspace_bytes", "ccd_score", "ccd_select", "ccd_compact", "ccd_compress", "ccd_append", "ccd_cr_rope",
           "ccd_compress_rope", "ccd_score_kcat", "ccd_compress_kcat", "ccd_score_lse", "ccd_compress_lse",
           "ccd_nuc_from_logits", "ccd_compress_noalloc", "ccd_profile_enable", "ccd_profile_stages", "ccd_profile_stage_name",
           "ccd_profile_collect", "ccd_strerror", "ccd_paged_plan", "ccd_rope_turns", "ccd_rope", "ccd_paged_append",
           "ccd_paged_workspace_bytes", "ccd_paged_attend", "ccd_paged_append_codes", "ccd_paged_read_codes", "ccd_codes_workspace_bytes",
           "ccd_paged_attend_codes", "ccd_paged_compact_codes")


class ccd_shape_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("B", "L", "Hq", "Hkv", "d", "n_valid", "n_cap", "k", "P", "T", "pool_w", "pool_mode", "dtype")]
    _fields_ += [("scale", ctypes.c_float), ("window", ctypes.c_int32), ("score_path", ctypes.c_int32)]
    _fields_ += [(n, ctypes.c_int64) for n in
                 ("kv_stride_b", "kv_stride_l", "kv_stride_h", "q_stride_b", "q_stride_l", "q_stride_h",
                  "nov_stride_b", "nov_stride_l", "nov_stride_h")]


class ccd_paged_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("B", "tokens", "Hq", "Hkv", "d", "dtype", "page", "n_pages", "table_width", "window", "behind", "max_new", "max_len")]
    _fields_ += [("scale", ctypes.c_float)]
    _fields_ += [(n, ctypes.c_int64) for n in
                 ("page_stride", "head_stride", "row_stride", "new_stride_t", "new_stride_h", "q_stride_b", "q_stride_t", "q_stride_h",
                  "o_stride_b", "o_stride_t", "o_stride_h", "lse_stride_b", "lse_stride_t", "lse_stride_h")]
    _appended = _attended = _read = _compacted = None   # the geometry, descriptor and tensors, of its last calls (below)


class ccd_rope_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("tokens", "heads", "d", "rot", "dtype", "layout", "inverse")]
    _fields_ += [("amplitude", ctypes.c_float)]
    _fields_ += [(n, ctypes.c_int64) for n in ("x_stride_t", "x_stride_h", "y_stride_t", "y_stride_h")]
    _fields_ += [("scaling", ctypes.c_int32), ("context", ctypes.c_int32)]
    _fields_ += [(n, ctypes.c_double) for n in ("base", "factor", "low", "high")]
    _turned = None


class ccd_codes_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("code", "scale_rows")]
    _fields_ += [(n, ctypes.c_int64) for n in ("scale_page_stride", "scale_head_stride", "new_rows", "new_stride_b")]


class CCDError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"libinfinipot: {text} (code {code})")
        self.code = code


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2410_01518_amd.build` "
                "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        vp, sp = ctypes.c_void_p, ctypes.POINTER(ccd_shape_t)
        L.ccd_workspace_bytes.restype = ctypes.c_size_t
        L.ccd_workspace_bytes.argtypes = [sp]
        L.ccd_score.restype = ctypes.c_int
        L.ccd_score.argtypes = [sp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.ccd_select.restype = ctypes.c_int
        L.ccd_select.argtypes = [sp, vp, vp, vp]
        L.ccd_compact.restype = ctypes.c_int
        L.ccd_compact.argtypes = [sp, vp, vp, vp, vp, vp, vp, vp]
        L.ccd_compress.restype = ctypes.c_int
        L.ccd_compress.argtypes = [sp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.ccd_append.restype = ctypes.c_int
        L.ccd_append.argtypes = [sp, vp, vp, vp, vp, vp, vp, ctypes.c_int32, vp]
        L.ccd_compress_noalloc.restype = ctypes.c_int
        L.ccd_compress_noalloc.argtypes = [sp, vp, vp, vp, vp, vp, vp, vp]
        L.ccd_cr_rope.restype = ctypes.c_int
        L.ccd_cr_rope.argtypes = [sp, vp, vp, vp, ctypes.c_int32, vp, vp]
        L.ccd_compress_rope.restype = ctypes.c_int
        L.ccd_compress_rope.argtypes = [sp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.ccd_score_lse.restype = ctypes.c_int
        L.ccd_score_lse.argtypes = [sp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.ccd_compress_lse.restype = ctypes.c_int
        L.ccd_compress_lse.argtypes = [sp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.ccd_score_kcat.restype = ctypes.c_int
        L.ccd_score_kcat.argtypes = [sp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.ccd_compress_kcat.restype = ctypes.c_int
        L.ccd_compress_kcat.argtypes = [sp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.ccd_nuc_from_logits.restype = ctypes.c_int
        L.ccd_nuc_from_logits.argtypes = [vp, vp, vp, ctypes.c_int64, ctypes.c_int32, ctypes.c_int64, ctypes.c_int32, vp]
        cp, rp = ctypes.POINTER(ccd_paged_t), ctypes.POINTER(ccd_rope_t)
        L.ccd_paged_plan.restype = ctypes.c_int
        L.ccd_paged_plan.argtypes = [cp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.ccd_rope_turns.restype = ctypes.c_int
        L.ccd_rope_turns.argtypes = [rp, vp]
        L.ccd_rope.restype = ctypes.c_int
        L.ccd_rope.argtypes = [rp, vp, vp, vp, vp, vp]
        L.ccd_paged_append.restype = ctypes.c_int
        L.ccd_paged_append.argtypes = [cp, rp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.ccd_paged_workspace_bytes.restype = ctypes.c_size_t
        L.ccd_paged_workspace_bytes.argtypes = [cp]
        L.ccd_paged_attend.restype = ctypes.c_int
        L.ccd_paged_attend.argtypes = [cp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        kp = ctypes.POINTER(ccd_codes_t)
        L.ccd_paged_append_codes.restype = ctypes.c_int
        L.ccd_paged_append_codes.argtypes = [cp, kp, rp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.ccd_paged_read_codes.restype = ctypes.c_int
        L.ccd_paged_read_codes.argtypes = [cp, kp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.ccd_codes_workspace_bytes.restype = ctypes.c_size_t
        L.ccd_codes_workspace_bytes.argtypes = [cp, kp]
        L.ccd_paged_attend_codes.restype = ctypes.c_int
        L.ccd_paged_attend_codes.argtypes = [cp, kp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.ccd_paged_compact_codes.restype = ctypes.c_int
        L.ccd_paged_compact_codes.argtypes = [cp, kp, vp, vp, vp, vp, vp, ctypes.c_int32, vp, vp]
        L.ccd_profile_enable.restype = ctypes.c_int
        L.ccd_profile_enable.argtypes = [ctypes.c_int]
        L.ccd_profile_stages.restype = ctypes.c_int
        L.ccd_profile_stages.argtypes = []
        L.ccd_profile_stage_name.restype = ctypes.c_char_p
        L.ccd_profile_stage_name.argtypes = [ctypes.c_int]
        L.ccd_profile_collect.restype = ctypes.c_int
        L.ccd_profile_collect.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
        L.ccd_strerror.restype = ctypes.c_char_p
        L.ccd_strerror.argtypes = [ctypes.c_int]
        _lib = L
    return _lib


def ccd_strerror(code: int) -> str:
    return lib().ccd_strerror(code).decode()


def _check(code: int) -> int:
    if code < 0:
        raise CCDError(code, ccd_strerror(code))
    return code


# The address and the stream handle go in as plain integers, which ctypes turns into pointers by the declared argument types.
# torch.cuda.current_stream() builds a Stream object through several layers of Python (6 us of a call that takes 30 us in
# all on a small pot); the raw handle is one C call.
def _ptr(t):
    return None if t is None else t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _dtype_code_of(dtype) -> int:
    if dtype == torch.float32:
        return CCD_FP32
    if dtype in (torch.bfloat16, torch.int16, torch.uint16):
        return CCD_BF16
    raise TypeError(f"unsupported cache dtype {dtype}")


def _dtype_code(t: torch.Tensor) -> int:
    return _dtype_code_of(t.dtype)


def make_shape(Q_cat, K, novelty, *, k, T=0, pool_w=1, pool_mode=CCD_POOL_MAX, scale=0.0, n_valid=None,
               window=0, score_path=CCD_PATH_AUTO) -> ccd_shape_t:
    """Shape descriptor from tensor geometry: Q_cat [B,L,Hq,P,d], K [B,L,Hkv,n_cap,d], novelty [B,n] or
    [B,L,Hkv,n_cap] (may be None when T == 0).  Q_cat may be None for calls that do not read it."""
    B, L, Hkv, n_cap, d = K.shape
    kb, kl, kh, kt, ke = K.stride()
    assert ke == 1 and kt == d, "K rows must be contiguous with stride d"
    if Q_cat is not None:
        Hq, P = Q_cat.shape[2], Q_cat.shape[3]
        qb, ql, qh, qt, qe = Q_cat.stride()
        assert qe == 1 and qt == d
    else:
        Hq, P = Hkv, 1
        qb, ql, qh = 0, 0, d
    nb = nl = nh = 0
    if novelty is not None:
        assert novelty.dtype == torch.float32 and novelty.stride(-1) == 1
        if novelty.dim() == 2:
            nb = novelty.stride(0)
        else:
            nb, nl, nh, _ = novelty.stride()
    return ccd_shape_t(B, L, Hq, Hkv, d, n_cap if n_valid is None else n_valid, n_cap, k, P, T, pool_w, pool_mode,
                       _dtype_code(K), scale, window, score_path, kb, kl, kh, qb, ql, qh, nb, nl, nh)


def ccd_workspace_bytes(shape: ccd_shape_t) -> int:
    return int(lib().ccd_workspace_bytes(ctypes.byref(shape)))


def alloc_workspace(shape: ccd_shape_t, device="cuda") -> torch.Tensor:
    nbytes = ccd_workspace_bytes(shape)
    if nbytes == 0:
        raise CCDError(CCD_EINVAL, "invalid shape")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def ccd_score(shape, Q_cat, K, novelty, scores, workspace, stream=None) -> int:
    return _check(lib().ccd_score(ctypes.byref(shape), _ptr(Q_cat), _ptr(K), _ptr(novelty), _ptr(scores),
                                  _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream(stream)))


def ccd_select(shape, scores, keep_idx, stream=None) -> int:
    return _check(lib().ccd_select(ctypes.byref(shape), _ptr(scores), _ptr(keep_idx), _stream(stream)))


def ccd_append(shape, K, V, novelty, K_new, V_new, novelty_new, stream=None) -> int:
    """Rows shape.n_valid .. + count - 1 of every unit of K, V (and novelty) <- the chunk K_new, V_new [B,L,Hkv,count,d]
    (dense) and novelty_new [B,count]; the caller raises n_valid afterwards."""
    assert K_new.is_contiguous() and V_new.is_contiguous() and (novelty_new is None or novelty_new.is_contiguous())
    return _check(lib().ccd_append(ctypes.byref(shape), _ptr(K), _ptr(V), _ptr(novelty), _ptr(K_new), _ptr(V_new),
                                   _ptr(novelty_new), int(K_new.shape[3]), _stream(stream)))


def ccd_compact(shape, K_src, V_src, keep_idx, K_dst, V_dst, novelty_inout=None, stream=None) -> int:
    return _check(lib().ccd_compact(ctypes.byref(shape), _ptr(K_src), _ptr(V_src), _ptr(keep_idx), _ptr(K_dst),
                                    _ptr(V_dst), _ptr(novelty_inout), _stream(stream)))


def ccd_compress(shape, Q_cat, K, V, novelty, keep_idx, workspace, scores=None, stream=None) -> int:
    return _check(lib().ccd_compress(ctypes.byref(shape), _ptr(Q_cat), _ptr(K), _ptr(V), _ptr(novelty), _ptr(scores),
                                     _ptr(keep_idx), _ptr(workspace), 0 if workspace is None else workspace.numel(),
                                     _stream(stream)))


NOALLOC_WORKSPACE_BYTES = (16 << 20) + (8 << 10)


def ccd_compress_noalloc(shape, Q_cat, K, V, novelty, keep_idx, scores=None, stream=None) -> int:
    """ccd_compress on the workspace the library holds itself (no allocation anywhere in the call)."""
    return _check(lib().ccd_compress_noalloc(ctypes.byref(shape), _ptr(Q_cat), _ptr(K), _ptr(V), _ptr(novelty), _ptr(scores),
                                             _ptr(keep_idx), _stream(stream)))


def ccd_nuc_from_logits(logits, labels, novelty, stream=None) -> int:
    """novelty[r] = cross entropy of labels[r] under logits[r, :]; logits [..., V] with a dense last axis and equally
    spaced rows, labels and novelty with the same leading shape (flattened row-major)."""
    V = logits.shape[-1]
    assert logits.stride(-1) == 1 and labels.dtype == torch.int32 and novelty.dtype == torch.float32
    assert labels.is_contiguous() and novelty.is_contiguous() and labels.numel() == novelty.numel()
    lead = logits.shape[:-1]
    rows = int(np.prod(lead)) if len(lead) else 1
    flat = logits.reshape(rows, V) if rows else logits
    assert rows == 0 or flat.data_ptr() == logits.data_ptr(), "rows must be equally spaced"
    esz = logits.element_size()
    stride = flat.stride(0) if rows > 1 else (V * esz + 15) // 16 * 16 // esz   # a single row: any legal stride
    return _check(lib().ccd_nuc_from_logits(_ptr(logits), _ptr(labels), _ptr(novelty), rows, V, stride,
                                            _dtype_code(logits), _stream(stream)))


def ccd_cr_rope(shape, K, rope_cos, rope_sin, count, K_rot, stream=None) -> int:
    return _check(lib().ccd_cr_rope(ctypes.byref(shape), _ptr(K), _ptr(rope_cos), _ptr(rope_sin), int(count), _ptr(K_rot),
                                    _stream(stream)))


def ccd_compress_rope(shape, Q_cat, K, V, novelty, keep_idx, rope_cos, rope_sin, K_rot, workspace, scores=None,
                      K_score=None, K_cap=None, lse=None, stream=None) -> int:
    assert lse is None or (lse.is_contiguous() and lse.dtype == torch.float32)
    return _check(lib().ccd_compress_rope(ctypes.byref(shape), _ptr(Q_cat), _ptr(K), _ptr(V), _ptr(novelty), _ptr(scores),
                                          _ptr(keep_idx), _ptr(K_score), _ptr(K_cap), _ptr(lse), _ptr(rope_cos), _ptr(rope_sin),
                                          _ptr(K_rot), _ptr(workspace), 0 if workspace is None else workspace.numel(),
                                          _stream(stream)))


def ccd_score_kcat(shape, Q_cat, K, K_cap, novelty, scores, workspace, stream=None) -> int:
    """K_cap [B, L, Hkv, P, d], contiguous."""
    assert K_cap is None or K_cap.is_contiguous()
    return _check(lib().ccd_score_kcat(ctypes.byref(shape), _ptr(Q_cat), _ptr(K), _ptr(K_cap), _ptr(novelty), _ptr(scores),
                                       _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream(stream)))


def ccd_score_lse(shape, Q_cat, K, lse, novelty, scores, workspace, stream=None) -> int:
    """lse [B, L, Hq, P] fp32, contiguous: the natural-log-sum-exp of every CaP query's attention row."""
    assert lse is None or (lse.is_contiguous() and lse.dtype == torch.float32)
    return _check(lib().ccd_score_lse(ctypes.byref(shape), _ptr(Q_cat), _ptr(K), _ptr(lse), _ptr(novelty), _ptr(scores),
                                      _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream(stream)))


def ccd_compress_lse(shape, Q_cat, K, V, lse, novelty, keep_idx, workspace, scores=None, stream=None) -> int:
    assert lse is None or (lse.is_contiguous() and lse.dtype == torch.float32)
    return _check(lib().ccd_compress_lse(ctypes.byref(shape), _ptr(Q_cat), _ptr(K), _ptr(V), _ptr(lse), _ptr(novelty),
                                         _ptr(scores), _ptr(keep_idx), _ptr(workspace),
                                         0 if workspace is None else workspace.numel(), _stream(stream)))


def ccd_compress_kcat(shape, Q_cat, K, V, K_cap, novelty, keep_idx, workspace, scores=None, stream=None) -> int:
    assert K_cap is None or K_cap.is_contiguous()
    return _check(lib().ccd_compress_kcat(ctypes.byref(shape), _ptr(Q_cat), _ptr(K), _ptr(V), _ptr(K_cap), _ptr(novelty),
                                          _ptr(scores), _ptr(keep_idx), _ptr(workspace),
                                          0 if workspace is None else workspace.numel(), _stream(stream)))


# ---- paged caches

# The checks below stand in the way of calls whose kernels take 4 us.  So attributes of a tensor are read once each, and a call of the same geometry as the
# descriptor's last one (its bytes, the tensors' types, shapes and strides) is not held against the rules again.
_I32 = torch.int32
_get_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _stream_here(stream, *tensors):
    """The stream to launch on; all tensors must be on the current device: kernels take their addresses as they are."""
    device = _get_device()
    for t in tensors:
        if t.get_device() != device:
            raise ValueError(f"a tensor on {t.device}, and the current device is cuda:{device}")
    if stream is not None:
        return stream.cuda_stream
    return torch.cuda.current_stream().cuda_stream if _raw_stream is None else _raw_stream(device)


def _int32(entries, *tensors):
    """Index tensors, and the entries that the descriptor says they have."""
    for t in tensors:
        if t.dtype is not _I32 or not t.is_contiguous():
            raise AssertionError("contiguous int32 needed")
        if t.numel() < entries:
            raise AssertionError(f"{t.numel()} entries, {entries} needed")


def _turns(turns, rope):
    if turns.dtype is not torch.int64 or turns.numel() < rope.rot // 2 or not turns.is_contiguous():
        raise AssertionError("turns as rope_turns gives them needed")


def _alike(a, b):
    if a.stride() != b.stride() or a.dtype is not b.dtype or a.shape != b.shape:
        raise AssertionError("keys and values differ in shape, strides or type")


def _holds(t, shape, strides, more=0):
    """t has what a descriptor of this geometry reaches: its own (more rows at most), or one that ends behind it.  `more`: elements
    that a batch of it lies further on."""
    own = t.shape
    if t.stride() == strides and own[0] >= shape[0] and own[1:] == shape[1:] and not more:
        return
    if min(shape) > 0 and more + sum((n - 1) * s for n, s in zip(shape, strides)) > sum((n - 1) * s for n, s in zip(own, t.stride())):
        raise AssertionError(f"a tensor of shape {tuple(own)} and strides {t.stride()}, and the descriptor has {shape}, {strides}")


def make_plan(block_table, *, tokens, page, n_pages) -> ccd_paged_t:
    """Descriptor of a step's plan alone: block_table [B, table_width], a cache of n_pages pages of `page` tokens, `tokens` entries in
    the slot map."""
    B, W = block_table.shape
    return ccd_paged_t(B=B, tokens=tokens, page=page, n_pages=n_pages, table_width=W)


def make_paged(K_pages, *, tokens, block_table=None, Q=None, out=None, lse=None, K_new=None, window=0, behind=False, max_new=0,
               max_len=0, scale=0.0, dtype=None) -> ccd_paged_t:
    """Descriptor from tensor geometry: K_pages (and V_pages) [n_pages, Hkv, page, d] in any order of the outer three
    dimensions, block_table [B, table_width].  Q and out are [tokens, Hq, d] with lse [tokens, Hq], or, `tokens` = B m,
    [B, Hq, m, d] with lse [B, Hq, m]; K_new (and V_new) [tokens, Hkv, d].  Where K_pages are codes, dtype is that of the others, an `out`
    without Q has Hkv heads (for reading back), and K_new may be [B, Hkv, m, d] (which make_codes then has to be told, too)."""
    n_pages, Hkv, page, d = K_pages.shape
    dtype = K_pages.dtype if dtype is None else dtype
    ps, hs, rs, es = K_pages.stride()
    assert es == 1, "rows of the cache must be contiguous"
    p = ccd_paged_t(B=1, tokens=tokens, Hq=Hkv, Hkv=Hkv, d=d, dtype=_dtype_code_of(dtype), page=page, n_pages=n_pages, table_width=1,
                    window=window, behind=int(behind), max_new=max_new, max_len=max_len, scale=scale, page_stride=ps, head_stride=hs,
                    row_stride=rs, new_stride_t=Hkv * d, new_stride_h=d)
    if block_table is not None:
        p.B, p.table_width = block_table.shape
    if K_new is not None and K_new.dim() == 4 and K_pages.dtype in CODE_TYPES:
        assert K_new.shape[0] * K_new.shape[2] == tokens and K_new.shape[1::2] == (Hkv, d) and K_new.stride(3) == 1 and K_new.dtype == dtype
        p.new_stride_t, p.new_stride_h = K_new.stride(2), K_new.stride(1)
    elif K_new is not None:
        assert tuple(K_new.shape) == (tokens, Hkv, d) and K_new.stride(2) == 1 and K_new.dtype == dtype
        p.new_stride_t, p.new_stride_h = K_new.stride(0), K_new.stride(1)
    p.Hq = Hkv if Q is None else Q.shape[1]
    for t, name, batched in ((Q, "q", 4), (out, "o", 4), (lse, "lse", 3)):
        if t is None:
            strides = (0, p.Hq, 1) if name == "lse" else (0, p.Hq * d, d)
        else:
            if name == "lse":
                assert t.dtype == torch.float32
            else:
                assert t.shape[-1] == d and t.stride(-1) == 1 and t.dtype == dtype
            assert t.shape[1] == p.Hq
            if t.dim() == batched:
                m = t.shape[2]
                assert t.shape[0] == p.B and p.B * m == tokens
                strides = (t.stride(0) - m * t.stride(2), t.stride(2), t.stride(1))
            else:
                assert t.shape[0] == tokens
                strides = (0, t.stride(0), t.stride(1))
        for axis, v in zip("bth", strides):
            setattr(p, f"{name}_stride_{axis}", v)
    return p


def make_rope(X, Y=None, *, rot=None, layout=CCD_ROPE_HALF, base=10000.0, scaling=CCD_ROPE_PLAIN, factor=1.0, context=0, low=1.0, high=4.0,
              amplitude=0.0, inverse=False) -> ccd_rope_t:
    """Descriptor from tensor geometry: X and Y [tokens, heads, d] with contiguous heads (Y: X where none is given)."""
    Y = X if Y is None else Y
    T, H, d = X.shape
    assert tuple(Y.shape) == (T, H, d) and X.stride(2) == 1 and Y.stride(2) == 1 and X.dtype == Y.dtype
    return ccd_rope_t(tokens=T, heads=H, d=d, rot=d if rot is None else rot, dtype=_dtype_code(X), layout=layout, inverse=int(inverse),
                      amplitude=amplitude, x_stride_t=X.stride(0), x_stride_h=X.stride(1), y_stride_t=Y.stride(0), y_stride_h=Y.stride(1),
                      scaling=scaling, context=context, base=base, factor=factor, low=low, high=high)


def rope_turns(rope: ccd_rope_t, device="cuda") -> torch.Tensor:
    """The descriptor's frequencies for ccd_rope and ccd_paged_append, int64 [rot / 2] on the device (fractions of 2^64)."""
    host = torch.empty(max(rope.rot, 2) // 2, dtype=torch.int64)
    _check(lib().ccd_rope_turns(ctypes.byref(rope), host.data_ptr()))
    return host.to(device)


def alloc_paged_workspace(paged: ccd_paged_t, device="cuda") -> torch.Tensor:
    nbytes = ccd_paged_workspace_bytes(paged)
    if nbytes == 0:
        raise CCDError(CCD_EINVAL, "invalid descriptor")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def ccd_paged_workspace_bytes(paged: ccd_paged_t) -> int:
    return int(lib().ccd_paged_workspace_bytes(ctypes.byref(paged)))


def ccd_paged_plan(paged, len_before, len_after, block_table, block_table_next, free_pages, cursor, cursor_next, q_start, slots, positions,
                   stream=None) -> int:
    """len_before, len_after [B], block_table and block_table_next [B, table_width] (may be one), free_pages [n_pages], cursor and
    cursor_next [4] (may be one), q_start [B + 1], slots and positions [tokens]: int32."""
    B, tokens = paged.B, paged.tokens
    table = B * paged.table_width
    # (one pass over ten tensors, without ten calls)
    for t, entries in ((len_before, B), (len_after, B), (block_table, table), (block_table_next, table), (free_pages, paged.n_pages), (cursor, 4), (cursor_next, 4),
                       (q_start, B + 1), (slots, tokens), (positions, tokens)):
        if t.dtype is not _I32 or t.numel() < entries or not t.is_contiguous():
            _int32(entries, t)
    stream = _stream_here(stream, len_before, len_after, block_table, block_table_next, free_pages, cursor, cursor_next, q_start, slots, positions)
    return _check(lib().ccd_paged_plan(ctypes.byref(paged), len_before.data_ptr(), len_after.data_ptr(), block_table.data_ptr(), block_table_next.data_ptr(),
                                       free_pages.data_ptr(), cursor.data_ptr(), cursor_next.data_ptr(), q_start.data_ptr(), slots.data_ptr(),
                                       positions.data_ptr(), stream))


def _check_rope(rope, X, positions, turns, Y):
    tokens, heads, d = shape = rope.tokens, rope.heads, rope.d
    _int32(tokens, positions)
    _turns(turns, rope)
    _holds(X, shape, (rope.x_stride_t, rope.x_stride_h, 1))
    _holds(Y, shape, (rope.y_stride_t, rope.y_stride_h, 1))
    if X.dtype is not Y.dtype or _dtype_code(X) != rope.dtype:
        raise AssertionError("X, Y and the descriptor differ in type")


def ccd_rope(rope, X, positions, turns, Y, stream=None) -> int:
    """positions int32 [tokens]; turns as rope_turns gives them; Y may be X."""
    geometry = (bytes(rope), X.dtype, X.shape, X.stride(), positions.dtype, positions.shape, positions.is_contiguous(), turns.dtype, turns.shape, turns.is_contiguous(),
                Y.dtype, Y.shape, Y.stride())
    if geometry != rope._turned:
        _check_rope(rope, X, positions, turns, Y)
        rope._turned = geometry
    stream = _stream_here(stream, X, positions, turns, Y)
    return _check(lib().ccd_rope(ctypes.byref(rope), X.data_ptr(), positions.data_ptr(), turns.data_ptr(), Y.data_ptr(), stream))


def _check_append(paged, rope, K_new, V_new, slots, K_pages, V_pages, positions, turns):
    tokens, Hkv, d = paged.tokens, paged.Hkv, paged.d
    _alike(K_new, V_new)
    _alike(K_pages, V_pages)
    if K_new.dtype is not K_pages.dtype or _dtype_code(K_pages) != paged.dtype:
        raise AssertionError("new keys, the cache and the descriptor differ in type")
    _holds(K_new, (tokens, Hkv, d), (paged.new_stride_t, paged.new_stride_h, 1))
    _holds(K_pages, (paged.n_pages, Hkv, paged.page, d), (paged.page_stride, paged.head_stride, paged.row_stride, 1))
    _int32(tokens, slots)
    if rope is not None:
        _int32(tokens, positions)
        _turns(turns, rope)


def ccd_paged_append(paged, K_new, V_new, slots, K_pages, V_pages, rope=None, positions=None, turns=None, stream=None) -> int:
    """K_new and V_new have the same strides, as have K_pages and V_pages; with a rope descriptor the keys are embedded at `positions`."""
    geometry = (bytes(paged), K_new.dtype, K_new.shape, K_new.stride(), V_new.dtype, V_new.shape, V_new.stride(), slots.dtype, slots.shape, slots.is_contiguous(),
                K_pages.dtype, K_pages.shape, K_pages.stride(), V_pages.dtype, V_pages.shape, V_pages.stride())
    if rope is not None:
        geometry += (bytes(rope), positions.dtype, positions.shape, positions.is_contiguous(), turns.dtype, turns.shape, turns.is_contiguous())
    if geometry != paged._appended:
        _check_append(paged, rope, K_new, V_new, slots, K_pages, V_pages, positions, turns)
        paged._appended = geometry
    if rope is None:
        return _check(lib().ccd_paged_append(ctypes.byref(paged), None, K_new.data_ptr(), V_new.data_ptr(), slots.data_ptr(), None, None, K_pages.data_ptr(),
                                             V_pages.data_ptr(), _stream_here(stream, K_new, V_new, slots, K_pages, V_pages)))
    return _check(lib().ccd_paged_append(ctypes.byref(paged), ctypes.byref(rope), K_new.data_ptr(), V_new.data_ptr(), slots.data_ptr(), positions.data_ptr(),
                                         turns.data_ptr(), K_pages.data_ptr(), V_pages.data_ptr(),
                                         _stream_here(stream, K_new, V_new, slots, K_pages, V_pages, positions, turns)))


def _check_attend(paged, Q, K_pages, V_pages, block_table, q_start, kv_len, out, lse):
    B, dtype, shape = paged.B, K_pages.dtype, (paged.tokens, paged.Hq, paged.d)
    _int32(B * paged.table_width, block_table)
    _int32(B + 1, q_start)
    _int32(B, kv_len)
    _alike(K_pages, V_pages)
    if Q.dtype is not dtype or out.dtype is not dtype or (lse is not None and lse.dtype is not torch.float32) or _dtype_code(K_pages) != paged.dtype:
        raise AssertionError("Q, out, the cache and the descriptor differ in type, or lse is not fp32")
    _holds(K_pages, (paged.n_pages, paged.Hkv, paged.page, paged.d), (paged.page_stride, paged.head_stride, paged.row_stride, 1))
    _holds(Q, shape, (paged.q_stride_t, paged.q_stride_h, 1), (B - 1) * paged.q_stride_b)
    _holds(out, shape, (paged.o_stride_t, paged.o_stride_h, 1), (B - 1) * paged.o_stride_b)
    if lse is not None:
        _holds(lse, shape[:2], (paged.lse_stride_t, paged.lse_stride_h), (B - 1) * paged.lse_stride_b)


def ccd_paged_attend(paged, Q, K_pages, V_pages, block_table, q_start, kv_len, out, lse, workspace, stream=None) -> int:
    """block_table [B, table_width], q_start [B + 1], kv_len [B]: int32; lse fp32 or None."""
    geometry = (bytes(paged), Q.dtype, Q.shape, Q.stride(), K_pages.dtype, K_pages.shape, K_pages.stride(), V_pages.dtype, V_pages.shape, V_pages.stride(),
                block_table.dtype, block_table.shape, block_table.is_contiguous(), q_start.dtype, q_start.shape, q_start.is_contiguous(),
                kv_len.dtype, kv_len.shape, kv_len.is_contiguous(), out.dtype, out.shape, out.stride())
    there = (Q, K_pages, V_pages, block_table, q_start, kv_len, out)
    if lse is not None:
        geometry += (lse.dtype, lse.shape, lse.stride())
        there += (lse,)
    if geometry != paged._attended:
        _check_attend(paged, Q, K_pages, V_pages, block_table, q_start, kv_len, out, lse)
        paged._attended = geometry
    stream = _stream_here(stream, *there) if workspace is None else _stream_here(stream, *there, workspace)
    return _check(lib().ccd_paged_attend(ctypes.byref(paged), Q.data_ptr(), K_pages.data_ptr(), V_pages.data_ptr(), block_table.data_ptr(), q_start.data_ptr(),
                                         kv_len.data_ptr(), out.data_ptr(), None if lse is None else lse.data_ptr(),
                                         *((None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel())), stream))


# ---- paged caches in 8 bits

CODE_TYPES = {torch.int8: CCD_INT8, torch.float8_e4m3fn: CCD_E4M3}


def make_codes(K_codes, K_scales, K_new=None) -> ccd_codes_t:
    """Descriptor from tensor geometry: K_codes (and V_codes) [n_pages, Hkv, page, d], int8 or float8_e4m3fn, K_scales (and V_scales)
    [n_pages, Hkv, page / scale_rows] fp32.  K_new [B, Hkv, m, d] (and V_new): new tokens in that order, where they are not [tokens, Hkv, d]."""
    n_pages, Hkv, page, d = K_codes.shape
    if K_codes.dtype not in CODE_TYPES:
        raise TypeError(f"unsupported code type {K_codes.dtype}")
    assert K_scales.dtype == torch.float32 and K_scales.shape[:2] == (n_pages, Hkv) and (K_scales.shape[2] == 1 or K_scales.stride(2) == 1)
    rows = page // max(1, K_scales.shape[2])
    assert rows * K_scales.shape[2] == page, "a scale for every scale_rows tokens"
    new_rows = new_b = 0
    if K_new is not None and K_new.dim() == 4:
        new_rows, new_b = K_new.shape[2], K_new.stride(0)
    return ccd_codes_t(CODE_TYPES[K_codes.dtype], rows, K_scales.stride(0), K_scales.stride(1), new_rows, new_b)


def ccd_codes_workspace_bytes(paged: ccd_paged_t, codes: ccd_codes_t) -> int:
    return int(lib().ccd_codes_workspace_bytes(ctypes.byref(paged), ctypes.byref(codes)))


def alloc_codes_workspace(paged: ccd_paged_t, codes: ccd_codes_t, device="cuda") -> torch.Tensor:
    nbytes = ccd_codes_workspace_bytes(paged, codes)
    if nbytes == 0:
        raise CCDError(CCD_EINVAL, "invalid descriptor")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _check_cache(paged, codes, K_codes, V_codes, K_scales, V_scales):
    """What the descriptors say of codes and scales; K or V may be None."""
    for a, b in ((K_codes, V_codes), (K_scales, V_scales)):
        if a is not None and b is not None:
            _alike(a, b)
    rows = codes.scale_rows
    for c, s in ((K_codes, K_scales), (V_codes, V_scales)):
        if c is None and s is None:
            continue
        if CODE_TYPES.get(c.dtype) != codes.code or s.dtype is not torch.float32:
            raise AssertionError("codes, scales and the descriptor differ in type")
        _holds(c, (paged.n_pages, paged.Hkv, paged.page, paged.d), (paged.page_stride, paged.head_stride, paged.row_stride, 1))
        _holds(s, (paged.n_pages, paged.Hkv, paged.page // rows if rows > 0 else 0), (codes.scale_page_stride, codes.scale_head_stride, 1))


def _check_append_codes(paged, codes, rope, K_new, V_new, slots, K_codes, V_codes, K_scales, V_scales, positions, turns):
    tokens, Hkv, d = paged.tokens, paged.Hkv, paged.d
    _alike(K_new, V_new)
    if _dtype_code(K_new) != paged.dtype:
        raise AssertionError("new keys and the descriptor differ in type")
    if codes.new_rows > 0 and K_new.dim() == 4:
        full = -(-tokens // codes.new_rows)
        _holds(K_new, (full, Hkv, codes.new_rows, d), (codes.new_stride_b, paged.new_stride_h, paged.new_stride_t, 1))
    else:
        if codes.new_rows > 0 or (K_new.dim() != 3 and tokens > 0):
            raise AssertionError("new keys [B, Hkv, m, d] needed" if codes.new_rows > 0 else "new keys [tokens, Hkv, d] needed, or a descriptor made for [B, Hkv, m, d]")
        _holds(K_new, (tokens, Hkv, d), (paged.new_stride_t, paged.new_stride_h, 1))
    _check_cache(paged, codes, K_codes, V_codes, K_scales, V_scales)
    _int32(tokens, slots)
    if rope is not None:
        _int32(tokens, positions)
        _turns(turns, rope)


def ccd_paged_append_codes(paged, codes, K_new, V_new, slots, K_codes, V_codes, K_scales, V_scales, rope=None, positions=None, turns=None, stream=None) -> int:
    """K_new and V_new have the same strides, as have codes and scales of keys and values; with a rope descriptor the keys are embedded at `positions`."""
    geometry = (bytes(paged), bytes(codes), K_new.dtype, K_new.shape, K_new.stride(), V_new.dtype, V_new.shape, V_new.stride(), slots.dtype, slots.shape, slots.stride(),
                K_codes.dtype, K_codes.shape, K_codes.stride(), V_codes.dtype, V_codes.shape, V_codes.stride(), K_scales.dtype, K_scales.shape, K_scales.stride(),
                V_scales.dtype, V_scales.shape, V_scales.stride())
    if rope is not None:
        geometry += (bytes(rope), positions.dtype, positions.shape, positions.stride(), turns.dtype, turns.shape, turns.stride())
    if geometry != paged._appended:
        _check_append_codes(paged, codes, rope, K_new, V_new, slots, K_codes, V_codes, K_scales, V_scales, positions, turns)
        paged._appended = geometry
    if rope is None:
        return _check(lib().ccd_paged_append_codes(ctypes.byref(paged), ctypes.byref(codes), None, K_new.data_ptr(), V_new.data_ptr(), slots.data_ptr(), None, None,
                                                   K_codes.data_ptr(), V_codes.data_ptr(), K_scales.data_ptr(), V_scales.data_ptr(),
                                                   _stream_here(stream, K_new, V_new, slots, K_codes, V_codes, K_scales, V_scales)))
    return _check(lib().ccd_paged_append_codes(ctypes.byref(paged), ctypes.byref(codes), ctypes.byref(rope), K_new.data_ptr(), V_new.data_ptr(), slots.data_ptr(),
                                               positions.data_ptr(), turns.data_ptr(), K_codes.data_ptr(), V_codes.data_ptr(), K_scales.data_ptr(), V_scales.data_ptr(),
                                               _stream_here(stream, K_new, V_new, slots, K_codes, V_codes, K_scales, V_scales, positions, turns)))


def _check_read_codes(paged, codes, K_codes, V_codes, K_scales, V_scales, block_table, q_start, kv_len, K_out, V_out):
    B = paged.B
    _int32(B * paged.table_width, block_table)
    _int32(B + 1, q_start)
    _int32(B, kv_len)
    if K_out is not None and V_out is not None:
        _alike(K_out, V_out)
    _check_cache(paged, codes, K_codes if K_out is not None else None, V_codes if V_out is not None else None, K_scales if K_out is not None else None,
                 V_scales if V_out is not None else None)
    for out in (K_out, V_out):
        if out is not None:
            if _dtype_code(out) != paged.dtype:
                raise AssertionError("the numbers read and the descriptor differ in type")
            _holds(out, (paged.tokens, paged.Hkv, paged.d), (paged.o_stride_t, paged.o_stride_h, 1), (B - 1) * paged.o_stride_b)


def ccd_paged_read_codes(paged, codes, K_codes, V_codes, K_scales, V_scales, block_table, q_start, kv_len, K_out, V_out, stream=None) -> int:
    """block_table [B, table_width], q_start [B + 1], kv_len [B]: int32; K_out or V_out may be None (its codes and scales then, too)."""
    geometry = (bytes(paged), bytes(codes), block_table.dtype, block_table.shape, block_table.stride(), q_start.dtype, q_start.shape, q_start.stride(), kv_len.dtype,
                kv_len.shape, kv_len.stride())
    there = (block_table, q_start, kv_len)
    if K_out is not None:
        geometry += (K_codes.dtype, K_codes.shape, K_codes.stride(), K_scales.dtype, K_scales.shape, K_scales.stride(), K_out.dtype, K_out.shape, K_out.stride())
        there += (K_codes, K_scales, K_out)
    if V_out is not None:
        geometry += (V_codes.dtype, V_codes.shape, V_codes.stride(), V_scales.dtype, V_scales.shape, V_scales.stride(), V_out.dtype, V_out.shape, V_out.stride(), K_out is None)
        there += (V_codes, V_scales, V_out)
    if geometry != paged._read:
        _check_read_codes(paged, codes, K_codes, V_codes, K_scales, V_scales, block_table, q_start, kv_len, K_out, V_out)
        paged._read = geometry
    return _check(lib().ccd_paged_read_codes(ctypes.byref(paged), ctypes.byref(codes), _ptr(K_codes), _ptr(V_codes), _ptr(K_scales), _ptr(V_scales), block_table.data_ptr(),
                                             q_start.data_ptr(), kv_len.data_ptr(), _ptr(K_out), _ptr(V_out), _stream_here(stream, *there)))


def _check_attend_codes(paged, codes, Q, K_codes, V_codes, K_scales, V_scales, block_table, q_start, kv_len, out, lse):
    B, shape = paged.B, (paged.tokens, paged.Hq, paged.d)
    _int32(B * paged.table_width, block_table)
    _int32(B + 1, q_start)
    _int32(B, kv_len)
    if Q.dtype is not out.dtype or _dtype_code(Q) != paged.dtype or (lse is not None and lse.dtype is not torch.float32):
        raise AssertionError("Q, out and the descriptor differ in type, or lse is not fp32")
    _check_cache(paged, codes, K_codes, V_codes, K_scales, V_scales)
    _holds(Q, shape, (paged.q_stride_t, paged.q_stride_h, 1), (B - 1) * paged.q_stride_b)
    _holds(out, shape, (paged.o_stride_t, paged.o_stride_h, 1), (B - 1) * paged.o_stride_b)
    if lse is not None:
        _holds(lse, shape[:2], (paged.lse_stride_t, paged.lse_stride_h), (B - 1) * paged.lse_stride_b)


def ccd_paged_attend_codes(paged, codes, Q, K_codes, V_codes, K_scales, V_scales, block_table, q_start, kv_len, out, lse, workspace, stream=None) -> int:
    """block_table [B, table_width], q_start [B + 1], kv_len [B]: int32; lse fp32 or None."""
    geometry = (bytes(paged), bytes(codes), Q.dtype, Q.shape, Q.stride(), K_codes.dtype, K_codes.shape, K_codes.stride(), V_codes.dtype, V_codes.shape, V_codes.stride(),
                K_scales.dtype, K_scales.shape, K_scales.stride(), V_scales.dtype, V_scales.shape, V_scales.stride(), block_table.dtype, block_table.shape, block_table.stride(),
                q_start.dtype, q_start.shape, q_start.stride(), kv_len.dtype, kv_len.shape, kv_len.stride(), out.dtype, out.shape, out.stride())
    there = (Q, K_codes, V_codes, K_scales, V_scales, block_table, q_start, kv_len, out)
    if lse is not None:
        geometry += (lse.dtype, lse.shape, lse.stride())
        there += (lse,)
    if geometry != paged._attended:
        _check_attend_codes(paged, codes, Q, K_codes, V_codes, K_scales, V_scales, block_table, q_start, kv_len, out, lse)
        paged._attended = geometry
    stream = _stream_here(stream, *there) if workspace is None else _stream_here(stream, *there, workspace)
    return _check(lib().ccd_paged_attend_codes(ctypes.byref(paged), ctypes.byref(codes), Q.data_ptr(), K_codes.data_ptr(), V_codes.data_ptr(), K_scales.data_ptr(),
                                               V_scales.data_ptr(), block_table.data_ptr(), q_start.data_ptr(), kv_len.data_ptr(), out.data_ptr(),
                                               None if lse is None else lse.data_ptr(), *((None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel())),
                                               stream))


def _check_compact_codes(paged, codes, K_codes, V_codes, K_scales, V_scales, keep_idx, novelty):
    _check_cache(paged, codes, K_codes, V_codes, K_scales, V_scales)
    _int32(paged.n_pages * paged.Hkv * keep_idx.shape[-1], keep_idx)
    if novelty is not None and (novelty.dtype is not torch.float32 or not novelty.is_contiguous() or novelty.numel() < paged.n_pages * paged.Hkv * paged.page):
        raise AssertionError("novelty [n_pages, Hkv, page] fp32, contiguous, needed")


def ccd_paged_compact_codes(paged, codes, K_codes, V_codes, K_scales, V_scales, keep_idx, novelty=None, stream=None) -> int:
    """keep_idx int32 [n_pages, Hkv, k], novelty fp32 [n_pages, Hkv, page] or None, both contiguous; in place."""
    geometry = (bytes(paged), bytes(codes), K_codes.dtype, K_codes.shape, K_codes.stride(), V_codes.dtype, V_codes.shape, V_codes.stride(), K_scales.dtype, K_scales.shape,
                K_scales.stride(), V_scales.dtype, V_scales.shape, V_scales.stride(), keep_idx.dtype, keep_idx.shape, keep_idx.stride())
    there = (K_codes, V_codes, K_scales, V_scales, keep_idx)
    if novelty is not None:
        geometry += (novelty.dtype, novelty.shape, novelty.stride())
        there += (novelty,)
    if geometry != paged._compacted:
        _check_compact_codes(paged, codes, K_codes, V_codes, K_scales, V_scales, keep_idx, novelty)
        paged._compacted = geometry
    return _check(lib().ccd_paged_compact_codes(ctypes.byref(paged), ctypes.byref(codes), K_codes.data_ptr(), V_codes.data_ptr(), K_scales.data_ptr(), V_scales.data_ptr(),
                                                keep_idx.data_ptr(), keep_idx.shape[-1], _ptr(novelty), _stream_here(stream, *there)))


def ccd_profile_enable(on: bool) -> int:
    return _check(lib().ccd_profile_enable(1 if on else 0))


def ccd_profile_collect():
    """(dict stage name -> total ms, number of ccd_compress calls covered) since profiling was enabled."""
    n = lib().ccd_profile_stages()
    ms = (ctypes.c_double * n)()
    calls = ctypes.c_int64(0)
    _check(lib().ccd_profile_collect(ms, ctypes.byref(calls)))
    return {lib().ccd_profile_stage_name(i).decode(): ms[i] for i in range(n)}, calls.value
