"""ctypes binding of libsift (include/sift.h).  Marshalling only: every step
of the hot path runs in the library's HIP kernels; torch provides device
memory and the current stream."""

from __future__ import annotations

import ctypes
import math
import os
import re

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsift.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "sift.h")
SERVE_HEADER = os.path.join(os.path.dirname(HERE), "include", "sift_serve.h")

SIFT_F32 = 0
SIFT_BF16 = 1

STATUS = {
    0: "SIFT_OK", 1: "SIFT_E_NULL", 2: "SIFT_E_SHAPE", 3: "SIFT_E_LAYOUT",
    4: "SIFT_E_UNSUPPORTED", 5: "SIFT_E_CAPACITY", 6: "SIFT_E_HIP", 7: "SIFT_E_PLAN",
}


class SiftError(RuntimeError):
    def __init__(self, fn: str, status: int, msg: str):
        super().__init__(f"{fn}: {STATUS.get(status, status)} ({msg})")
        self.status = status


class SiftTensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("tokens", ctypes.c_int32),
                ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


class SiftLayout(ctypes.Structure):
    _fields_ = [("num_prompts", ctypes.c_int32),
                ("prompt_seg_ptr", ctypes.POINTER(ctypes.c_int32)),
                ("seg_offsets", ctypes.POINTER(ctypes.c_int32))]


class SiftPlanInfo(ctypes.Structure):
    _fields_ = [("num_tokens", ctypes.c_int32), ("num_segments", ctypes.c_int32),
                ("num_tiles", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("tile", ctypes.c_int32), ("num_work_units", ctypes.c_int32),
                ("num_rows", ctypes.c_int64), ("list_capacity", ctypes.c_int64),
                ("la_bytes", ctypes.c_int64), ("ca_bytes", ctypes.c_int64),
                ("scratch_bytes", ctypes.c_int64)]


class SiftScore(ctypes.Structure):
    _fields_ = [("softmax_scale", ctypes.c_float), ("cap", ctypes.c_float),
                ("slopes", ctypes.c_void_p)]


class SiftCacheKv(ctypes.Structure):
    _fields_ = [("k_pages", ctypes.POINTER(SiftTensor)), ("v_pages", ctypes.POINTER(SiftTensor)),
                ("page_table", ctypes.c_void_p), ("lens", ctypes.c_void_p),
                ("page_lens", ctypes.c_void_p), ("key_pos", ctypes.c_void_p)]


class SiftCacheRows(ctypes.Structure):
    _fields_ = [("row_ptr", ctypes.c_void_p), ("row_pos", ctypes.c_void_p)]


MASKS = {"causal": 0, "document": 1, "prefix": 2}

_P = ctypes.c_void_p
_SIGS = {
    "sift_status_string": (ctypes.c_char_p, [ctypes.c_int32]),
    "sift_plan_create": (ctypes.c_int, [ctypes.POINTER(SiftLayout), ctypes.c_int32, ctypes.c_int32,
                                        ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(_P)]),
    "sift_plan_destroy": (ctypes.c_int, [_P]),
    "sift_plan_get_info": (ctypes.c_int, [_P, ctypes.POINTER(SiftPlanInfo)]),
    "sift_plan_exact_passes": (ctypes.c_int, [_P, ctypes.POINTER(ctypes.c_int64)]),
    "sift_plan_decode_tiles": (ctypes.c_int, [_P, _P, _P, _P, _P, ctypes.c_int64, _P]),
    "sift_decode_workspace_bytes": (ctypes.c_int, [ctypes.POINTER(SiftLayout), ctypes.c_int32,
                                                   ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]),
    "sift_decode_tiles": (ctypes.c_int, [ctypes.POINTER(SiftLayout), _P, _P, ctypes.c_int32,
                                         ctypes.c_int32, _P, _P, ctypes.c_int64, _P,
                                         ctypes.c_size_t, _P]),
    "sift_sparse_attention": (ctypes.c_int, [_P, ctypes.POINTER(SiftTensor), ctypes.POINTER(SiftTensor),
                                             ctypes.POINTER(SiftTensor), _P, _P, ctypes.c_int64,
                                             ctypes.c_float, ctypes.POINTER(SiftTensor), _P]),
    "sift_plan_decode": (ctypes.c_int, [_P, _P, _P, _P]),
    "sift_plan_attention": (ctypes.c_int, [_P, ctypes.POINTER(SiftTensor), ctypes.POINTER(SiftTensor),
                                           ctypes.POINTER(SiftTensor), ctypes.c_float,
                                           ctypes.POINTER(SiftTensor), _P]),
    "sift_plan_run": (ctypes.c_int, [_P, ctypes.POINTER(SiftTensor), ctypes.POINTER(SiftTensor),
                                     ctypes.POINTER(SiftTensor), _P, _P, ctypes.c_float,
                                     ctypes.POINTER(SiftTensor), _P]),
    "sift_plan_run_paged": (ctypes.c_int, [_P, ctypes.POINTER(SiftTensor), ctypes.POINTER(SiftTensor),
                                           ctypes.POINTER(SiftTensor), _P, _P, _P, ctypes.c_float,
                                           ctypes.POINTER(SiftTensor), _P]),
    "sift_sparse_prefill": (ctypes.c_int, [ctypes.POINTER(SiftTensor), ctypes.POINTER(SiftTensor),
                                           ctypes.POINTER(SiftTensor), ctypes.POINTER(SiftLayout),
                                           _P, _P, ctypes.c_int32, ctypes.POINTER(SiftTensor), _P]),
    "sift_workspace_bytes": (ctypes.c_int, [ctypes.POINTER(SiftLayout), ctypes.c_int32, ctypes.c_int32,
                                            ctypes.c_int32, ctypes.c_int32,
                                            ctypes.POINTER(ctypes.c_size_t)]),
    "sift_sparse_prefill_ex": (ctypes.c_int, [ctypes.POINTER(SiftTensor), ctypes.POINTER(SiftTensor),
                                              ctypes.POINTER(SiftTensor), ctypes.POINTER(SiftLayout),
                                              _P, _P, ctypes.c_int32, ctypes.c_float, _P,
                                              ctypes.c_size_t, ctypes.POINTER(SiftTensor), _P]),
    "sift_sparse_prefill_static": (ctypes.c_int, [ctypes.POINTER(SiftTensor),
                                                  ctypes.POINTER(SiftTensor),
                                                  ctypes.POINTER(SiftTensor),
                                                  ctypes.POINTER(SiftLayout), _P, _P,
                                                  ctypes.c_int32, ctypes.c_float,
                                                  ctypes.POINTER(SiftTensor), _P]),
    "sift_static_scratch_bytes": (ctypes.c_size_t, []),
    "sift_rope": (ctypes.c_int, [ctypes.POINTER(SiftTensor), ctypes.POINTER(SiftTensor), _P, _P, _P]),
    "sift_extract_sizes": (ctypes.c_int, [ctypes.c_int32, _P, ctypes.c_int32, ctypes.c_int32,
                                          ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(ctypes.c_size_t),
                                          ctypes.POINTER(ctypes.c_size_t)]),
    "sift_extract_bits": (ctypes.c_int, [ctypes.POINTER(SiftTensor), ctypes.POINTER(SiftTensor),
                                         ctypes.c_int32, _P, ctypes.c_int32, ctypes.c_double,
                                         ctypes.c_double, ctypes.c_double, ctypes.c_float, _P, _P, _P,
                                         ctypes.c_size_t, _P]),
}

# include/sift_serve.h
_SERVE_SIGS = {
    "sift_plan_dense": (ctypes.c_int, [_P, ctypes.POINTER(SiftTensor), ctypes.POINTER(SiftTensor),
                                       ctypes.POINTER(SiftTensor), ctypes.c_int32,
                                       ctypes.POINTER(SiftScore), ctypes.POINTER(SiftTensor), _P,
                                       _P]),
    "sift_cache_create": (ctypes.c_int, [ctypes.c_int32] * 7 + [ctypes.POINTER(_P)]),
    "sift_cache_destroy": (ctypes.c_int, [_P]),
    "sift_cache_attention": (ctypes.c_int, [_P, ctypes.POINTER(SiftCacheKv),
                                            ctypes.POINTER(SiftCacheRows),
                                            ctypes.POINTER(SiftTensor), ctypes.POINTER(SiftTensor),
                                            ctypes.POINTER(SiftTensor), _P, ctypes.c_int32,
                                            ctypes.POINTER(SiftScore), ctypes.POINTER(SiftTensor),
                                            _P, _P]),
    "sift_cache_accumulate": (ctypes.c_int, [_P, ctypes.POINTER(SiftCacheKv),
                                             ctypes.POINTER(SiftCacheRows),
                                             ctypes.POINTER(SiftTensor), _P, _P,
                                             ctypes.POINTER(SiftScore), _P, ctypes.c_float, _P,
                                             _P]),
    "sift_cache_evict": (ctypes.c_int, [_P, ctypes.POINTER(SiftCacheKv), _P, _P, ctypes.c_int32,
                                        ctypes.c_int32, ctypes.c_int32, _P, _P, _P, _P]),
}

# entries of the decoder layer (csrc/layer_api.h), not part of sift.h
_LAYER_SIGS = {
    "sift_layer_rms_norm": (ctypes.c_int, [_P, _P, ctypes.c_int64, ctypes.c_int32, ctypes.c_float, _P,
                                           _P]),
    "sift_layer_silu_mul": (ctypes.c_int, [_P, _P, ctypes.c_int64, _P, _P]),
}

_lib = None


def header_functions(header: str = HEADER) -> list[str]:
    """Names of the functions include/sift.h (or another header) declares."""
    with open(header) as f:
        text = f.read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(sift_[a-z_]+)\s*\(", text)))


def lib() -> ctypes.CDLL:
    """Load libsift.so once.  Raises if it has not been built: there is no
    fallback path."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2606_09441_amd.build` (no fallback exists)")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in (*_SIGS.items(), *_SERVE_SIGS.items(), *_LAYER_SIGS.items()):
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def check(fn: str, status: int) -> None:
    if status != 0:
        msg = lib().sift_status_string(status).decode()
        raise SiftError(fn, status, msg)


# ----------------------------------------------------------------------------
# torch marshalling
# ----------------------------------------------------------------------------


_torch_module = None
_dtypes, _kinds = {}, {}


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _dtypes.update(uint8=torch.uint8, int32=torch.int32, int64=torch.int64,
                       float32=torch.float32)
        _kinds.update({torch.bfloat16: SIFT_BF16, torch.float32: SIFT_F32})
        _torch_module = torch
    return _torch_module


def tensor_desc(t) -> SiftTensor:
    _torch()
    if not getattr(t, "is_cuda", False):
        raise SiftError("tensor_desc", 4, "tensors must be in GPU memory")
    shape = t.shape
    if len(shape) != 3:
        raise ValueError("expected a [tokens, heads, head_dim] tensor")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    kind = _kinds.get(t.dtype)
    if kind is None:
        raise ValueError(f"unsupported dtype {t.dtype}")
    return SiftTensor(t.data_ptr(), kind, *shape)


def require(fn: str, t, name: str, dtype: str, min_numel: int, device=None) -> None:
    """Check a device buffer before its pointer goes to the library, which
    cannot see buffer sizes: a GPU tensor (on `device` when given), of
    `dtype` ("uint8", "int32", "int64", "float32"), contiguous, with at least
    min_numel elements.  Raises SiftError otherwise."""
    torch = _torch()
    want = _dtypes[dtype]
    if t is None:
        if min_numel > 0:
            raise SiftError(fn, 1, f"{name} is required")
        return
    if not isinstance(t, torch.Tensor):
        raise SiftError(fn, 4, f"{name} must be a torch tensor")
    if t.dtype is not want:
        raise SiftError(fn, 4, f"{name} must be {dtype}, not {t.dtype}")
    if not t.is_contiguous():
        raise SiftError(fn, 2, f"{name} must be contiguous")
    if t.numel() < min_numel:
        raise SiftError(fn, 5, f"{name} holds {t.numel()} elements, needs {min_numel}")
    if not t.is_cuda:
        raise SiftError(fn, 4, f"{name} must be a GPU tensor")
    if device is not None and t.device != device:
        raise SiftError(fn, 7, f"{name} is on {t.device}, the plan on {device}")


def bitmap_bytes(seg_offsets, prompt_seg_ptr, num_q_heads: int, tile: int) -> tuple[int, int]:
    """(LA bytes, CA bytes) the bit-vector buffers of a layout hold, from the
    library (sift_extract_sizes over the layout's documents in order)."""
    so = np.asarray(seg_offsets, dtype=np.int64)
    ps = np.asarray(prompt_seg_ptr, dtype=np.int64)
    lens = [int(so[s + 1] - so[s]) for b in range(len(ps) - 1)
            for s in range(int(ps[b]), int(ps[b + 1]) - 1)]
    if not lens:
        return 0, 0
    if min(lens) < 1:
        raise SiftError("bitmap_bytes", 3, "documents must hold at least one token")
    offs = np.ascontiguousarray(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32))
    la, ca = ctypes.c_size_t(), ctypes.c_size_t()
    check("sift_extract_sizes", lib().sift_extract_sizes(len(lens), offs.ctypes.data_as(_P),
                                                         num_q_heads, tile, ctypes.byref(la),
                                                         ctypes.byref(ca), None))
    return la.value, ca.value


def require_laid_out(fn: str, t, name: str, dtype: str, sizes: tuple, device=None) -> None:
    """require of a buffer that the library reads as one of these sizes."""
    n = 1
    for x in sizes:
        n *= x
    require(fn, t, name, dtype, n, device)
    if t is not None and t.numel() != n:
        check_laid_out(fn, name, t.shape, sizes)


def check_laid_out(fn: str, name: str, shape, sizes: tuple) -> None:
    """A contiguous buffer of more elements than the library reads has to hold those
    at the same places: it may have more rows, or be flat, but no longer rows."""
    for i in range(1, min(len(shape), len(sizes))):   # dimensions from the last on
        if shape[-i] != sizes[-i] and math.prod(sizes[:-i]) > 1:
            raise SiftError(fn, 2, f"{name} is {tuple(shape)}, has to be {sizes}")


def layout_struct(seg_offsets, prompt_seg_ptr):
    so = np.ascontiguousarray(np.asarray(seg_offsets, dtype=np.int32))
    ps = np.ascontiguousarray(np.asarray(prompt_seg_ptr, dtype=np.int32))
    lay = SiftLayout(len(ps) - 1, ps.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                     so.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)))
    return lay, (so, ps)  # keep the arrays alive with the struct


def _stream_ptr(stream):
    if stream is not None:
        return ctypes.c_void_p(stream.cuda_stream)
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # without a Stream object
    if raw is not None:
        return raw(torch.cuda.current_device())
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _ptr(t):
    return ctypes.c_void_p(0 if t is None else t.data_ptr())


class Plan:
    """A validated prompt layout with its device tables (sift_plan_*)."""

    def __init__(self, seg_offsets, prompt_seg_ptr, num_q_heads, num_kv_heads, head_dim, tile=64):
        self._h = None
        lay, keep = layout_struct(seg_offsets, prompt_seg_ptr)
        h = ctypes.c_void_p()
        check("sift_plan_create", lib().sift_plan_create(ctypes.byref(lay), num_q_heads, num_kv_heads,
                                                         head_dim, tile, ctypes.byref(h)))
        self._h = h
        torch = _torch()
        self.device = torch.device("cuda", torch.cuda.current_device())
        inf = SiftPlanInfo()
        check("sift_plan_get_info", lib().sift_plan_get_info(self._h, ctypes.byref(inf)))
        self.info = {name: getattr(inf, name) for name, _ in SiftPlanInfo._fields_}

    def close(self):
        if self._h is not None:
            check("sift_plan_destroy", lib().sift_plan_destroy(self._h))
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def _bits(self, fn, la, ca):
        require(fn, la, "local_bitmap", "uint8", self.info["la_bytes"], self.device)
        require(fn, ca, "cross_bitmap", "uint8", self.info["ca_bytes"], self.device)

    def decode(self, la, ca, row_ptr=None, col_idx=None, stream=None):
        """Decoded lists (Section 5.1) as device int32 tensors (row_ptr, col_idx)."""
        torch = _torch()
        self._bits("sift_plan_decode_tiles", la, ca)
        dev = la.device
        if row_ptr is None:
            row_ptr = torch.empty(self.info["num_rows"] + 1, dtype=torch.int32, device=dev)
        if col_idx is None:
            col_idx = torch.empty(max(1, self.info["list_capacity"]), dtype=torch.int32, device=dev)
        require("sift_plan_decode_tiles", row_ptr, "row_ptr", "int32", self.info["num_rows"] + 1,
                self.device)
        require("sift_plan_decode_tiles", col_idx, "col_idx", "int32", self.info["list_capacity"],
                self.device)
        check("sift_plan_decode_tiles", lib().sift_plan_decode_tiles(
            self._h, _ptr(la), _ptr(ca), _ptr(row_ptr), _ptr(col_idx), col_idx.numel(),
            _stream_ptr(stream)))
        return row_ptr, col_idx

    def attention(self, q, k, v, row_ptr, col_idx, scale=None, out=None, out_dtype=None, stream=None):
        """Sparse attention over given lists (Section 5.2)."""
        torch = _torch()
        require("sift_sparse_attention", row_ptr, "row_ptr", "int32", self.info["num_rows"] + 1,
                self.device)
        require("sift_sparse_attention", col_idx, "col_idx", "int32", 0, self.device)
        if out is None:
            out = torch.empty(q.shape, dtype=out_dtype or q.dtype, device=q.device)
        qd, kd, vd, od = tensor_desc(q), tensor_desc(k), tensor_desc(v), tensor_desc(out)
        check("sift_sparse_attention", lib().sift_sparse_attention(
            self._h, ctypes.byref(qd), ctypes.byref(kd), ctypes.byref(vd), _ptr(row_ptr),
            _ptr(col_idx), col_idx.numel(), ctypes.c_float(0.0 if scale is None else scale),
            ctypes.byref(od), _stream_ptr(stream)))
        return out

    def exact_passes(self) -> int:
        """Attention launches on this plan that needed the exact second pass
        (sift_plan_exact_passes; waits for the plan's last stream)."""
        n = ctypes.c_int64()
        check("sift_plan_exact_passes", lib().sift_plan_exact_passes(self._h, ctypes.byref(n)))
        return n.value

    def decode_internal(self, la, ca, stream=None):
        """Decode into the plan's own scratch (sift_plan_decode)."""
        self._bits("sift_plan_decode", la, ca)
        check("sift_plan_decode", lib().sift_plan_decode(self._h, _ptr(la), _ptr(ca),
                                                         _stream_ptr(stream)))

    def attention_internal(self, q, k, v, scale=None, out=None, out_dtype=None, stream=None):
        """Attention over the plan's last decode (sift_plan_attention)."""
        torch = _torch()
        if out is None:
            out = torch.empty(q.shape, dtype=out_dtype or q.dtype, device=q.device)
        qd, kd, vd, od = tensor_desc(q), tensor_desc(k), tensor_desc(v), tensor_desc(out)
        check("sift_plan_attention", lib().sift_plan_attention(
            self._h, ctypes.byref(qd), ctypes.byref(kd), ctypes.byref(vd),
            ctypes.c_float(0.0 if scale is None else scale), ctypes.byref(od), _stream_ptr(stream)))
        return out

    def run(self, q, k, v, la, ca, scale=None, out=None, out_dtype=None, stream=None):
        """Decode + attention for one layer (sift_plan_run)."""
        torch = _torch()
        self._bits("sift_plan_run", la, ca)
        if out is None:
            out = torch.empty(q.shape, dtype=out_dtype or q.dtype, device=q.device)
        qd, kd, vd, od = tensor_desc(q), tensor_desc(k), tensor_desc(v), tensor_desc(out)
        check("sift_plan_run", lib().sift_plan_run(
            self._h, ctypes.byref(qd), ctypes.byref(kd), ctypes.byref(vd), _ptr(la), _ptr(ca),
            ctypes.c_float(0.0 if scale is None else scale), ctypes.byref(od), _stream_ptr(stream)))
        return out

    def run_paged(self, q, k_pages, v_pages, page_table, la, ca, scale=None, out=None,
                  out_dtype=None, stream=None):
        """Decode + attention with K/V in a page pool (sift_plan_run_paged):
        k_pages/v_pages [num_pages * T, Hkv, D], page_table int32 [num_tiles]."""
        torch = _torch()
        self._bits("sift_plan_run_paged", la, ca)
        require("sift_plan_run_paged", page_table, "page_table", "int32", self.info["num_tiles"],
                self.device)
        if out is None:
            out = torch.empty(q.shape, dtype=out_dtype or q.dtype, device=q.device)
        qd, kd, vd, od = tensor_desc(q), tensor_desc(k_pages), tensor_desc(v_pages), tensor_desc(out)
        check("sift_plan_run_paged", lib().sift_plan_run_paged(
            self._h, ctypes.byref(qd), ctypes.byref(kd), ctypes.byref(vd), _ptr(page_table),
            _ptr(la), _ptr(ca), ctypes.c_float(0.0 if scale is None else scale), ctypes.byref(od),
            _stream_ptr(stream)))
        return out


    def dense(self, q, k, v, mask="causal", scale=None, cap=0.0, slopes=None, out=None, lse=None,
              stream=None):
        """Dense attention with transformed scores (sift_plan_dense): mask "causal",
        "document" or "prefix"; scores capped by cap * tanh(s / cap) (cap > 0) and
        biased by -slopes[h] * distance (float32 [Hq]).  lse: float32 [tokens, Hq]
        buffer that receives the rows' log sum exp."""
        fn = "sift_plan_dense"
        if mask not in MASKS:
            raise SiftError(fn, 4, f"mask must be one of {sorted(MASKS)}")
        score = score_struct(fn, scale, cap, slopes, self.info["num_q_heads"], self.device)
        if lse is not None:
            require_laid_out(fn, lse, "lse", "float32",
                             (self.info["num_tokens"], self.info["num_q_heads"]), self.device)
        if out is None:
            out = _empty_like(q, stream)
        dev = self.device
        check(fn, lib().sift_plan_dense(
            self._h, _desc(fn, q, "q", dev), _desc(fn, k, "k", dev), _desc(fn, v, "v", dev),
            MASKS[mask], score, _desc(fn, out, "out", dev), _address(lse), _stream_ptr(stream)))
        return out


def _empty_like(t, stream):
    """A buffer for a call to write, of the pool of the stream that it runs on."""
    torch = _torch()
    if stream is None:
        return torch.empty_like(t)
    with torch.cuda.stream(stream):
        return torch.empty_like(t)


def _empty(shape, dtype, device, stream):
    torch = _torch()
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _desc(fn, t, name, device) -> SiftTensor:
    if getattr(t, "device", None) != device:
        raise SiftError(fn, 7, f"{name} is not on {device}")
    return tensor_desc(t)


def _address(t):
    return None if t is None else t.data_ptr()


def score_struct(fn, scale, cap, slopes, num_q_heads, device) -> SiftScore:
    """The score transform's arguments, its slopes checked."""
    if slopes is not None:
        require(fn, slopes, "slopes", "float32", num_q_heads, device)
    return SiftScore(0.0 if scale is None else scale, cap, 0 if slopes is None else slopes.data_ptr())


def sparse_prefill(q, k, v, seg_offsets, prompt_seg_ptr, la, ca, tile=64, out=None, stream=None):
    """One-shot sift_sparse_prefill: stream-ordered scratch, decode and attention
    enqueued on the stream; returns without waiting."""
    torch = _torch()
    _check_bits("sift_sparse_prefill", q, la, ca, seg_offsets, prompt_seg_ptr, tile)
    if out is None:
        out = torch.empty_like(q)
    lay, keep = layout_struct(seg_offsets, prompt_seg_ptr)
    qd, kd, vd, od = tensor_desc(q), tensor_desc(k), tensor_desc(v), tensor_desc(out)
    check("sift_sparse_prefill", lib().sift_sparse_prefill(
        ctypes.byref(qd), ctypes.byref(kd), ctypes.byref(vd), ctypes.byref(lay), _ptr(la), _ptr(ca),
        tile, ctypes.byref(od), _stream_ptr(stream)))
    return out


def _check_bits(fn, q, la, ca, seg_offsets, prompt_seg_ptr, tile):
    """The bit-vector buffers of a one-shot call, against the layout's sizes."""
    if not getattr(q, "is_cuda", False):
        raise SiftError(fn, 4, "q must be a GPU tensor")
    la_n, ca_n = bitmap_bytes(seg_offsets, prompt_seg_ptr, q.shape[1], tile)
    require(fn, la, "local_bitmap", "uint8", la_n, q.device)
    require(fn, ca, "cross_bitmap", "uint8", ca_n, q.device)


def workspace_bytes(seg_offsets, prompt_seg_ptr, num_q_heads, num_kv_heads, head_dim, tile=64):
    """Device workspace bytes of sparse_prefill_ex (sift_workspace_bytes)."""
    lay, keep = layout_struct(seg_offsets, prompt_seg_ptr)
    n = ctypes.c_size_t()
    check("sift_workspace_bytes", lib().sift_workspace_bytes(
        ctypes.byref(lay), num_q_heads, num_kv_heads, head_dim, tile, ctypes.byref(n)))
    return n.value


def sparse_prefill_ex(q, k, v, seg_offsets, prompt_seg_ptr, la, ca, tile=64, scale=None,
                      workspace=None, out=None, stream=None):
    """One-shot form with the caller's scale and workspace (sift_sparse_prefill_ex):
    no device allocation in the library; returns once the work is enqueued.
    workspace: a uint8 device tensor of at least workspace_bytes(...) bytes
    (allocated here when None)."""
    torch = _torch()
    _check_bits("sift_sparse_prefill_ex", q, la, ca, seg_offsets, prompt_seg_ptr, tile)
    if out is None:
        out = torch.empty_like(q)
    n = workspace_bytes(seg_offsets, prompt_seg_ptr, q.shape[1], k.shape[1], q.shape[2], tile)
    if workspace is None:
        workspace = torch.empty(max(n, 1), dtype=torch.uint8, device=q.device)
    require("sift_sparse_prefill_ex", workspace, "workspace", "uint8", n, q.device)
    lay, keep = layout_struct(seg_offsets, prompt_seg_ptr)
    qd, kd, vd, od = tensor_desc(q), tensor_desc(k), tensor_desc(v), tensor_desc(out)
    check("sift_sparse_prefill_ex", lib().sift_sparse_prefill_ex(
        ctypes.byref(qd), ctypes.byref(kd), ctypes.byref(vd), ctypes.byref(lay), _ptr(la), _ptr(ca),
        tile, ctypes.c_float(0.0 if scale is None else scale), _ptr(workspace),
        workspace.numel() * workspace.element_size(), ctypes.byref(od), _stream_ptr(stream)))
    return out


def sparse_prefill_static(q, k, v, seg_offsets, prompt_seg_ptr, la, ca, tile=64, scale=None,
                          out=None, stream=None):
    """The one-shot form on the library's static device scratch
    (sift_sparse_prefill_static): nothing is allocated on the device; calls
    on one GPU must not overlap."""
    torch = _torch()
    _check_bits("sift_sparse_prefill_static", q, la, ca, seg_offsets, prompt_seg_ptr, tile)
    if out is None:
        out = torch.empty_like(q)
    lay, keep = layout_struct(seg_offsets, prompt_seg_ptr)
    qd, kd, vd, od = tensor_desc(q), tensor_desc(k), tensor_desc(v), tensor_desc(out)
    check("sift_sparse_prefill_static", lib().sift_sparse_prefill_static(
        ctypes.byref(qd), ctypes.byref(kd), ctypes.byref(vd), ctypes.byref(lay), _ptr(la), _ptr(ca),
        tile, ctypes.c_float(0.0 if scale is None else scale), ctypes.byref(od),
        _stream_ptr(stream)))
    return out


def static_scratch_bytes() -> int:
    """Bytes of the static scratch of sparse_prefill_static (per GPU)."""
    return int(lib().sift_static_scratch_bytes())


def decode_workspace_bytes(seg_offsets, prompt_seg_ptr, num_q_heads, tile=64):
    """Device workspace bytes of decode_tiles (sift_decode_workspace_bytes)."""
    lay, keep = layout_struct(seg_offsets, prompt_seg_ptr)
    n = ctypes.c_size_t()
    check("sift_decode_workspace_bytes", lib().sift_decode_workspace_bytes(
        ctypes.byref(lay), num_q_heads, tile, ctypes.byref(n)))
    return n.value


def list_capacity(seg_offsets, prompt_seg_ptr, num_q_heads, tile=64):
    """Hq x (causal tiles of all prompts): the col_idx size that bounds any
    decode of this layout."""
    so = np.asarray(seg_offsets, dtype=np.int64)
    ps = np.asarray(prompt_seg_ptr, dtype=np.int64)
    total = 0
    for b in range(len(ps) - 1):
        before = 0
        for s in range(int(ps[b]), int(ps[b + 1])):
            P = -(-int(so[s + 1] - so[s]) // tile)
            total += P * before + P * (P + 1) // 2
            before += P
    return num_q_heads * total


def decode_tiles(seg_offsets, prompt_seg_ptr, la, ca, num_q_heads, tile=64, row_ptr=None,
                 col_idx=None, workspace=None, stream=None):
    """Decoded lists without a plan (sift_decode_tiles): (row_ptr, col_idx)
    device int32 tensors; workspace is allocated here when None."""
    torch = _torch()
    fn = "sift_decode_tiles"
    dev = la.device if la is not None else ca.device
    la_n, ca_n = bitmap_bytes(seg_offsets, prompt_seg_ptr, num_q_heads, tile)
    require(fn, la, "local_bitmap", "uint8", la_n)
    require(fn, ca, "cross_bitmap", "uint8", ca_n)
    M = sum(-(-int(seg_offsets[s + 1] - seg_offsets[s]) // tile)
            for s in range(len(seg_offsets) - 1))
    cap = list_capacity(seg_offsets, prompt_seg_ptr, num_q_heads, tile)
    if row_ptr is None:
        row_ptr = torch.empty(num_q_heads * M + 1, dtype=torch.int32, device=dev)
    if col_idx is None:
        col_idx = torch.empty(max(1, cap), dtype=torch.int32, device=dev)
    n = decode_workspace_bytes(seg_offsets, prompt_seg_ptr, num_q_heads, tile)
    if workspace is None:
        workspace = torch.empty(max(n, 1), dtype=torch.uint8, device=dev)
    require(fn, row_ptr, "row_ptr", "int32", num_q_heads * M + 1, dev)
    require(fn, col_idx, "col_idx", "int32", cap, dev)
    require(fn, workspace, "workspace", "uint8", n, dev)
    lay, keep = layout_struct(seg_offsets, prompt_seg_ptr)
    check(fn, lib().sift_decode_tiles(ctypes.byref(lay), _ptr(la), _ptr(ca), tile, num_q_heads,
                                      _ptr(row_ptr), _ptr(col_idx), col_idx.numel(),
                                      _ptr(workspace), workspace.numel(), _stream_ptr(stream)))
    return row_ptr, col_idx


def extract_sizes(doc_offsets, num_q_heads, tile):
    """(LA bytes, CA bytes, workspace bytes) of sift_extract_bits."""
    import numpy as np
    offs = np.ascontiguousarray(np.asarray(doc_offsets, dtype=np.int32))
    la, ca, ws = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    check("sift_extract_sizes", lib().sift_extract_sizes(
        len(offs) - 1, offs.ctypes.data_as(_P), num_q_heads, tile, ctypes.byref(la), ctypes.byref(ca),
        ctypes.byref(ws)))
    return la.value, ca.value, ws.value


def extract_bits(q, k, doc_offsets, tile=64, alpha=0.001, beta=0.01, gamma=0.1, scale=None,
                 workspace=None, stream=None):
    """Offline metadata of documents prefilled alone (sift_extract_bits).

    q [tokens, Hq, D] and k [tokens, Hkv, D] are bf16 on the GPU; doc_offsets
    (host, [N+1]) delimit the documents.  Returns (la, ca) uint8 device
    tensors in the layout the online path reads."""
    import numpy as np
    torch = _torch()
    offs = np.ascontiguousarray(np.asarray(doc_offsets, dtype=np.int32))
    la_n, ca_n, ws_n = extract_sizes(offs, q.shape[1], tile)
    la = torch.empty(max(la_n, 1), dtype=torch.uint8, device=q.device)
    ca = torch.empty(max(ca_n, 1), dtype=torch.uint8, device=q.device)
    if workspace is None or workspace.numel() < ws_n:
        workspace = torch.empty(max(ws_n, 1), dtype=torch.uint8, device=q.device)
    qd, kd = tensor_desc(q), tensor_desc(k)
    require("sift_extract_bits", workspace, "workspace", "uint8", ws_n, q.device)
    check("sift_extract_bits", lib().sift_extract_bits(
        ctypes.byref(qd), ctypes.byref(kd), len(offs) - 1, offs.ctypes.data_as(_P), tile,
        float(alpha), float(beta), float(gamma), ctypes.c_float(0.0 if scale is None else scale),
        _ptr(la), _ptr(ca), _ptr(workspace), workspace.numel(), _stream_ptr(stream)))
    return la[:la_n], ca[:ca_n]


def rope_(q, k, positions, inv_freq, stream=None):
    """In-place rotary embedding of bf16 q and k (sift_rope)."""
    qd, kd = tensor_desc(q), tensor_desc(k)
    require("sift_rope", positions, "positions", "int32", q.shape[0], q.device)
    require("sift_rope", inv_freq, "inv_freq", "float32", q.shape[2] // 2, q.device)
    check("sift_rope", lib().sift_rope(ctypes.byref(qd), ctypes.byref(kd), _ptr(positions),
                                       _ptr(inv_freq), _stream_ptr(stream)))
    return q, k


def _plain(*ts) -> bool:
    """Whether the library can take these tensors as they are, in place of
    framework operations on them: bf16, contiguous, 16-byte aligned, on one
    GPU, and nothing recorded or transformed (autograd, forward mode,
    tracing, tensor subclasses)."""
    torch = _torch()
    # the dual level is no public name: where it is missing a level may be open
    level = getattr(torch.autograd.forward_ad, "_current_level", 0)
    if torch.jit.is_tracing() or level >= 0:
        return False
    grad = torch.is_grad_enabled()
    return all(type(t) in (torch.Tensor, torch.nn.Parameter) and t.is_cuda
               and t.device == ts[0].device and t.dtype == torch.bfloat16 and t.is_contiguous()
               and not (grad and t.requires_grad) and t.data_ptr() % 16 == 0 for t in ts)


def rms_norm(x, weight, eps: float, stream=None):
    """RMSNorm of the rows of x [rows, width] (sift_layer_rms_norm).  None when
    the library does not take these tensors."""
    torch = _torch()
    if not (_plain(x, weight) and x.dim() == 2 and weight.shape == x.shape[1:]
            and 8 <= x.shape[1] <= 16384 and x.shape[1] % 8 == 0 and x.shape[0] < 1 << 24
            and x.device.index == torch.cuda.current_device()):
        return None
    out = torch.empty_like(x)
    check("sift_layer_rms_norm", lib().sift_layer_rms_norm(
        _ptr(x), _ptr(weight), x.shape[0], x.shape[1], ctypes.c_float(eps), _ptr(out),
        _stream_ptr(stream)))
    return out


def silu_mul(gate, up, stream=None):
    """silu(gate) * up (sift_layer_silu_mul), in gate's memory.  None when the
    library does not take these tensors."""
    torch = _torch()
    if not (_plain(gate, up) and gate.shape == up.shape and gate.numel() % 8 == 0
            and gate.device.index == torch.cuda.current_device()):
        return None
    check("sift_layer_silu_mul", lib().sift_layer_silu_mul(
        _ptr(gate), _ptr(up), gate.numel(), _ptr(gate), _stream_ptr(stream)))
    return gate


def default_scale(head_dim: int) -> float:
    return 1.0 / math.sqrt(head_dim)


class CachePages:
    """The page pools and tables of a batch's caches (sift_cache_kv): k_pages and
    v_pages [num_pages * page, Hkv, D], page_table int32 [seqs, max_pages], lens
    int32 [seqs]; page_lens int32 [seqs, max_pages] where pages end early, key_pos
    int32 [seqs, Hkv, max_pages * page] where a key's position is not its slot.
    The tensors are used where they are: write into them, or make another."""

    def __init__(self, k_pages, v_pages, page_table, lens, page_lens=None, key_pos=None):
        fn = "CachePages"
        kd, vd = tensor_desc(k_pages), tensor_desc(v_pages)
        dev = k_pages.device
        for name, t in (("page_table", page_table), ("lens", lens), ("page_lens", page_lens),
                        ("key_pos", key_pos)):
            if t is not None or name in ("page_table", "lens"):
                require(fn, t, name, "int32", 1, dev)
        if v_pages.device != dev:
            raise SiftError(fn, 7, f"v_pages is on {v_pages.device}, k_pages on {dev}")
        self.k_pages, self.v_pages, self.page_table, self.lens = k_pages, v_pages, page_table, lens
        self.page_lens, self.key_pos = page_lens, key_pos
        self._held = (k_pages, v_pages, page_table, lens, page_lens, key_pos, kd, vd)
        self.sizes = (dev, *(None if t is None else (t.numel(), t.shape)
                             for t in (page_table, lens, page_lens, key_pos)))
        self.struct = SiftCacheKv(ctypes.pointer(kd), ctypes.pointer(vd), page_table.data_ptr(),
                                  lens.data_ptr(), 0 if page_lens is None else page_lens.data_ptr(),
                                  0 if key_pos is None else key_pos.data_ptr())


class Cache:
    """A handle for the paged caches of a batch (sift_cache_*): sizes and scratch."""

    def __init__(self, num_seqs, num_q_heads, num_kv_heads, head_dim, page=64, max_pages=1,
                 max_rows=1):
        self._h = None
        h = ctypes.c_void_p()
        check("sift_cache_create", lib().sift_cache_create(
            num_seqs, num_q_heads, num_kv_heads, head_dim, page, max_pages, max_rows,
            ctypes.byref(h)))
        self._h = h
        torch = _torch()
        self.device = torch.device("cuda", torch.cuda.current_device())
        self.num_seqs, self.hq, self.hkv, self.d = num_seqs, num_q_heads, num_kv_heads, head_dim
        self.page, self.max_pages, self.max_rows = page, max_pages, max_rows
        self.slots = max_pages * page
        self._slot_sizes = (num_seqs, num_kv_heads, self.slots)
        sizes = (("page_table", (num_seqs, max_pages)), ("lens", (num_seqs,)),
                 ("page_lens", (num_seqs, max_pages)), ("key_pos", self._slot_sizes))
        self._tables = tuple((name, math.prod(x), x) for name, x in sizes)

    def close(self):
        if self._h is not None:
            check("sift_cache_destroy", lib().sift_cache_destroy(self._h))
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def _kv(self, fn, kv):
        """The tables' sizes, which the library cannot see."""
        device, *have = kv.sizes
        if device != self.device:
            raise SiftError(fn, 7, f"the pages are on {device}, the cache on {self.device}")
        for t, (name, n, sizes) in zip(have, self._tables):
            if t is None or t[0] == n:
                continue
            if t[0] < n:
                raise SiftError(fn, 5, f"{name} holds {t[0]} elements, needs {n}")
            check_laid_out(fn, name, t[1], sizes)
        return kv.struct

    def _rows(self, fn, q, row_ptr, row_pos):
        if row_ptr is not None:
            require(fn, row_ptr, "row_ptr", "int32", self.num_seqs + 1, self.device)
        if row_pos is not None:
            require(fn, row_pos, "row_pos", "int32", q.shape[0], self.device)
        return SiftCacheRows(0 if row_ptr is None else row_ptr.data_ptr(),
                             0 if row_pos is None else row_pos.data_ptr())

    def attention(self, q, k_new, v_new, kv, row_ptr=None, tree_mask=None, row_pos=None, scale=None,
                  cap=0.0, slopes=None, out=None, lse=None, stream=None):
        """Attention of new tokens over the cache and each other
        (sift_cache_attention): q [rows, Hq, D], k_new and v_new [rows, Hkv, D], kv a
        CachePages.  row_ptr int32 [seqs + 1] delimits the sequences' rows (None: as
        many of each); tree_mask int64 [rows, words] holds each row's visible new
        tokens as bits (None: those up to itself); row_pos int32 [rows].  lse: float32
        [rows, Hq] buffer that receives the rows' log sum exp."""
        fn = "sift_cache_attention"
        rows = self._rows(fn, q, row_ptr, row_pos)
        words = 0
        if tree_mask is not None:
            words = (self.max_rows + 63) // 64
            if tree_mask.dim() == 2:
                words = max(words, tree_mask.shape[1])
            require(fn, tree_mask, "tree_mask", "int64", q.shape[0] * words, self.device)
        score = score_struct(fn, scale, cap, slopes, self.hq, self.device)
        if lse is not None:
            require_laid_out(fn, lse, "lse", "float32", (q.shape[0], self.hq), self.device)
        if out is None:
            out = _empty_like(q, stream)
        dev = self.device
        check(fn, lib().sift_cache_attention(
            self._h, self._kv(fn, kv), rows, _desc(fn, q, "q", dev), _desc(fn, k_new, "k_new", dev),
            _desc(fn, v_new, "v_new", dev), _address(tree_mask), words, score,
            _desc(fn, out, "out", dev), _address(lse), _stream_ptr(stream)))
        return out

    def _slot_buffer(self, fn, t, name, dtype="float32"):
        require_laid_out(fn, t, name, dtype, self._slot_sizes, self.device)

    def accumulate(self, q, lse, kv, weights=None, decay=1.0, row_ptr=None, row_pos=None,
                   row_weight=None, scale=None, cap=0.0, slopes=None, out=None, stream=None):
        """decay * weights plus the attention weight that the new tokens q give to each
        cached key (sift_cache_accumulate): weights and out float32 [seqs, Hkv,
        max_pages * page] (weights None: zeros), lse as the attention left it.
        row_weight float32 [rows] scales a token's part, 0 leaves it out.  out: the
        weights themselves when None (a new buffer where there are none)."""
        torch = _torch()
        fn = "sift_cache_accumulate"
        rows = self._rows(fn, q, row_ptr, row_pos)
        require_laid_out(fn, lse, "lse", "float32", (q.shape[0], self.hq), self.device)
        if row_weight is not None:
            require(fn, row_weight, "row_weight", "float32", q.shape[0], self.device)
        if weights is not None:
            self._slot_buffer(fn, weights, "weights")
        if out is None:
            out = weights
        if out is None:
            out = _empty((self.num_seqs, self.hkv, self.slots), torch.float32, self.device, stream)
            with torch.cuda.stream(stream):  # (None: the current one)
                out.zero_()
        self._slot_buffer(fn, out, "out")
        score = score_struct(fn, scale, cap, slopes, self.hq, self.device)
        check(fn, lib().sift_cache_accumulate(
            self._h, self._kv(fn, kv), rows, _desc(fn, q, "q", self.device), _address(lse),
            _address(row_weight), score, _address(weights), decay, _address(out),
            _stream_ptr(stream)))
        return out

    def evict(self, kv, weights, budget, sinks=0, recent=0, next_pos=None, weights_out=None,
              pos_out=None, lens_out=None, stream=None):
        """Keeps `budget` keys of every (sequence, kv head), those of the largest weights
        beside the protected first `sinks` and last `recent` positions, in its first slots
        (sift_cache_evict; K and V move in place).  Returns (weights, key_pos, lens) of
        the cache as it is then: a CachePages of them has no page_lens."""
        torch = _torch()
        fn = "sift_cache_evict"
        self._slot_buffer(fn, weights, "weights")
        if next_pos is not None:
            require(fn, next_pos, "next_pos", "int32", self.num_seqs, self.device)
        shape = (self.num_seqs, self.hkv, self.slots)
        if weights_out is None:
            weights_out = _empty(shape, torch.float32, self.device, stream)
        else:
            self._slot_buffer(fn, weights_out, "weights_out")
        if pos_out is None:
            pos_out = _empty(shape, torch.int32, self.device, stream)
        else:
            self._slot_buffer(fn, pos_out, "pos_out", "int32")
        if lens_out is None:
            lens_out = _empty((self.num_seqs,), torch.int32, self.device, stream)
        else:
            require(fn, lens_out, "lens_out", "int32", self.num_seqs, self.device)
        check(fn, lib().sift_cache_evict(
            self._h, self._kv(fn, kv), _address(weights), _address(next_pos), budget, sinks, recent,
            _address(weights_out), _address(pos_out), _address(lens_out), _stream_ptr(stream)))
        return weights_out, pos_out, lens_out
