"""Thin ctypes binding of the C ABI in ``include/dam.h``.

Argument marshalling only: every step of the path runs inside the CUDA library.  PyTorch is used for
device memory and streams.  There is no CPU fallback: if ``libdam_b200.so`` is missing or a call
fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import List, Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdam_b200.so")

DAM_BF16, DAM_F32 = 0, 1
STATUS = {0: "DAM_OK", 1: "DAM_ERR_INVALID_ARGUMENT", 2: "DAM_ERR_UNSUPPORTED", 3: "DAM_ERR_BUFFER_TOO_SMALL",
          4: "DAM_ERR_CUDA", 5: "DAM_ERR_DEVICE_TIMEOUT", 6: "DAM_ERR_INTERNAL"}

EXPORTS = ["dam_version", "dam_status_string", "dam_mask_sizes", "dam_build_masks", "dam_build_masks_from_scores",
           "dam_mask_all_ones", "dam_sparse_attention", "dam_mask_stats", "dam_mask_expand_rows", "dam_poll_status",
           "dam_prefill_host", "dam_build_masks_static", "dam_static_scratch_bytes", "dam_selftest_bounded_wait",
           "dam_decode_attention", "dam_sparse_attention_rows", "dam_capture_accumulate", "dam_capture_average",
           "dam_selftest_device_table", "dam_cache_sizes", "dam_cache_write", "dam_cache_read", "dam_cache_decode_attention"]


class DamError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {STATUS.get(code, code)}")


class dam_shape_t(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("num_seqs", ctypes.c_int32),
                ("cu_seqlens_host", ctypes.c_void_p), ("cu_seqlens_dev", ctypes.c_void_p),
                ("total_tokens", ctypes.c_int32), ("max_seqlen", ctypes.c_int32),
                ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("q_stride_tok", ctypes.c_int64), ("q_stride_head", ctypes.c_int64),
                ("k_stride_tok", ctypes.c_int64), ("k_stride_head", ctypes.c_int64),
                ("v_stride_tok", ctypes.c_int64), ("v_stride_head", ctypes.c_int64),
                ("o_stride_tok", ctypes.c_int64), ("o_stride_head", ctypes.c_int64)]


class dam_cache_t(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("num_seqs", ctypes.c_int32),
                ("cu_seqlens_host", ctypes.c_void_p), ("cu_seqlens_dev", ctypes.c_void_p),
                ("total_tokens", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("code", ctypes.c_int32), ("block_tokens", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("k_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p),
                ("k_stride_tok", ctypes.c_int64), ("k_stride_head", ctypes.c_int64),
                ("v_stride_tok", ctypes.c_int64), ("v_stride_head", ctypes.c_int64)]


class dam_rule_t(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("pcl_max", ctypes.c_int32), ("tau", ctypes.c_float),
                ("mu", ctypes.c_float), ("lambda_", ctypes.c_float), ("eps", ctypes.c_float),
                ("softmax_scale", ctypes.c_float), ("min_support", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("transform", ctypes.c_int32)]


TRANSFORMS = {"boxcox": 0, "log": 1, "sqrt": 2, "arcsinh": 3, "yeo_johnson": 4, "average": 5, "zscore": 6, "minmax": 7, "sum": 8}


# argument types, one letter each: p pointer, z size_t, i int32, u uint32, f float.  With them ctypes converts the plain
# integers that data_ptr() and numel() return by itself; an object made here for every argument is most of what a call
# costs on the host (a generation step for one sequence is bound by that: 9.8 us to issue, 6 with plain integers).
_ARGS = {"dam_status_string": "i", "dam_mask_sizes": "ppippp", "dam_build_masks": "pppppzpzpp",
         "dam_build_masks_from_scores": "ppppzpzp", "dam_mask_all_ones": "pipzp", "dam_sparse_attention": "pppppiifpppzp",
         "dam_mask_stats": "ppppp", "dam_mask_expand_rows": "ppiiiiipp", "dam_poll_status": "pp",
         "dam_prefill_host": "pppppippppp", "dam_build_masks_static": "pppppzp", "dam_selftest_bounded_wait": "pzup",
         "dam_decode_attention": "ppppppifpppzp", "dam_sparse_attention_rows": "pppppiifpppppzp",
         "dam_capture_accumulate": "ppippp", "dam_capture_average": "ppifppp", "dam_selftest_device_table": "pipp",
         "dam_cache_sizes": "pipp", "dam_cache_write": "pppppppp", "dam_cache_read": "pppppppp",
         "dam_cache_decode_attention": "ppppiifppppp"}
_CTYPE = {"p": ctypes.c_void_p, "z": ctypes.c_size_t, "i": ctypes.c_int32, "u": ctypes.c_uint32, "f": ctypes.c_float}

_lib = None


def _declare(so):
    for name in EXPORTS:
        fn = getattr(so, name)
        fn.restype = ctypes.c_int
        fn.argtypes = [_CTYPE[a] for a in _ARGS.get(name, "")]
    so.dam_status_string.restype = ctypes.c_char_p
    so.dam_static_scratch_bytes.restype = ctypes.c_size_t
    return so


def lib():
    """The loaded shared library; raises if it was not built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2506_11104_b200.build` "
                               "(there is no fallback path)")
        _lib = _declare(ctypes.CDLL(LIB_PATH))
    return _lib


def _check(code: int, where: str):
    if code != 0:
        raise DamError(code, where)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


# the handle without the Stream object that torch.cuda.current_stream makes (0.1 us instead of 2.3), where torch has it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
# indices of the CUDA devices asked for so far (device.type makes a string by way of a C++ stream: 4 us of a first pass)
_cuda_index = {}


def _stream(device) -> int:
    """Handle of the device's current stream; ValueError for a device that is not a GPU (every entry point asks for the
    stream of its first tensor's device: host memory never reaches a kernel by that argument)."""
    index = _cuda_index.get(device)
    if index is None:
        d = torch.device(device) if isinstance(device, str) else device
        if isinstance(d, torch.device) and d.type != "cuda":
            raise ValueError(f"expected tensors on a CUDA device, got {d}")
        if not isinstance(d, torch.device) or d.index is None or _raw_stream is None:
            return torch.cuda.current_stream(device).cuda_stream
        index = _cuda_index[device] = d.index
    return _raw_stream(index)


# the same for the index of a CUDA device
_index_stream = _raw_stream if _raw_stream is not None else lambda index: torch.cuda.current_stream(index).cuda_stream


class _ByReference:
    """`ref` is the reference to the structure `c`, made when c is set (every call passes it; byref takes as long as a check), and
    `address` its address; `index`: the CUDA device that cu_dev is on, -1 for none."""

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        if name == "c":
            object.__setattr__(self, "ref", ctypes.byref(value))
            object.__setattr__(self, "address", ctypes.addressof(value))
        elif name == "cu_dev":
            object.__setattr__(self, "index", -1 if value is None else value.get_device())


@dataclass
class Shape(_ByReference):
    """Python-side owner of a dam_shape_t and the cu_seqlens buffers it points to."""
    c: dam_shape_t
    cu_host: np.ndarray
    cu_dev: Optional[torch.Tensor]
    lengths: List[int]
    kv = None                    # what the K and V rows look like to torch, see _kv_rows

    def __setattr__(self, name, value):
        super().__setattr__(name, value)
        if name == "c":
            self.kv = _kv_rows(value)


_BF16, _F32, _I32 = torch.bfloat16, torch.float32, torch.int32


def _kv_rows(s: dam_shape_t):
    """(shape of the K and V rows, dtype, whether there are no gaps in them, strides of K, of V)"""
    rows = T, H, d = (s.total_tokens, s.num_kv_heads, s.head_dim)
    ks, vs = (s.k_stride_tok, s.k_stride_head, 1), (s.v_stride_tok, s.v_stride_head, 1)
    return rows, _BF16 if s.dtype == DAM_BF16 else _F32, ks == vs == (H * d, d, 1), ks, vs


def make_shape(cu_seqlens: Sequence[int], Hq: int, Hkv: int, d: int, dtype: torch.dtype, device=None,
               q_strides=None, k_strides=None, v_strides=None, o_strides=None) -> Shape:
    cu_host = np.ascontiguousarray(cu_seqlens, dtype=np.int32)
    cu_dev = torch.from_numpy(cu_host.copy()).to(device) if device is not None else None
    lengths = [int(b - a) for a, b in zip(cu_host[:-1], cu_host[1:])]
    s = dam_shape_t()
    s.struct_size = ctypes.sizeof(dam_shape_t)
    s.num_seqs = len(lengths)
    s.cu_seqlens_host = cu_host.ctypes.data
    s.cu_seqlens_dev = cu_dev.data_ptr() if cu_dev is not None else 1   # non-null placeholder for host-only calls
    s.total_tokens = int(cu_host[-1])
    s.max_seqlen = max(lengths) if lengths else 0
    s.num_q_heads, s.num_kv_heads, s.head_dim = Hq, Hkv, d
    s.dtype = DAM_BF16 if dtype == torch.bfloat16 else DAM_F32
    qs = q_strides or (Hq * d, d)
    ks = k_strides or (Hkv * d, d)
    vs = v_strides or (Hkv * d, d)
    os_ = o_strides or (Hq * d, d)
    s.q_stride_tok, s.q_stride_head = qs
    s.k_stride_tok, s.k_stride_head = ks
    s.v_stride_tok, s.v_stride_head = vs
    s.o_stride_tok, s.o_stride_head = os_
    return Shape(c=s, cu_host=cu_host, cu_dev=cu_dev, lengths=lengths)


DAM_RULE_GATHER_COLUMNS = 1
DAM_ROW_RANGES_BY_VALUE = 16


def make_rule(pcl_max: int, tau: float, mu: float, lam: float = 0.5, eps: float = 1e-8,
              softmax_scale: float = 0.0, min_support: int = 1, gather_columns: bool = False,
              transform: str = "boxcox") -> dam_rule_t:
    r = dam_rule_t()
    r.struct_size = ctypes.sizeof(dam_rule_t)
    r.pcl_max, r.tau, r.mu, r.lambda_, r.eps = pcl_max, tau, mu, lam, eps
    r.softmax_scale, r.min_support, r.flags = softmax_scale, min_support, (DAM_RULE_GATHER_COLUMNS if gather_columns else 0)
    r.transform = TRANSFORMS[transform]
    return r


def dam_version() -> int:
    return int(lib().dam_version())


def dam_status_string(code: int) -> str:
    return lib().dam_status_string(code).decode()


def dam_mask_sizes(shape: Shape, rule: Optional[dam_rule_t], causal: bool = True):
    m, b, a = ctypes.c_size_t(0), ctypes.c_size_t(0), ctypes.c_size_t(0)
    rc = lib().dam_mask_sizes(shape.ref, ctypes.byref(rule) if rule is not None else None, int(causal),
                              ctypes.byref(m), ctypes.byref(b), ctypes.byref(a))
    _check(rc, "dam_mask_sizes")
    return m.value, b.value, a.value


def _alloc(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(256, nbytes), dtype=torch.uint8, device=device)


def dam_build_masks(Q: torch.Tensor, K: torch.Tensor, shape: Shape, rule: dam_rule_t, mask: Optional[torch.Tensor] = None,
                    scratch: Optional[torch.Tensor] = None, scores_dump: Optional[torch.Tensor] = None):
    """Enqueues stage 1 on the current stream.  Returns (mask blob, scratch)."""
    if mask is None or scratch is None:
        mb, sb, _ = dam_mask_sizes(shape, rule)
        mask = mask if mask is not None else _alloc(mb, Q.device)
        scratch = scratch if scratch is not None else _alloc(sb, Q.device)
    rc = lib().dam_build_masks(_ptr(Q), _ptr(K), shape.ref, ctypes.byref(rule), _ptr(mask),
                               mask.numel(), _ptr(scratch), scratch.numel(),
                               _ptr(scores_dump), _stream(Q.device))
    _check(rc, "dam_build_masks")
    return mask, scratch


def dam_build_masks_static(Q: torch.Tensor, K: torch.Tensor, shape: Shape, rule: dam_rule_t, mask: torch.Tensor):
    """Stage 1 with the library's built-in scratch: for callers that cannot allocate device memory.
    `mask` must already exist (size from dam_mask_sizes); nothing is allocated here or in the library."""
    rc = lib().dam_build_masks_static(_ptr(Q), _ptr(K), shape.ref, ctypes.byref(rule), _ptr(mask),
                                      mask.numel(), _stream(Q.device))
    _check(rc, "dam_build_masks_static")
    return mask


def dam_static_scratch_bytes() -> int:
    return int(lib().dam_static_scratch_bytes())


def dam_build_masks_from_scores(P: torch.Tensor, shape: Shape, rule: dam_rule_t, mask: Optional[torch.Tensor] = None,
                                scratch: Optional[torch.Tensor] = None):
    if mask is None or scratch is None:
        mb, sb, _ = dam_mask_sizes(shape, rule)
        mask = mask if mask is not None else _alloc(mb, P.device)
        scratch = scratch if scratch is not None else _alloc(sb, P.device)
    rc = lib().dam_build_masks_from_scores(_ptr(P), shape.ref, ctypes.byref(rule), _ptr(mask),
                                           mask.numel(), _ptr(scratch),
                                           scratch.numel(), _stream(P.device))
    _check(rc, "dam_build_masks_from_scores")
    return mask, scratch


def dam_mask_all_ones(shape: Shape, causal: bool, device, mask: Optional[torch.Tensor] = None) -> torch.Tensor:
    if mask is None:
        mb, _, _ = dam_mask_sizes(shape, None, causal)
        mask = _alloc(mb, device)
    rc = lib().dam_mask_all_ones(shape.ref, int(causal), _ptr(mask), mask.numel(), _stream(device))
    _check(rc, "dam_mask_all_ones")
    return mask


def dam_sparse_attention(Q, K, V, mask, shape: Shape, causal: bool = True, softmax_scale: float = 0.0,
                         O: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                         scratch: Optional[torch.Tensor] = None):
    """Enqueues stage 2 on the current stream.  Returns (O, LSE [Hq, T] fp32, scratch)."""
    if O is None:
        O = torch.empty_like(Q)
    if lse is None:
        lse = torch.empty(shape.c.num_q_heads, shape.c.total_tokens, dtype=torch.float32, device=Q.device)
    if scratch is None:
        # a blob with gathered-column tiles records the scratch size it needs in its header
        off = _HDR.fields["attn_scratch_bytes"][1]
        need = int(mask[off: off + 8].cpu().numpy().view(np.uint64)[0]) if mask.numel() >= 256 else 256
        scratch = _alloc(max(256, need), Q.device)
    rc = lib().dam_sparse_attention(_ptr(Q), _ptr(K), _ptr(V), _ptr(mask), shape.ref, int(causal),
                                    shape.c.num_q_heads // shape.c.num_kv_heads, softmax_scale,
                                    _ptr(O), _ptr(lse), _ptr(scratch), scratch.numel(),
                                    _stream(Q.device))
    _check(rc, "dam_sparse_attention")
    return O, lse, scratch


def dam_capture_accumulate(P: torch.Tensor, shape: Shape, pcl_max: int, A: torch.Tensor, C: torch.Tensor):
    """A += the window maps of one batch of samples (P: the scores_dump of that batch), C += valid counts per row."""
    Hq = shape.c.num_q_heads
    assert A.dtype == torch.float32 and A.numel() == Hq * pcl_max * pcl_max and A.is_contiguous()
    assert C.dtype == torch.int32 and C.numel() == pcl_max
    assert P.dtype == torch.float32 and P.numel() == sum(Hq * min(S, pcl_max) ** 2 for S in shape.lengths)
    rc = lib().dam_capture_accumulate(_ptr(P), shape.ref, pcl_max, _ptr(A), _ptr(C), _stream(P.device))
    _check(rc, "dam_capture_accumulate")


def dam_capture_average(A: torch.Tensor, C: torch.Tensor, pcl_max: int, eps: float, shape: Shape) -> torch.Tensor:
    """Averaged maps for the sequences of `shape`, in the layout dam_build_masks_from_scores reads."""
    n = sum(shape.c.num_q_heads * min(S, pcl_max) ** 2 for S in shape.lengths)
    P = torch.empty(n, dtype=torch.float32, device=A.device)
    rc = lib().dam_capture_average(_ptr(A), _ptr(C), pcl_max, eps, shape.ref, _ptr(P),
                                   _stream(A.device))
    _check(rc, "dam_capture_average")
    return P


def dam_sparse_attention_rows(Q, K, V, mask, shape: Shape, row_ranges, O: torch.Tensor, lse: torch.Tensor,
                              causal: bool = True, softmax_scale: float = 0.0,
                              scratch: Optional[torch.Tensor] = None):
    """Chunked prefill: stage 2 for the query rows [begin, end) of every sequence (row_ranges: [(begin, end)] per
    sequence).  O and LSE are updated in place on those rows only.  Returns scratch."""
    flat = [int(x) for pair in row_ranges for x in pair]
    assert len(flat) == 2 * shape.c.num_seqs
    host = (ctypes.c_int32 * len(flat))(*flat)
    # so many sequences' ranges the library hands to the kernel itself; beyond, a copy on the device, queued without
    # waiting for the stream (CUDA has taken its own copy of a small pageable source when the call returns)
    if shape.c.num_seqs <= DAM_ROW_RANGES_BY_VALUE:
        dev = shape.c.cu_seqlens_dev
    else:
        with torch.cuda.device(Q.device):
            if torch.cuda.is_current_stream_capturing():     # (a replay would copy from host memory that is long gone)
                raise RuntimeError("the row ranges of more than %d sequences cannot be captured" % DAM_ROW_RANGES_BY_VALUE)
        dev_copy = torch.tensor(flat, dtype=torch.int32).to(Q.device, non_blocking=True)
        dev = dev_copy.data_ptr()
    if scratch is None:
        off = _HDR.fields["attn_scratch_bytes"][1]
        need = int(mask[off: off + 8].cpu().numpy().view(np.uint64)[0]) if mask.numel() >= 256 else 256
        scratch = _alloc(max(256, need), Q.device)
    rc = lib().dam_sparse_attention_rows(_ptr(Q), _ptr(K), _ptr(V), _ptr(mask), shape.ref, int(causal),
                                         shape.c.num_q_heads // shape.c.num_kv_heads, softmax_scale,
                                         _ptr(O), _ptr(lse), host, dev, _ptr(scratch),
                                         scratch.numel(), _stream(Q.device))
    _check(rc, "dam_sparse_attention_rows")
    return scratch


def dam_decode_attention(q, K, V, mask, shape: Shape, positions: torch.Tensor, softmax_scale: float = 0.0,
                         O: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                         scratch: Optional[torch.Tensor] = None):
    """One new token per sequence against the KV cache `shape` describes (q, O: [B, Hq, d]; positions int32 [B]).

    Returns (O, LSE [B, Hq] fp32, scratch)."""
    B, Hq = shape.c.num_seqs, shape.c.num_q_heads
    assert q.is_contiguous() and q.shape == (B, Hq, shape.c.head_dim)
    assert positions.dtype == torch.int32 and positions.numel() == B and positions.is_contiguous()
    if O is None:
        O = torch.empty_like(q)
    if lse is None:
        lse = torch.empty(B, Hq, dtype=torch.float32, device=q.device)
    if scratch is None:
        scratch = _alloc(256, q.device)
    rc = lib().dam_decode_attention(_ptr(q), _ptr(K), _ptr(V), _ptr(mask), shape.ref, _ptr(positions),
                                    Hq // shape.c.num_kv_heads, softmax_scale, _ptr(O), _ptr(lse),
                                    _ptr(scratch), scratch.numel(), _stream(q.device))
    _check(rc, "dam_decode_attention")
    return O, lse, scratch


CACHE_CODES = {"int8": (0, torch.int8), "e4m3": (1, torch.float8_e4m3fn)}


@dataclass
class Cache(_ByReference):
    """Python-side owner of a dam_cache_t and the buffers it points to."""
    c: dam_cache_t
    cu_host: np.ndarray
    cu_dev: Optional[torch.Tensor]
    lengths: List[int]
    k_codes: Optional[torch.Tensor]
    v_codes: Optional[torch.Tensor]
    k_scales: Optional[torch.Tensor]
    v_scales: Optional[torch.Tensor]
    num_seqs: int                # (as in c; a field of a ctypes structure takes several times as long to read)
    head_dim: int


def make_cache(cu_seqlens: Sequence[int], Hkv: int, d: int, code: str = "int8", block_tokens: int = 64, device=None,
               k_codes: Optional[torch.Tensor] = None, v_codes: Optional[torch.Tensor] = None,
               k_scales: Optional[torch.Tensor] = None, v_scales: Optional[torch.Tensor] = None) -> Cache:
    """A KV cache held in 8 bits, with room for cu_seqlens[b + 1] - cu_seqlens[b] tokens of sequence b.

    Buffers that are not given are allocated on `device` (zeros); codes [tokens, Hkv, d] of one byte, any strides with the
    last dimension contiguous; scales fp32 [rows, Hkv], contiguous; all on `device`.  Without a device: a description for
    host-only calls."""
    cu_host = np.ascontiguousarray(cu_seqlens, dtype=np.int32)
    lengths = [int(b - a) for a, b in zip(cu_host[:-1], cu_host[1:])]
    T, (number, dtype) = int(cu_host[-1]), CACHE_CODES[code]
    c = dam_cache_t()
    c.struct_size = ctypes.sizeof(dam_cache_t)
    c.num_seqs, c.total_tokens, c.num_kv_heads, c.head_dim = len(lengths), T, Hkv, d
    c.code, c.block_tokens = number, block_tokens
    c.cu_seqlens_host = cu_host.ctypes.data
    cu_dev = None
    codes, scales = [k_codes, v_codes], [k_scales, v_scales]
    if device is None:
        c.cu_seqlens_dev = 1                                  # non-null placeholder for host-only calls
    else:
        cu_dev = torch.from_numpy(cu_host.copy()).to(device)
        c.cu_seqlens_dev = cu_dev.data_ptr()
        rows = T // block_tokens + len(lengths)
        codes = [torch.zeros(T, Hkv, d, dtype=dtype, device=device) if x is None else x for x in codes]
        scales = [torch.zeros(rows, Hkv, dtype=torch.float32, device=device) if x is None else x for x in scales]
        for x in codes:
            assert x.element_size() == 1 and x.shape == (T, Hkv, d) and (x.stride(2) == 1 or x.numel() == 0)
        for x in scales:
            assert x.dtype == torch.float32 and x.is_contiguous() and x.numel() >= rows * Hkv
        for x in codes + scales:
            if x.device != cu_dev.device:
                raise ValueError(f"the cache's buffers belong on the device {cu_dev.device}: got a tensor of {x.device}")
        (c.k_codes, c.v_codes), (c.k_scales, c.v_scales) = map(_ptr, codes), map(_ptr, scales)
    (c.k_stride_tok, c.k_stride_head), (c.v_stride_tok, c.v_stride_head) = (
        (Hkv * d, d) if x is None or x.numel() == 0 else (x.stride(0), x.stride(1)) for x in codes)
    return Cache(c, cu_host, cu_dev, lengths, *codes, *scales, len(lengths), d)


def dam_cache_sizes(cache: Cache, Hq: int):
    """(rows of the scales, bytes of dam_cache_decode_attention's scratch)."""
    rows, scratch = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(lib().dam_cache_sizes(cache.ref, Hq, ctypes.byref(rows), ctypes.byref(scratch)), "dam_cache_sizes")
    return rows.value, scratch.value


# The checks of the calls below are written for their usual case, a few attributes each: the host's part of a call is what bounds a
# generation step of few tokens.  (Addresses as numbers, too: ctypes takes longer over a reference or a size_t.)
def _per_sequence(x: torch.Tensor, n: int) -> int:
    """Pointer of an int32 tensor with one element per sequence."""
    assert x.dtype is _I32 and x.numel() == n and x.is_contiguous()
    return x.data_ptr()


def _check_device(index: int, **tensors):
    """ValueError unless all of them (None: not there) are on the CUDA device; Shape and Cache stand for their cu_seqlens."""
    for name, x in tensors.items():
        where = index if x is None else x.index if isinstance(x, _ByReference) else x.get_device()
        if index < 0 or where != index:
            of = f", which is on {x.device}" if isinstance(x, torch.Tensor) else ", which was made for another"
            raise ValueError(f"every tensor of a call belongs on the device it runs on: not so {name}{of}")


def _check_rows(tokens: "Shape", K: torch.Tensor, V: torch.Tensor):
    """ValueError unless the rows that `tokens` describes lie inside K and V where K and V have them: K, V [tokens, heads,
    head_dim] or longer, or [heads, tokens, head_dim], with the strides of `tokens`; or flattened in another way (their last
    element is no further than K's and V's own).  The calls compare the usual case, the very shape, by themselves."""
    tokens.kv = rows, dtype, _, *strides = _kv_rows(tokens.c)
    T, H, d = rows
    for name, x, (st, sh, _) in zip("KV", (K, V), strides):
        if T == 0:
            continue
        if x.dtype is not dtype:
            raise ValueError(f"{name} is of {x.dtype}, its rows are described as {dtype}")
        # (the stride of a dimension that one element is taken from says nothing)
        ok = x.dim() == 3 and any(all(x.shape[k] >= n and (n == 1 or x.stride(k) == w) for k, n, w in zip(order, rows, (st, sh, 1)))
                                  for order in ((0, 1, 2), (1, 0, 2)))
        if x.dim() != 3 or (not ok and x.is_contiguous() and (H == 1 or x.shape[2] != d)):
            last = sum((n - 1) * w for n, w in zip(x.shape, x.stride())) if x.numel() else -1
            ok = (T - 1) * st + (H - 1) * sh + d - 1 <= last
        if not ok:
            raise ValueError(f"{name} of shape {tuple(x.shape)} and strides {x.stride()} does not have the rows that `tokens` "
                             f"describes: {rows}, strides {(st, sh, 1)}")


def dam_cache_write(K: torch.Tensor, V: torch.Tensor, tokens: Shape, cache: Cache, starts: Optional[torch.Tensor] = None,
                    scratch: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Quantises the packed rows K, V (`tokens` says how many each sequence gets) into the cache, from token starts[b] of
    sequence b on (int32 on the device; None: token 0).  Returns scratch.  ValueError for K or V that are not what `tokens`
    describes, and for a tensor on another device than K."""
    at = None if starts is None else _per_sequence(starts, cache.num_seqs)
    index = K.get_device()
    if scratch is None:
        scratch = _alloc(256, K.device)
    rows, dtype, dense, ks, vs = tokens.kv
    if not (K.shape == rows and V.shape == rows and K.dtype is dtype and V.dtype is dtype
            and (K.is_contiguous() and V.is_contiguous() if dense else K.stride() == ks and V.stride() == vs)):
        _check_rows(tokens, K, V)
    if not (V.get_device() == index == scratch.get_device() and tokens.index == index == cache.index >= 0
            and (at is None or starts.get_device() == index)):
        _check_device(index, K=K, V=V, scratch=scratch, tokens=tokens, cache=cache, starts=starts)
    rc = (_lib or lib()).dam_cache_write(K.data_ptr(), V.data_ptr(), tokens.address, at, cache.address, scratch.data_ptr(), scratch.numel(),
                                         _index_stream(index))
    if rc:
        _check(rc, "dam_cache_write")
    return scratch


def dam_cache_read(cache: Cache, tokens: Shape, starts: Optional[torch.Tensor] = None, K: Optional[torch.Tensor] = None,
                   V: Optional[torch.Tensor] = None, scratch: Optional[torch.Tensor] = None):
    """Reads tokens starts[b] ... of every sequence back, as packed rows (`tokens` says how many, of which type and strides).
    Returns (K, V, scratch).  ValueError for K or V that are not what `tokens` describes, and for a tensor on another device
    than the cache."""
    at = None if starts is None else _per_sequence(starts, cache.num_seqs)
    index = cache.index
    if scratch is None:
        scratch = _alloc(256, cache.cu_dev.device)
    if K is None or V is None:
        shape, dtype, _, *strides = _kv_rows(tokens.c)
        rows = [torch.empty_strided(shape, x, device=cache.cu_dev.device, dtype=dtype) for x in strides]
        K, V = K if K is not None else rows[0], V if V is not None else rows[1]
    rows, dtype, dense, ks, vs = tokens.kv
    if not (K.shape == rows and V.shape == rows and K.dtype is dtype and V.dtype is dtype
            and (K.is_contiguous() and V.is_contiguous() if dense else K.stride() == ks and V.stride() == vs)):
        _check_rows(tokens, K, V)
    if not (K.get_device() == V.get_device() == index == scratch.get_device() and tokens.index == index >= 0
            and (at is None or starts.get_device() == index)):
        _check_device(index, K=K, V=V, scratch=scratch, tokens=tokens, starts=starts)
    rc = (_lib or lib()).dam_cache_read(cache.address, tokens.address, at, K.data_ptr(), V.data_ptr(), scratch.data_ptr(), scratch.numel(),
                                        _index_stream(index))
    if rc:
        _check(rc, "dam_cache_read")
    return K, V, scratch


def _check_result(x: torch.Tensor, name: str, numel: int, dtype: torch.dtype):
    if x.dtype is not dtype or not x.is_contiguous() or x.numel() < numel:
        raise ValueError(f"{name} takes {numel} contiguous elements of {dtype}: got {tuple(x.shape)} of {x.dtype}, strides {x.stride()}")


def dam_cache_decode_attention(q: torch.Tensor, cache: Cache, positions: torch.Tensor, mask: Optional[torch.Tensor] = None,
                               softmax_scale: float = 0.0, O: Optional[torch.Tensor] = None,
                               lse: Optional[torch.Tensor] = None, scratch: Optional[torch.Tensor] = None):
    """One new token per sequence against an 8-bit cache (q, O: [B, Hq, d]; positions int32 [B]): every key up to its position,
    or, with a mask blob, those that its patterns keep.  Returns (O, LSE [B, Hq] fp32, scratch).  ValueError for an O or lse
    that cannot take the result, and for a tensor on another device than q."""
    n, Hq, d = shape = q.shape
    dtype = q.dtype
    assert shape == (cache.num_seqs, Hq, cache.head_dim) and q.is_contiguous() and (dtype is _BF16 or dtype is _F32)
    at = _per_sequence(positions, n)
    index = q.get_device()
    if scratch is None:
        scratch = _alloc(dam_cache_sizes(cache, Hq)[1], q.device)
    if O is None:
        O = torch.empty_like(q)
    if lse is None:
        lse = torch.empty(n, Hq, dtype=torch.float32, device=q.device)
    if not (O.get_device() == lse.get_device() == index == scratch.get_device() and positions.get_device() == index == cache.index >= 0
            and (mask is None or mask.get_device() == index)):
        _check_device(index, q=q, O=O, lse=lse, scratch=scratch, positions=positions, cache=cache, mask=mask)
    if not (O.dtype is dtype and O.is_contiguous() and O.shape == shape):
        _check_result(O, "O", n * Hq * d, dtype)
    if not (lse.dtype is _F32 and lse.is_contiguous() and lse.numel() == n * Hq):
        _check_result(lse, "lse", n * Hq, _F32)
    rc = (_lib or lib()).dam_cache_decode_attention(q.data_ptr(), cache.address, None if mask is None else mask.data_ptr(), at, Hq,
                                                    DAM_BF16 if dtype is _BF16 else DAM_F32, softmax_scale, O.data_ptr(), lse.data_ptr(),
                                                    scratch.data_ptr(), scratch.numel(), _index_stream(index))
    if rc:
        _check(rc, "dam_cache_decode_attention")
    return O, lse, scratch


def dam_mask_stats(mask: torch.Tensor, shape: Shape, active_elements: bool = False) -> dict:
    """Counts of a mask blob; with active_elements=True also the active cells per (sequence, head), counted by
    the library on the device (int64 tensor [num_seqs, num_q_heads], key "active_elements")."""
    out = (ctypes.c_uint64 * 5)()
    ae = torch.zeros(shape.c.num_seqs, shape.c.num_q_heads, dtype=torch.int64, device=mask.device) if active_elements else None
    rc = lib().dam_mask_stats(_ptr(mask), shape.ref, out, _ptr(ae), _stream(mask.device))
    _check(rc, "dam_mask_stats")
    st = {"tiles": int(out[0]), "full_tiles": int(out[1]), "causal_tiles": int(out[2]), "bytes_used": int(out[3]),
          "mask_tiles": int(out[4])}
    off = _HDR.fields["exec_tiles"][1]
    st["executed_tiles"] = int(mask[off: off + 8].cpu().numpy().view(np.uint64)[0])    # by the tensor-core kernel
    if active_elements:
        st["active_elements"] = ae
    return st


def dam_selftest_device_table(ordinals):
    """Runs the library's per-device table on a private table with a fake device query (no device needed).
    Returns (status code, sm_counts, (queries, set-up steps))."""
    n = len(ordinals)
    arr = (ctypes.c_int32 * max(1, n))(*ordinals)
    sm = (ctypes.c_int32 * max(1, n))()
    cnt = (ctypes.c_int32 * 2)()
    rc = lib().dam_selftest_device_table(arr, n, sm, cnt)
    return int(rc), [int(x) for x in sm[:n]], (int(cnt[0]), int(cnt[1]))


def dam_mask_expand_rows(mask: torch.Tensor, shape: Shape, seq: int, head: int, row_begin: int, nrows: int,
                         causal: bool = True) -> torch.Tensor:
    S = shape.lengths[seq]
    words = ((S + 127) // 128) * 4
    out = torch.empty(nrows, words, dtype=torch.int32, device=mask.device)
    rc = lib().dam_mask_expand_rows(_ptr(mask), shape.ref, seq, head, row_begin, nrows, int(causal), _ptr(out),
                                    _stream(mask.device))
    _check(rc, "dam_mask_expand_rows")
    return out


def attention_ran_on_tensor_cores(scratch: torch.Tensor) -> bool:
    """Test hook: word 4 of the attention scratch block says whether the tcgen05 kernel served the last call."""
    return int(scratch[16:20].cpu().numpy().view(np.uint32)[0]) == 1


def dam_poll_status(buf: torch.Tensor) -> int:
    return int(lib().dam_poll_status(_ptr(buf), _stream(buf.device)))


def dam_selftest_bounded_wait(device, limit_us: int = 20000):
    """Runs the bounded-wait self-test; returns (status read back, nanoseconds waited by the clock)."""
    status, words = bounded_wait_words(device, limit_us)
    return status, words[0]


def bounded_wait_words(device, limit_us: int = 20000):
    """The same; returns the status and what the self-test leaves behind it: nanoseconds of the wait by the clock, of a full count
    of polls and of the wait that was released, and how many of the three gave up."""
    scr = torch.zeros(256, dtype=torch.uint8, device=device)
    rc = lib().dam_selftest_bounded_wait(_ptr(scr), 256, limit_us, _stream(device))
    _check(rc, "dam_selftest_bounded_wait")
    status = dam_poll_status(scr)
    return status, [int(x) for x in scr[8:40].cpu().numpy().view(np.uint64)]


def dam_prefill_host(Qh: torch.Tensor, Kh: torch.Tensor, Vh: torch.Tensor, shape: Shape, rule: dam_rule_t,
                     Oh: torch.Tensor, lse_h: torch.Tensor, workspace: Optional[torch.Tensor], device,
                     causal: bool = True):
    """Host buffers in, host buffers out (copies inside the call).  workspace=None returns the size."""
    n = ctypes.c_size_t(0 if workspace is None else workspace.numel())
    rc = lib().dam_prefill_host(_ptr(Qh), _ptr(Kh), _ptr(Vh), shape.ref, ctypes.byref(rule), int(causal),
                                _ptr(Oh), _ptr(lse_h), _ptr(workspace), ctypes.byref(n), _stream(device))
    _check(rc, "dam_prefill_host")
    return n.value


# ----------------------------------------------------------------------------------------------
# Blob reader (host side, for tests and statistics): unpacks the sections of a mask blob.
# ----------------------------------------------------------------------------------------------
_HDR = np.dtype([("magic", "<u4"), ("status", "<u4"), ("version", "<u4"), ("flags", "<u4"),
                 ("num_seqs", "<i4"), ("num_q_heads", "<i4"), ("total_qblocks", "<i4"), ("rows", "<i4"),
                 ("tile_capacity", "<u4"), ("total_tiles", "<u4"), ("full_tiles", "<u4"), ("pcl_max", "<u4"),
                 ("off_seq", "<u8"), ("off_qbseq", "<u8"), ("off_dv", "<u8"), ("off_true", "<u8"),
                 ("off_tile_ptr", "<u8"), ("off_work", "<u8"), ("off_tiles", "<u8"), ("bytes_used", "<u8"),
                 ("causal_tiles", "<u8"), ("off_pairtab", "<u8"), ("total_pairs", "<i4"), ("prows", "<i4"),
                 ("gath_tiles", "<u8"), ("attn_scratch_bytes", "<u8"), ("mask_tiles", "<u8"), ("head_tile_cap", "<u8"), ("reserved", "<u8", (7,)),
                 ("off_lone", "<u8"), ("off_cols", "<u8"), ("off_lone2", "<u8"), ("exec_tiles", "<u8")])
_SEQ = np.dtype([("tok_start", "<i4"), ("S", "<i4"), ("L", "<i4"), ("nq", "<i4"), ("first_qblock", "<i4"),
                 ("W", "<i4"), ("nL", "<i4"), ("first_pair", "<i4"), ("dv_off", "<u8"), ("true_off", "<u8"),
                 ("p_off", "<u8"), ("cnt_off", "<u8"), ("gath_off", "<u8"), ("tile_base", "<u8")])


_ITEM = np.dtype([("head", "<i4"), ("tok0", "<i4"), ("qb0", "<i4"), ("S", "<i4"), ("a0", "<u4"), ("a1", "<u4"),
                  ("b1", "<u4"), ("seq_hasB", "<u4")])


def _unpack_bits(words: np.ndarray, n: int) -> np.ndarray:
    """uint32 words [..., W] -> uint8 bits [..., n] (bit j % 32 of word j / 32)."""
    b = np.unpackbits(words.astype("<u4").view(np.uint8), axis=-1, bitorder="little")
    return b[..., :n]


class MaskBlob:
    """Host copy of a mask blob with accessors for its sections."""

    def __init__(self, blob: torch.Tensor):
        hdr_bytes = blob[:256].cpu().numpy()
        self.hdr = np.frombuffer(hdr_bytes.tobytes(), dtype=_HDR)[0]
        assert self.hdr["magic"] == 0x4B4D4144, "not a DAM mask blob"
        used = int(max(self.hdr["bytes_used"], self.hdr["off_tiles"]))
        self.raw = blob[:used].cpu().numpy().tobytes()
        B = int(self.hdr["num_seqs"])
        self.seqs = np.frombuffer(self.raw, dtype=_SEQ, count=B, offset=int(self.hdr["off_seq"]))
        rows = int(self.hdr["rows"])
        self.tile_ptr = np.frombuffer(self.raw, dtype="<u4", count=rows + 1, offset=int(self.hdr["off_tile_ptr"]))
        self.items = np.frombuffer(self.raw, dtype=_ITEM, count=int(self.hdr["prows"]),
                                   offset=int(self.hdr["off_work"]))
        self.pair_tab = np.frombuffer(self.raw, dtype="<u4", count=int(self.hdr["total_pairs"]),
                                      offset=int(self.hdr["off_pairtab"]))
        # every row owns a fixed range of tiles[]: its entries, then possibly zero entries (kind 0) as padding
        self.tiles = np.frombuffer(self.raw, dtype="<u4", count=int(self.tile_ptr[rows]),
                                   offset=int(self.hdr["off_tiles"]))

    @property
    def scored_on_tensor_cores(self) -> bool:
        """Test hook: the window map of this blob was computed by the tcgen05 scoring kernel."""
        return int(self.hdr["reserved"][0]) == 1

    @property
    def scoring_groups(self) -> int:
        """Test hook: softmax groups of that kernel's CTAs, 4 (one CTA per SM) or 2 (two)."""
        return int(self.hdr["reserved"][1])

    def pattern_bits(self, seq: int, head: int):
        """(D, Drev, V) as uint8 [L]."""
        s = self.seqs[seq]
        L, W = int(s["L"]), int(s["W"])
        off = int(self.hdr["off_dv"]) + 4 * (int(s["dv_off"]) + head * 3 * W)
        w = np.frombuffer(self.raw, dtype="<u4", count=3 * W, offset=off).reshape(3, W)
        bits = _unpack_bits(w, L)
        return bits[0], bits[1], bits[2]

    def true_mask(self, seq: int, head: int) -> np.ndarray:
        s = self.seqs[seq]
        L, W = int(s["L"]), int(s["W"])
        off = int(self.hdr["off_true"]) + 4 * (int(s["true_off"]) + head * L * W)
        w = np.frombuffer(self.raw, dtype="<u4", count=L * W, offset=off).reshape(L, W)
        return _unpack_bits(w, L)

    def row_tiles(self, seq: int, head: int, qb: int):
        """(kv tile indices, kinds) of query block qb of (seq, head)."""
        row = head * int(self.hdr["total_qblocks"]) + int(self.seqs[seq]["first_qblock"]) + qb
        e = self.row_entries(seq, head, qb)
        kinds = (e >> 28).astype(np.int64)
        idx = np.where(kinds == 3, e & 0xFFFF, e & 0x0FFFFFFF).astype(np.int64)
        return idx, kinds

    def row_entries(self, seq: int, head: int, qb: int) -> np.ndarray:
        row = head * int(self.hdr["total_qblocks"]) + int(self.seqs[seq]["first_qblock"]) + qb
        e = self.tiles[self.tile_ptr[row]: self.tile_ptr[row + 1]]
        return e[(e >> 28) != 0]                                    # without the padding
