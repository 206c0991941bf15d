"""Python binding of the SemKV C ABI (include/semkv.h).

Argument marshalling only: every function below forwards to the function of the
same name in libsemkv.so, passing device pointers of torch tensors and the
current CUDA stream.  PyTorch provides device memory and streams; every step of
the cache's hot path runs in the library's CUDA kernels.  If the library has not
been built (``paper_2608_28911_gb300.build.build()``) importing this module
raises: there is no fallback.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

import torch

from . import build as _build

BASE_AFFINE, BASE_TQ, BASE_AFFINE_HAD, BASE_TQ_DENSE = 0, 1, 2, 3
HEAD_DIM = 128

_STATUS = {0: "ok", 1: "invalid argument", 2: "misaligned pointer or capacity",
           3: "capacity exceeded", 4: "unsupported", 5: "CUDA error", 6: "workspace too small"}


class SemkvError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn} failed: {_STATUS.get(status, status)} (status {status})")
        self.status = status


class QuantDescStruct(ctypes.Structure):
    _fields_ = [("base", ctypes.c_int32), ("levels_hi", ctypes.c_int32),
                ("levels_lo", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("signs", ctypes.c_void_p), ("centroids_hi", ctypes.c_void_p),
                ("thresholds_hi", ctypes.c_void_p), ("centroids_lo", ctypes.c_void_p),
                ("thresholds_lo", ctypes.c_void_p), ("rotation", ctypes.c_void_p)]


class CacheStruct(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("layers", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("q_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block", ctypes.c_int32),
                ("hi_pool", ctypes.c_void_p), ("lo_pool", ctypes.c_void_p),
                ("hi_cap", ctypes.c_int64), ("lo_cap", ctypes.c_int64),
                ("hi_tok", ctypes.c_void_p), ("lo_tok", ctypes.c_void_p),
                ("hi_count", ctypes.c_int64), ("lo_count", ctypes.c_int64),
                ("n_tokens", ctypes.c_int64),
                ("stage_k", ctypes.c_void_p), ("stage_v", ctypes.c_void_p),
                ("stage_score", ctypes.c_void_p), ("stage_n", ctypes.c_int32),
                ("blk_is_high", ctypes.c_void_p), ("blk_slot", ctypes.c_void_p),
                ("dev_error", ctypes.c_void_p)]


class KV4CacheStruct(ctypes.Structure):
    _fields_ = [("layers", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_tokens", ctypes.c_int32),
                ("num_pages", ctypes.c_int32), ("max_seqs", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("pages", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("table", ctypes.c_void_p), ("length", ctypes.c_void_p),
                ("refs", ctypes.c_void_p), ("dev_error", ctypes.c_void_p)]


class KV4BatchStruct(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("total", ctypes.c_int32), ("max_count", ctypes.c_int32),
                ("seqs", ctypes.c_void_p), ("cu", ctypes.c_void_p), ("start", ctypes.c_void_p)]


class KV4RotationStruct(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("rows", ctypes.c_int32),
                ("cos_sin", ctypes.c_void_p)]


def _load():
    path = _build.LIB
    if not os.path.exists(path):
        raise ImportError(f"libsemkv.so is not built ({path}); run "
                          "paper_2608_28911_gb300.build.build() first")
    L = ctypes.CDLL(path)
    p, i32, i64, u32, sz = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32,
                            ctypes.c_size_t)
    L.semkv_row_bytes.argtypes = [i32]
    L.semkv_row_bytes.restype = sz
    L.semkv_record_bytes.argtypes = [i32, i32]
    L.semkv_record_bytes.restype = sz
    L.semkv_high_count_floor.argtypes = [u32, u32, u32]
    L.semkv_high_count_floor.restype = u32
    L.semkv_block_high_count.argtypes = [u32, u32, u32]
    L.semkv_block_high_count.restype = u32
    L.semkv_lloyd_max_gaussian.argtypes = [i32, p, p]
    L.semkv_lloyd_max_gaussian.restype = ctypes.c_int
    L.semkv_rank_workspace_bytes.argtypes = [i32, i32, i32]
    L.semkv_rank_workspace_bytes.restype = sz
    L.semkv_rank_assign.argtypes = [p, i32, i32, u32, p, p, p, p, sz, p]
    L.semkv_rank_assign.restype = ctypes.c_int
    L.semkv_score_kv_norm.argtypes = [p, i32, i32, i32, i32, i32, i32, p, p]
    L.semkv_fake_quant.argtypes = [p, p, p, i32, i32, i32, i32, p, p, p, p]
    L.semkv_fake_quant.restype = ctypes.c_int
    L.semkv_score_kv_norm.restype = ctypes.c_int
    L.semkv_quantize_pack.argtypes = [ctypes.POINTER(QuantDescStruct), p, p, i32, p, p, u32,
                                      ctypes.POINTER(CacheStruct), p]
    L.semkv_quantize_pack.restype = ctypes.c_int
    L.semkv_append_block.argtypes = [ctypes.POINTER(QuantDescStruct),
                                     ctypes.POINTER(CacheStruct), u32, u32, p]
    L.semkv_append_block.restype = ctypes.c_int
    L.semkv_decode_workspace_bytes.argtypes = [ctypes.POINTER(CacheStruct)]
    L.semkv_decode_workspace_bytes.restype = sz
    L.semkv_decode_attention.argtypes = [ctypes.POINTER(QuantDescStruct),
                                         ctypes.POINTER(CacheStruct), i32, p, p,
                                         ctypes.c_float, p, sz, p]
    L.semkv_decode_attention.restype = ctypes.c_int
    L.semkv_decode_attention_noalloc.argtypes = [ctypes.POINTER(QuantDescStruct),
                                                 ctypes.POINTER(CacheStruct), i32, p, p,
                                                 ctypes.c_float, p]
    L.semkv_decode_attention_noalloc.restype = ctypes.c_int
    L.semkv_debug_wait_timeout.argtypes = [p, u32, p]
    L.semkv_debug_wait_timeout.restype = ctypes.c_int
    L.semkv_status_string.argtypes = [ctypes.c_int]
    L.semkv_status_string.restype = ctypes.c_char_p
    L.semkv_kv4_tile_bytes.argtypes = [i32]
    L.semkv_kv4_pages_workspace_bytes.argtypes = [p, i32, i32]
    L.semkv_kv4_attention_workspace_bytes.argtypes = [p, p, i32]
    for f in (L.semkv_kv4_tile_bytes, L.semkv_kv4_pages_workspace_bytes,
              L.semkv_kv4_attention_workspace_bytes):
        f.restype = sz
    L.semkv_kv4_reserve.argtypes = [p, p, p, sz, p]
    L.semkv_kv4_write.argtypes = [p, p, i32, i32, p, i64, p, i64, p]
    L.semkv_kv4_read.argtypes = [p, p, i32, i32, p, p, p]
    L.semkv_kv4_write_rotated.argtypes = [p, p, i32, p, p, i32, p, i64, i32, p, i64, p, i64, p, i64, p]
    L.semkv_kv4_attention.argtypes = [p, p, i32, i32, p, i64, i32, p, p, ctypes.c_float, i32, p,
                                      sz, p]
    L.semkv_kv4_fork.argtypes = [p, i32, p, p, p]
    L.semkv_kv4_free.argtypes = [p, i32, p, p]
    L.semkv_kv4_compact.argtypes = [p, i32, p, p, i32, p, sz, p]
    L.semkv_kv4_reorder.argtypes = [p, i32, p, p, p, sz, p]
    L.semkv_beam_select_workspace_bytes.argtypes = [i32] * 5
    L.semkv_beam_select_workspace_bytes.restype = sz
    L.semkv_beam_select.argtypes = [i32, i32, i32, i32, p, i64, p, p, i32, i32, p, p, p, p, p, sz, p]
    for f in (L.semkv_kv4_reserve, L.semkv_kv4_write, L.semkv_kv4_write_rotated, L.semkv_kv4_read,
              L.semkv_kv4_attention, L.semkv_kv4_fork, L.semkv_kv4_free, L.semkv_kv4_reorder,
              L.semkv_kv4_compact, L.semkv_beam_select):
        f.restype = ctypes.c_int
    return L


LIB = _load()
EXPORTED = ["semkv_row_bytes", "semkv_record_bytes", "semkv_high_count_floor",
            "semkv_block_high_count", "semkv_lloyd_max_gaussian", "semkv_rank_workspace_bytes",
            "semkv_rank_assign", "semkv_score_kv_norm", "semkv_fake_quant", "semkv_quantize_pack", "semkv_append_block",
            "semkv_decode_workspace_bytes", "semkv_decode_attention",
            "semkv_decode_attention_noalloc", "semkv_debug_wait_timeout", "semkv_status_string",
            "semkv_kv4_tile_bytes", "semkv_kv4_pages_workspace_bytes", "semkv_kv4_reserve",
            "semkv_kv4_write", "semkv_kv4_read", "semkv_kv4_attention_workspace_bytes",
            "semkv_kv4_attention", "semkv_kv4_fork", "semkv_kv4_free", "semkv_kv4_compact",
            "semkv_kv4_write_rotated", "semkv_kv4_reorder", "semkv_beam_select_workspace_bytes",
            "semkv_beam_select"]


def _ptr(t):
    if t is None:
        return None
    assert t.is_contiguous(), "tensors passed to libsemkv must be contiguous"
    return t.data_ptr()   # (the argument types make it a void*)


# The current stream's raw handle: building a torch Stream object took 3 of a decode call's
# 18 us.  The two names are private to torch, so a release without them takes the object.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _raw_device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_raw_device())


def _check(fn, status):
    if status != 0:
        raise SemkvError(fn, status)


# ------------------------------------------------------------- plain calls ----

def semkv_row_bytes(levels: int) -> int:
    return LIB.semkv_row_bytes(levels)


def semkv_record_bytes(base: int, levels: int) -> int:
    return LIB.semkv_record_bytes(base, levels)


def semkv_high_count_floor(T: int, r_num: int, r_den: int) -> int:
    return LIB.semkv_high_count_floor(T, r_num, r_den)


def semkv_block_high_count(n: int, r_num: int, r_den: int) -> int:
    return LIB.semkv_block_high_count(n, r_num, r_den)


def semkv_lloyd_max_gaussian(levels: int):
    """Host fp64 Lloyd-Max codebook -> (centroids f32 [L], thresholds f32 [L-1])."""
    c = (ctypes.c_float * levels)()
    t = (ctypes.c_float * max(levels - 1, 1))()
    _check("semkv_lloyd_max_gaussian", LIB.semkv_lloyd_max_gaussian(levels, c, t))
    return (torch.tensor(list(c), dtype=torch.float32),
            torch.tensor(list(t)[:levels - 1], dtype=torch.float32))


def semkv_rank_workspace_bytes(batch: int, T: int, want_rank: bool = True) -> int:
    return LIB.semkv_rank_workspace_bytes(batch, T, 1 if want_rank else 0)


def semkv_rank_assign(scores: torch.Tensor, n_high: int, is_high: torch.Tensor,
                      slot: torch.Tensor, rank=None, ws=None, stream=None):
    B, T = scores.shape
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check("semkv_rank_assign",
           LIB.semkv_rank_assign(_ptr(scores), B, T, n_high, _ptr(is_high), _ptr(slot),
                                 _ptr(rank), _ptr(ws), ws_bytes, _stream(stream)))


def semkv_fake_quant(desc: "QuantDesc", k: torch.Tensor, v: torch.Tensor, k_out: torch.Tensor,
                     v_out: torch.Tensor, is_high=None, stream=None):
    """Quantize + reconstruct every row of k, v [B][NL][H][T][128] fp16 into k_out, v_out."""
    B, NL, H, T, _ = k.shape
    _check("semkv_fake_quant",
           LIB.semkv_fake_quant(ctypes.byref(desc.s), _ptr(k), _ptr(v), B, NL, H, T,
                                _ptr(is_high), _ptr(k_out), _ptr(v_out), _stream(stream)))


def semkv_score_kv_norm(x: torch.Tensor, scores: torch.Tensor, layer_begin: int = 0,
                        layer_end=None, stream=None):
    """KV-norm importance scores of x [B][NL][H][T][128] fp16 into scores [B][T] f32."""
    B, NL, H, T, _ = x.shape
    le = NL if layer_end is None else layer_end
    _check("semkv_score_kv_norm",
           LIB.semkv_score_kv_norm(_ptr(x), B, NL, H, T, layer_begin, le, _ptr(scores),
                                   _stream(stream)))


def semkv_quantize_pack(desc: "QuantDesc", k: torch.Tensor, v: torch.Tensor, is_high, slot,
                        n_high: int, cache: "KVCache", stream=None):
    T = k.shape[3]
    _check("semkv_quantize_pack",
           LIB.semkv_quantize_pack(ctypes.byref(desc.s), _ptr(k), _ptr(v), T, _ptr(is_high),
                                   _ptr(slot), n_high, ctypes.byref(cache.s), _stream(stream)))


def semkv_append_block(desc: "QuantDesc", cache: "KVCache", r_num: int, r_den: int,
                       stream=None):
    _check("semkv_append_block",
           LIB.semkv_append_block(ctypes.byref(desc.s), ctypes.byref(cache.s), r_num, r_den,
                                  _stream(stream)))


def semkv_decode_workspace_bytes(cache: "KVCache") -> int:
    return LIB.semkv_decode_workspace_bytes(ctypes.byref(cache.s))


def semkv_decode_attention(desc: "QuantDesc", cache: "KVCache", layer: int, q: torch.Tensor,
                           out: torch.Tensor, softmax_scale: float, ws: torch.Tensor,
                           stream=None):
    _check("semkv_decode_attention",
           LIB.semkv_decode_attention(ctypes.byref(desc.s), ctypes.byref(cache.s), layer,
                                      _ptr(q), _ptr(out), softmax_scale, _ptr(ws),
                                      ws.numel() * ws.element_size(), _stream(stream)))


def semkv_decode_attention_noalloc(desc: "QuantDesc", cache: "KVCache", layer: int,
                                   q: torch.Tensor, out: torch.Tensor, softmax_scale: float,
                                   stream=None):
    """Decode attention with the library's static split-K scratch (no workspace):
    for callers that cannot allocate device memory.  See include/semkv.h."""
    _check("semkv_decode_attention_noalloc",
           LIB.semkv_decode_attention_noalloc(ctypes.byref(desc.s), ctypes.byref(cache.s), layer,
                                              _ptr(q), _ptr(out), softmax_scale,
                                              _stream(stream)))


def semkv_debug_wait_timeout(dev_error: torch.Tensor, polls: int, stream=None):
    """Run the kernels' bounded mbarrier wait on a barrier nothing arrives on, giving up
    after `polls` polls: the wait reports a timeout (1) in dev_error (device int32)."""
    _check("semkv_debug_wait_timeout",
           LIB.semkv_debug_wait_timeout(_ptr(dev_error), polls, _stream(stream)))


# ------------------------------------------- the paged cache held in 4 bits ----

_KV4_TYPES = {torch.float16: 0, torch.bfloat16: 1}


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _here(*tensors):
    """The calls run on the current device, so what they take has to be there."""
    dev = torch.cuda.current_device() if _raw_device is None else _raw_device()
    for t in tensors:
        if t.get_device() != dev:
            raise ValueError("tensors have to be on the current CUDA device")


def _ints(t, n, what):
    if t.dtype != torch.int32 or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{what} is a contiguous int32 tensor of {n}")
    return t.data_ptr()


def _list(t, n, what):
    if t is not None:
        _ints(t, n, what)
        _here(t)
    return t


def _rows(t, what, total, heads, head_dim):
    """Rows [total][heads][head_dim] with any stride between rows: the stride."""
    st = t.stride()
    if t.shape != (total, heads, head_dim) or st[2] != 1 or (st[1] != head_dim and heads > 1):
        raise ValueError(f"{what} is [{total}][{heads}][{head_dim}] with the heads of a row side by "
                         f"side: got {tuple(t.shape)}, strides {st}")
    return st[0] if total > 1 else heads * head_dim


def _type16(t, other, what):
    dtype = t.dtype
    kind = _KV4_TYPES.get(dtype)
    if kind is None or other.dtype != dtype:
        raise ValueError(f"{what} have one type, float16 or bfloat16")
    return kind


def semkv_kv4_tile_bytes(head_dim: int) -> int:
    return LIB.semkv_kv4_tile_bytes(head_dim)


def semkv_kv4_reserve(cache: "KV4Cache", batch: "KV4Batch", ws: torch.Tensor, stream=None):
    """Room for the batch's rows: pages, lengths, and batch.start."""
    _here(cache.pages, batch.start, ws)
    _check("semkv_kv4_reserve",
           LIB.semkv_kv4_reserve(cache.ref, batch.ref, _ptr(ws), ws.nbytes, _stream(stream)))


def semkv_kv4_write(cache: "KV4Cache", batch: "KV4Batch", layer: int, k: torch.Tensor,
                    v: torch.Tensor, stream=None):
    """Quantize rows k, v [total][kv_heads][head_dim] (any row stride) into the layer's pages."""
    total, heads, head_dim = batch.total, cache.kv_heads, cache.head_dim
    kind = _type16(k, v, "k and v")
    ks = _rows(k, "k", total, heads, head_dim)
    vs = _rows(v, "v", total, heads, head_dim)
    _here(cache.pages, batch.start, k, v)
    _check("semkv_kv4_write",
           LIB.semkv_kv4_write(cache.ref, batch.ref, layer, kind, k.data_ptr(), ks, v.data_ptr(), vs,
                               _stream(stream)))


def semkv_kv4_write_rotated(cache: "KV4Cache", batch: "KV4Batch", layer: int, rotation: "KV4Rotation",
                            k: torch.Tensor, v: torch.Tensor, q=None, q_out=None, positions=None,
                            stream=None):
    """semkv_kv4_write with keys turned by their positions on the way, and the step's queries
    q [total][q_heads][head_dim] (any row stride) turned into q_out, which may be q.  positions:
    int32 [total], or None for the rows' places in their sequences."""
    total, heads, head_dim = batch.total, cache.kv_heads, cache.head_dim
    kind = _type16(k, v, "k and v")
    ks = _rows(k, "k", total, heads, head_dim)
    vs = _rows(v, "v", total, heads, head_dim)
    q_heads = qs = ostr = 0
    qp = op = None
    if q is not None or q_out is not None:
        _need(q is not None and q_out is not None and q.dim() == 3 and q.dtype == q_out.dtype == k.dtype,
              "q and q_out come together, [total][q_heads][head_dim] of k's type")
        q_heads = q.shape[1]
        qs, ostr = _rows(q, "q", total, q_heads, head_dim), _rows(q_out, "q_out", total, q_heads, head_dim)
        qp, op = q.data_ptr(), q_out.data_ptr()
        _here(cache.pages, batch.start, rotation.cos_sin, k, v, q, q_out)
    else:
        _here(cache.pages, batch.start, rotation.cos_sin, k, v)
    where = None
    if positions is not None:
        where = _ints(positions, total, "positions")
        _here(positions)
    _check("semkv_kv4_write_rotated",
           LIB.semkv_kv4_write_rotated(cache.ref, batch.ref, layer, rotation.ref, where, kind,
                                       qp, qs, q_heads, op, ostr, k.data_ptr(), ks, v.data_ptr(), vs,
                                       _stream(stream)))


def semkv_kv4_read(cache: "KV4Cache", batch: "KV4Batch", layer: int, k_out: torch.Tensor,
                   v_out: torch.Tensor, stream=None):
    """The values of the batch's rows into k_out, v_out [total][kv_heads][head_dim]."""
    total, heads, head_dim = batch.total, cache.kv_heads, cache.head_dim
    kind = _type16(k_out, v_out, "k_out and v_out")
    _rows(k_out, "k_out", total, heads, head_dim)
    _rows(v_out, "v_out", total, heads, head_dim)
    _here(cache.pages, batch.start, k_out, v_out)
    _check("semkv_kv4_read",
           LIB.semkv_kv4_read(cache.ref, batch.ref, layer, kind, _ptr(k_out), _ptr(v_out),
                              _stream(stream)))


def semkv_kv4_attention(cache: "KV4Cache", batch: "KV4Batch", layer: int, q: torch.Tensor,
                        out: torch.Tensor, softmax_scale: float, ws: torch.Tensor, lse=None,
                        window: int = 0, stream=None):
    """Causal attention of the batch's rows q [total][q_heads][head_dim] over their sequences."""
    kind = _type16(q, out, "q and out")
    shape = q.shape
    heads = shape[1]
    qs = _rows(q, "q", batch.total, heads, cache.head_dim)
    _need(out.shape == shape, "out is as q")
    if lse is not None:
        _need(lse.dtype == torch.float32 and lse.shape == shape[:2], "lse is float32 [total][q_heads]")
        _here(lse)
    _here(cache.pages, batch.start, q, out, ws)  # (a batch's tensors are on one device)
    _check("semkv_kv4_attention",
           LIB.semkv_kv4_attention(cache.ref, batch.ref, layer, kind, q.data_ptr(), qs, heads,
                                   _ptr(out), _ptr(lse), softmax_scale, window, _ptr(ws), ws.nbytes,
                                   _stream(stream)))


def semkv_kv4_fork(cache: "KV4Cache", src: torch.Tensor, dst: torch.Tensor, stream=None):
    """dst[i] becomes a branch of src[i]: its length, and its pages shared."""
    n = src.numel()
    _here(cache.pages)
    _check("semkv_kv4_fork",
           LIB.semkv_kv4_fork(cache.ref, n, _list(src, n, "src").data_ptr(),
                              _list(dst, n, "dst").data_ptr(), _stream(stream)))


def semkv_kv4_free(cache: "KV4Cache", seqs: torch.Tensor, stream=None):
    """Empties sequences; pages that nobody else holds are free again."""
    n = seqs.numel()
    _here(cache.pages)
    _check("semkv_kv4_free",
           LIB.semkv_kv4_free(cache.ref, n, _list(seqs, n, "seqs").data_ptr(), _stream(stream)))


def semkv_kv4_reorder(cache: "KV4Cache", seqs, parent: torch.Tensor, ws: torch.Tensor, stream=None):
    """The i-th sequence of the list becomes a branch of what its parent[i]-th was before the call; -1
    empties it.  seqs: int32, or None for 0 .. n-1.  ws: cache.pages_workspace(n, 0)."""
    n = parent.numel()
    at = _ints(parent, n, "parent")
    if seqs is None:
        of = None
        _here(cache.pages, parent, ws)
    else:
        of = _ints(seqs, n, "seqs")
        _here(cache.pages, parent, ws, seqs)
    _check("semkv_kv4_reorder",
           LIB.semkv_kv4_reorder(cache.ref, n, of, at, _ptr(ws), ws.nbytes, _stream(stream)))


def semkv_kv4_compact(cache: "KV4Cache", seqs: torch.Tensor, keep: torch.Tensor, ws: torch.Tensor,
                      stream=None):
    """Prunes sequences to the tokens with keep[i][t] != 0 (and all from keep.shape[1] on)."""
    n = seqs.numel()
    _need(keep.dtype == torch.uint8 and keep.dim() == 2 and keep.shape[0] == n,
          "keep is uint8 [sequences][tokens]")
    _here(cache.pages, keep, ws)
    _check("semkv_kv4_compact",
           LIB.semkv_kv4_compact(cache.ref, n, _list(seqs, n, "seqs").data_ptr(), _ptr(keep),
                                 keep.shape[1], _ptr(ws), ws.nbytes, _stream(stream)))


# ------------------------------------------------------------ beam search ----

_BEAM_TYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}


def semkv_beam_select_workspace_bytes(groups: int, beams: int, vocab: int, dtype: torch.dtype,
                                      k: int) -> int:
    _need(dtype in _BEAM_TYPES, "logits are float16, bfloat16 or float32")
    return LIB.semkv_beam_select_workspace_bytes(groups, beams, vocab, _BEAM_TYPES[dtype], k)


def beam_select_workspace(logits: torch.Tensor, scores: torch.Tensor, k: int):
    """For semkv_beam_select of logits and scores of these shapes and this type."""
    size = semkv_beam_select_workspace_bytes(*scores.shape, logits.shape[1], logits.dtype, k)
    return torch.empty(size, dtype=torch.uint8, device=logits.device)


def semkv_beam_select(logits: torch.Tensor, scores: torch.Tensor, parent: torch.Tensor,
                      token: torch.Tensor, score: torch.Tensor, ws: torch.Tensor, done=None,
                      end_token: int = 0, dev_error=None, stream=None):
    """The k best continuations of each group's beams into parent, token (int32) and score (float32)
    [groups][k].  logits [groups * beams][vocab] (any row stride), scores float32 [groups][beams],
    done: uint8 or bool, one for each beam, or None."""
    _need(scores.dim() == 2 and parent.dim() == 2 and logits.dim() == 2,
          "scores is [groups][beams], parent [groups][k], logits [groups * beams][vocab]")
    (groups, beams), k, (rows, vocab), steps = scores.shape, parent.shape[1], logits.shape, logits.stride()
    kind = _BEAM_TYPES.get(logits.dtype)
    _need(kind is not None and rows == groups * beams and (vocab <= 1 or steps[1] == 1),
          "logits is float16, bfloat16 or float32 [groups * beams][vocab], a row's values side by side")
    shape = (groups, k)
    _need(scores.dtype == score.dtype == torch.float32 and parent.dtype == token.dtype == torch.int32
          and parent.shape == shape and token.shape == shape and score.shape == shape
          and scores.is_contiguous() and parent.is_contiguous() and token.is_contiguous()
          and score.is_contiguous(),
          "scores (float32), parent, token (int32) and score (float32) are contiguous and fit each other")
    if done is not None:
        _need(done.dtype in (torch.uint8, torch.bool) and done.is_contiguous() and done.numel() == groups * beams,
              "done is contiguous uint8 or bool, one for each beam")
        _here(done)
    if dev_error is not None:
        _here(_list(dev_error, 1, "dev_error"))
    _here(logits, scores, parent, token, score, ws)
    _check("semkv_beam_select",
           LIB.semkv_beam_select(groups, beams, vocab, kind, logits.data_ptr(), steps[0] if rows > 1 else vocab,
                                 scores.data_ptr(), None if done is None else done.data_ptr(), end_token, k,
                                 parent.data_ptr(), token.data_ptr(), score.data_ptr(), _ptr(dev_error), _ptr(ws),
                                 ws.nbytes, _stream(stream)))


# ------------------------------------------------------- owning wrappers ------

class QuantDesc:
    """A semkv_quant_desc whose device tables are torch tensors kept alive here."""

    def __init__(self, base: int, levels_hi: int, levels_lo: int, signs=None,
                 device="cuda", rotation=None):
        self.base, self.levels_hi, self.levels_lo = base, levels_hi, levels_lo
        self._keep = []
        s = QuantDescStruct(base=base, levels_hi=levels_hi, levels_lo=levels_lo,
                            head_dim=HEAD_DIM)
        if base in (BASE_TQ, BASE_TQ_DENSE):
            if base == BASE_TQ:
                assert signs is not None, "the TQ base needs a sign vector per (layer, head)"
                sg = torch.as_tensor(signs, dtype=torch.int8).to(device).contiguous()
                self._keep.append(sg)
                s.signs = sg.data_ptr()
                self.signs = sg
            else:
                assert rotation is not None, "the dense TQ base needs a rotation per (layer, head)"
                rt = torch.as_tensor(np.ascontiguousarray(rotation).view(np.int16)).to(device)
                self._keep.append(rt.contiguous())
                s.rotation = self._keep[-1].data_ptr()
                self.rotation = self._keep[-1]
            ch, th = semkv_lloyd_max_gaussian(levels_hi)
            cl, tl = semkv_lloyd_max_gaussian(levels_lo)
            tabs = [t.to(device).contiguous() for t in (ch, th, cl, tl)]
            self._keep += tabs
            s.centroids_hi, s.thresholds_hi, s.centroids_lo, s.thresholds_lo = \
                [t.data_ptr() for t in tabs]
            self.codebooks = {"hi": (ch, th), "lo": (cl, tl)}
        elif base == BASE_AFFINE_HAD:
            assert signs is not None, "the rotated affine base needs a sign vector per (layer, head)"
            sg = torch.as_tensor(signs, dtype=torch.int8).to(device).contiguous()
            self._keep.append(sg)
            s.signs = sg.data_ptr()
            self.signs = sg
        self.s = s


def _round16(n: int) -> int:
    return (n + 15) // 16 * 16


class KVCache:
    """Owns the device buffers of one semkv_cache (torch allocations) and the
    struct the library reads and updates."""

    def __init__(self, desc: QuantDesc, batch: int, layers: int, kv_heads: int, q_heads: int,
                 hi_cap: int, lo_cap: int, block: int = 128, device="cuda"):
        self.desc = desc
        hi_cap, lo_cap = _round16(max(hi_cap, 16)), _round16(max(lo_cap, 16))
        rh = semkv_record_bytes(desc.base, desc.levels_hi)
        rl = semkv_record_bytes(desc.base, desc.levels_lo)
        dev = torch.device(device)
        u8 = dict(dtype=torch.uint8, device=dev)
        self.hi_pool = torch.zeros((batch, layers, kv_heads, hi_cap, rh), **u8)
        self.lo_pool = torch.zeros((batch, layers, kv_heads, lo_cap, rl), **u8)
        self.hi_tok = torch.full((batch, hi_cap), -1, dtype=torch.int32, device=dev)
        self.lo_tok = torch.full((batch, lo_cap), -1, dtype=torch.int32, device=dev)
        self.stage_k = torch.zeros((batch, layers, kv_heads, block, HEAD_DIM), dtype=torch.float16,
                                   device=dev)
        self.stage_v = torch.zeros_like(self.stage_k)
        self.stage_score = torch.zeros((batch, block), dtype=torch.float32, device=dev)
        self.blk_is_high = torch.zeros((batch, block), **u8)
        self.blk_slot = torch.zeros((batch, block), dtype=torch.int32, device=dev)
        self.dev_error = torch.zeros(1, dtype=torch.int32, device=dev)
        self.s = CacheStruct(batch=batch, layers=layers, kv_heads=kv_heads, q_heads=q_heads,
                             head_dim=HEAD_DIM, block=block,
                             hi_pool=self.hi_pool.data_ptr(), lo_pool=self.lo_pool.data_ptr(),
                             hi_cap=hi_cap, lo_cap=lo_cap, hi_tok=self.hi_tok.data_ptr(),
                             lo_tok=self.lo_tok.data_ptr(), hi_count=0, lo_count=0, n_tokens=0,
                             stage_k=self.stage_k.data_ptr(), stage_v=self.stage_v.data_ptr(),
                             stage_score=self.stage_score.data_ptr(), stage_n=0,
                             blk_is_high=self.blk_is_high.data_ptr(),
                             blk_slot=self.blk_slot.data_ptr(),
                             dev_error=self.dev_error.data_ptr())

    # host mirrors kept by the library
    @property
    def hi_count(self):
        return self.s.hi_count

    @property
    def lo_count(self):
        return self.s.lo_count

    @property
    def n_tokens(self):
        return self.s.n_tokens

    @property
    def stage_n(self):
        return self.s.stage_n

    def stage_token(self, k_tok: torch.Tensor, v_tok: torch.Tensor, score: torch.Tensor):
        """Algorithm 2: append a generated token at full precision and record its
        score (a device copy into staging slot stage_n; no per-token decision)."""
        n = self.s.stage_n
        if n >= self.s.block:
            raise SemkvError("stage_token", 3)
        self.stage_k[:, :, :, n].copy_(k_tok)
        self.stage_v[:, :, :, n].copy_(v_tok)
        self.stage_score[:, n].copy_(score)
        self.s.stage_n = n + 1

    def workspace(self):
        nbytes = semkv_decode_workspace_bytes(self)
        return torch.empty(nbytes // 4, dtype=torch.float32, device=self.hi_pool.device)


class KV4Cache:
    """A paged cache held in 4 bits: its device buffers and the struct the library reads.
    k_scale, v_scale: float32 [layers][kv_heads] (None: 1)."""

    def __init__(self, layers: int, kv_heads: int, head_dim: int, page_tokens: int, num_pages: int,
                 max_seqs: int, max_pages: int, k_scale=None, v_scale=None, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        tile = semkv_kv4_tile_bytes(head_dim)
        _need(tile and page_tokens in (16, 32, 64, 128),
              "head_dim is 64 or 128, page_tokens 16, 32, 64 or 128")
        self._hold(torch.zeros((layers, num_pages, kv_heads, page_tokens // 16, tile),
                               dtype=torch.uint8, device=device),
                   torch.full((max_seqs, max_pages), -1, **i32), torch.zeros(max_seqs, **i32),
                   torch.zeros(num_pages, **i32), head_dim, k_scale, v_scale)

    @classmethod
    def over(cls, pages, table, length, refs, head_dim: int, k_scale=None, v_scale=None):
        """A cache over buffers that are there already."""
        self = cls.__new__(cls)
        self._hold(pages, table, length, refs, head_dim, k_scale, v_scale)
        return self

    def _hold(self, pages, table, length, refs, head_dim, k_scale, v_scale):
        _need(pages.dtype == torch.uint8 and pages.dim() == 5 and pages.is_contiguous()
              and pages.shape[4] == semkv_kv4_tile_bytes(head_dim),
              "pages is uint8 [layers][pages][kv_heads][page_tokens / 16][tile]")
        layers, num_pages, kv_heads, tiles, _ = pages.shape
        _need(table.dim() == 2, "table is int32 [sequences][pages of each]")
        for t, shape in ((table, table.shape), (length, table.shape[:1]), (refs, (num_pages,))):
            _need(t.dtype == torch.int32 and t.is_contiguous() and t.shape == shape,
                  "table, length and refs are contiguous int32 tensors that fit each other")
        _need(pages.data_ptr() % 16 == 0 and refs.data_ptr() % 16 == 0,
              "pages and refs begin on a multiple of 16 bytes")
        for t in (k_scale, v_scale):
            _need(t is None or (t.dtype == torch.float32 and t.is_contiguous()
                                and t.shape == (layers, kv_heads)),
                  "the scales are contiguous float32 [layers][kv_heads]")
        self.pages, self.table, self.length, self.refs = pages, table, length, refs
        self.kv_heads, self.head_dim = kv_heads, head_dim
        self.k_scale, self.v_scale = k_scale, v_scale
        self.dev_error = torch.zeros(1, dtype=torch.int32, device=pages.device)
        for t in (table, length, refs, k_scale, v_scale):
            _need(t is None or t.device == pages.device, "a cache lies on one device")
        self.s = KV4CacheStruct(layers=layers, kv_heads=kv_heads, head_dim=head_dim,
                                page_tokens=16 * tiles, num_pages=num_pages,
                                max_seqs=table.shape[0], max_pages=table.shape[1],
                                pages=_ptr(pages), k_scale=_ptr(k_scale), v_scale=_ptr(v_scale),
                                table=_ptr(table), length=_ptr(length), refs=_ptr(refs),
                                dev_error=_ptr(self.dev_error))
        self.ref = ctypes.byref(self.s)

    def pages_workspace(self, n: int, tokens: int = -1):
        """For reserve, or with keep's columns `tokens` for compact, of up to n sequences."""
        size = LIB.semkv_kv4_pages_workspace_bytes(self.ref, n, tokens)
        return torch.empty(size, dtype=torch.uint8, device=self.pages.device)

    def attention_workspace(self, batch: "KV4Batch", q_heads: int):
        size = LIB.semkv_kv4_attention_workspace_bytes(self.ref, batch.ref, q_heads)
        return torch.empty(size, dtype=torch.uint8, device=self.pages.device)


class KV4Batch:
    """The rows of one step over a KV4Cache (semkv_kv4_batch).  cu: int32 [n + 1], or None
    for one row to a sequence; seqs: int32 [n], or None for 0 .. n-1; total: rows of the
    step's tensors; max_count: no sequence has more rows (one that has is left out).  With
    cu it is `total` unless named; the step's own largest count makes for faster kernels."""

    def __init__(self, n: int, cu=None, seqs=None, start=None, total=None, max_count=None,
                 device="cuda"):
        _need(total is not None or cu is None, "total: the rows of the step's tensors")
        self.cu, self.seqs = _list(cu, n + 1, "cu"), _list(seqs, n, "seqs")
        self.start = (torch.zeros(n, dtype=torch.int32, device=device) if start is None
                      else _list(start, n, "start"))
        for t in (self.cu, self.seqs):
            _need(t is None or t.get_device() == self.start.get_device(), "a batch lies on one device")
        self.total = n if total is None else total
        if max_count is None:
            max_count = 1 if cu is None else self.total
        self.s = KV4BatchStruct(n=n, total=self.total, max_count=max_count,
                                seqs=_ptr(self.seqs), cu=_ptr(self.cu), start=_ptr(self.start))
        self.ref = ctypes.byref(self.s)


class KV4Rotation:
    """A table of positions' cosines and sines, float32 [positions][rot_dim]: rot_dim / 2 cosines, then
    the sines.  The first rot_dim dims of a head are turned, in pairs (j, j + rot_dim / 2) or, with
    pairs, (2 j, 2 j + 1)."""

    def __init__(self, cos_sin: torch.Tensor, pairs: bool = False):
        _need(cos_sin.dtype == torch.float32 and cos_sin.dim() == 2 and cos_sin.is_contiguous()
              and cos_sin.shape[0] > 0 and cos_sin.shape[1] > 0 and cos_sin.shape[1] % 16 == 0
              and cos_sin.data_ptr() % 16 == 0,
              "cos_sin is contiguous float32 [positions][rot_dim], rot_dim a multiple of 16, on a multiple "
              "of 16 bytes")
        self.cos_sin = cos_sin
        self.s = KV4RotationStruct(rot_dim=cos_sin.shape[1], layout=1 if pairs else 0, rows=cos_sin.shape[0],
                                   cos_sin=_ptr(cos_sin))
        self.ref = ctypes.byref(self.s)
