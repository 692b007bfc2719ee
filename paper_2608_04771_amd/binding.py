"""Thin Python binding of libreco.so (argument marshalling only).

Each function has the name of the C entry point it calls and forwards device
pointers (``tensor.data_ptr()``) and the current HIP stream of torch.  Every
step of the computation runs in the HIP kernels of the library; nothing here
computes a result.  The library must have been built in-tree
(``python -m paper_2608_04771_amd.build``); importing it otherwise fails.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os
import threading
from typing import Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libreco.so")

RECO_OK = 0
RECO_ERR_INVALID_ARG = 1
RECO_ERR_UNSUPPORTED = 2
RECO_ERR_WORKSPACE = 3
RECO_ERR_HIP = 4
RECO_F32 = 0
RECO_BF16 = 1
RECO_SCORE_CAUSAL = 1
RECO_POOL_MAX = 0
RECO_POOL_MEAN = 1
DEV_ERRORS = {0: "ok", 1: "append overflow", 2: "bad retention", 3: "bad score", 4: "bad token id",
              5: "bad length", 6: "bad logit row", 7: "bad page", 8: "bad budget", 9: "stalled eviction", 10: "bad group"}

EXPORTED = [
    "reco_score_workspace_size", "reco_score", "reco_select_compact_workspace_size", "reco_select_compact",
    "reco_pool_scores", "reco_layer_retention",
    "reco_decode_attn_workspace_size", "reco_decode_attn", "reco_decode_attn_noalloc", "reco_logit_penalty",
    "reco_penalty_sample_workspace_size", "reco_penalty_sample",
    "reco_paged_decode_attn_workspace_size", "reco_paged_decode_attn",
    "reco_paged_prefill_attn_workspace_size", "reco_paged_prefill_attn",
    "reco_paged_evict_workspace_size", "reco_paged_evict", "reco_rope", "reco_paged_append",
    "reco_paged_shared_decode_attn_workspace_size", "reco_paged_shared_decode_attn",
    "reco_answer_ppl_workspace_size", "reco_answer_ppl", "reco_retention_from_reward", "reco_retention_eq1",
    "reco_kept_count", "reco_status_str", "reco_abi_version",
]


class RecoKVCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("len", ctypes.c_void_p),
                ("n_layers", ctypes.c_int32), ("batch", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("capacity", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class RecoPagedCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("pages", ctypes.c_void_p), ("len", ctypes.c_void_p),
                ("weight", ctypes.c_void_p),
                ("n_layers", ctypes.c_int32), ("batch", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("n_pages", ctypes.c_int32), ("page_rows", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class RecoRows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("layer", ctypes.c_int64), ("seq", ctypes.c_int64),
                ("head", ctypes.c_int64), ("token", ctypes.c_int64)]


class RecoRope(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_void_p), ("pos", ctypes.c_void_p), ("axis", ctypes.POINTER(ctypes.c_int32)),
                ("n_axes", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32)]


_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libreco.so; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"HIP library missing: {path} (build it with `python -m paper_2608_04771_amd.build`)")
    lib = ctypes.CDLL(path)
    P, I32, I64, F32, F64, SZ, U32, U64 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float,
                                           ctypes.c_double, ctypes.c_size_t, ctypes.c_uint32, ctypes.c_uint64)
    C = ctypes.POINTER(RecoKVCache)
    PC = ctypes.POINTER(RecoPagedCache)
    RR = ctypes.POINTER(RecoRows)
    RP = ctypes.POINTER(RecoRope)
    sig = {
        "reco_score_workspace_size": (SZ, [C, I32, I32, I32]),
        "reco_score": (I32, [C, I32, I32, P, I32, I32, F32, U32, P, P, P, SZ, P, P]),
        "reco_select_compact_workspace_size": (SZ, [C, I32]),
        "reco_select_compact": (I32, [C, I32, I32, P, P, I64, I32, P, P, SZ, P, P]),
        "reco_pool_scores": (I32, [C, I32, I32, I32, P, P, I32, I32, P, P]),
        "reco_layer_retention": (F64, [F64, I32, I32, F64]),
        "reco_decode_attn_workspace_size": (SZ, [C, I32, I32]),
        "reco_decode_attn": (I32, [C, I32, I32, P, I32, F32, P, P, P, P, P, P, SZ, P, P]),
        "reco_decode_attn_noalloc": (I32, [C, I32, I32, P, I32, F32, P, P, P, P, P, P, P]),
        "reco_paged_decode_attn_workspace_size": (SZ, [PC, I32, I32]),
        "reco_paged_decode_attn": (I32, [PC, I32, I32, P, I32, F32, I32, I32, P, P, P, P, P, SZ, P, P]),
        "reco_paged_prefill_attn_workspace_size": (SZ, [PC, I32, I32, I32]),
        "reco_paged_prefill_attn": (I32, [PC, I32, I32, P, I32, I32, P, F32, I32, I32, P, P, P, P, P, SZ, P, P]),
        "reco_paged_evict_workspace_size": (SZ, [PC, I32]),
        "reco_paged_evict": (I32, [PC, I32, I32, P, I64, I32, I32, P, P, SZ, P, P]),
        "reco_paged_shared_decode_attn_workspace_size": (SZ, [PC, I32, I32, I32]),
        "reco_paged_shared_decode_attn": (I32, [PC, I32, I32, P, I32, F32, I32, I32, P, I32, P, I64, P, P, P, P, P, SZ,
                                                P, P]),
        "reco_rope": (I32, [RP, RR, RR, I32, I32, I32, I32, I32, I32, P, P, P]),
        "reco_paged_append": (I32, [PC, I32, I32, RP, I32, P, RR, RR, RR, RR, I32, P, P]),
        "reco_logit_penalty": (I32, [P, I32, I32, I64, P, I32, P, F32, F32, F32, F32, F32, P, P]),
        "reco_penalty_sample_workspace_size": (SZ, [I32, I32]),
        "reco_penalty_sample": (I32, [P, I32, I32, I64, P, I32, P, F32, F32, F32, F32, F32, F32, U64, U64, P, P, SZ,
                                      P, P]),
        "reco_answer_ppl_workspace_size": (SZ, [I32, I32, I32]),
        "reco_answer_ppl": (I32, [P, P, I32, I32, I32, F32, P, P, P, SZ, P, P]),
        "reco_retention_from_reward": (F64, [F64, F64, F64]),
        "reco_retention_eq1": (F64, [ctypes.POINTER(ctypes.c_double), I32, F64, F64]),
        "reco_kept_count": (I32, [I32, I32, F64]),
        "reco_status_str": (ctypes.c_char_p, [I32]),
        "reco_abi_version": (I32, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


# torch's current-stream handle without building a Stream object (a few
# microseconds per call otherwise); the public call is the fallback.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device) -> ctypes.c_void_p:
    if _raw_stream is not None:
        idx = device.index if device.index is not None else torch.cuda.current_device()
        return ctypes.c_void_p(_raw_stream(idx))
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _check(status: int, what: str):
    if status != RECO_OK:
        msg = load_library().reco_status_str(status).decode()
        raise RuntimeError(f"{what} failed: {msg} (status {status})")


def _need_cuda(*ts):
    """Every given tensor (None skipped) is a contiguous tensor on one GPU."""
    dev = None
    for t in ts:
        if t is not None:
            if not t.is_cuda:
                raise ValueError("tensors must live on the GPU")
            if not t.is_contiguous():
                raise ValueError("tensors must be contiguous")
            d = t.get_device()
            if dev is None:
                dev = d
            elif d != dev:
                raise ValueError("tensors of one call must live on the same GPU")


def _same_gpu(a: torch.Tensor, b: torch.Tensor):
    if not a.is_cuda or a.get_device() != b.get_device():
        raise ValueError("tensors of one call must live on the same GPU")


_DT = {torch.float32: "float32", torch.bfloat16: "bfloat16", torch.float64: "float64", torch.int32: "int32",
       torch.uint8: "uint8"}


def _expect(t: Optional[torch.Tensor], what: str, shape, dtype: torch.dtype):
    """The C ABI sees only pointers, so every tensor it indexes is checked here
    against the exact shape and dtype the call reads or writes: an undersized
    or mistyped buffer would otherwise be read or written out of bounds."""
    if t is None:
        return
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        raise ValueError(f"{what} must be {_DT.get(dtype, dtype)} {list(shape)}, "
                         f"got {_DT.get(t.dtype, t.dtype)} {list(t.shape)}")


def _expect_dev_err(dev_err: Optional[torch.Tensor]):
    if dev_err is not None and (dev_err.dtype != torch.int32 or dev_err.numel() < 1):
        raise ValueError("dev_err must be an int32 tensor with at least one element")


def _nbytes(t: torch.Tensor) -> int:
    return t.numel() * t.element_size()


class KVCache:
    """A KV cache in the library's layout: K and V ``[NL][B][H][Cap][D]``
    (fp32 or bf16), ``length`` ``[NL][B][H]`` int32, all on the GPU."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, length: torch.Tensor):
        if k.shape != v.shape or k.dim() != 5 or k.dtype != v.dtype:
            raise ValueError("k and v must share a [NL][B][H][Cap][D] shape and dtype")
        if k.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("cache dtype must be float32 or bfloat16")
        if length.dtype != torch.int32 or tuple(length.shape) != tuple(k.shape[:3]):
            raise ValueError("length must be int32 [NL][B][H]")
        _need_cuda(k, v, length)
        self.k, self.v, self.length = k, v, length
        NL, B, H, Cap, D = k.shape
        self.struct = RecoKVCache(k.data_ptr(), v.data_ptr(), length.data_ptr(), NL, B, H, Cap, D,
                                  RECO_F32 if k.dtype == torch.float32 else RECO_BF16)

    @property
    def shape(self):
        return tuple(self.k.shape)

    def ref(self):
        return ctypes.byref(self.struct)


class PagedKVCache:
    """A KV cache in pages: K and V ``[n_pages][page_rows][D]`` (fp32 or bf16; a
    page holds rows of one unit), the page ids of every unit ``pages``
    ``[NL][B][H][max_pages]`` int32, ``length`` ``[NL][B][H]`` int32 and, where
    attention weights are kept, ``weight`` ``[NL][B][H][max_pages * page_rows]``
    fp32, all on the GPU.  Allocating pages and listing them is the caller's; a
    unit's list has to reach the rows that a call appends."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, pages: torch.Tensor, length: torch.Tensor,
                 weight: Optional[torch.Tensor] = None):
        if k.shape != v.shape or k.dim() != 3 or k.dtype != v.dtype:
            raise ValueError("k and v must share a [n_pages][page_rows][D] shape and dtype")
        if k.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("cache dtype must be float32 or bfloat16")
        if pages.dtype != torch.int32 or pages.dim() != 4:
            raise ValueError("pages must be int32 [NL][B][H][max_pages]")
        if length.dtype != torch.int32 or tuple(length.shape) != tuple(pages.shape[:3]):
            raise ValueError("length must be int32 [NL][B][H]")
        n_pages, page_rows, D = k.shape
        NL, B, H, max_pages = pages.shape
        _expect(weight, "weight", (NL, B, H, max_pages * page_rows), torch.float32)
        _need_cuda(k, v, pages, length, weight)
        self.k, self.v, self.pages, self.length, self.weight = k, v, pages, length, weight
        self.struct = RecoPagedCache(k.data_ptr(), v.data_ptr(), pages.data_ptr(), length.data_ptr(),
                                     None if weight is None else weight.data_ptr(), NL, B, H, n_pages, page_rows,
                                     max_pages, D, RECO_F32 if k.dtype == torch.float32 else RECO_BF16)

    @property
    def shape(self):
        """(NL, B, H, capacity of a unit, D)"""
        (NL, B, H, max_pages), (_, page_rows, D) = self.pages.shape, self.k.shape
        return NL, B, H, max_pages * page_rows, D

    def ref(self):
        return ctypes.byref(self.struct)


def _on(t: torch.Tensor):
    """The tensor's GPU as the current one: launches and compute-unit counts go by that."""
    if torch.cuda.current_device() == t.get_device():
        return contextlib.nullcontext()
    return torch.cuda.device(t.get_device())


def _layers(cache: KVCache, layer0: int, n_layers: Optional[int]):
    layer0 = int(layer0)
    nl = (cache.shape[0] - layer0) if n_layers is None else int(n_layers)
    if layer0 < 0 or nl < 1 or layer0 + nl > cache.shape[0]:
        raise ValueError(f"layers [{layer0}, {layer0 + nl}) outside the cache's {cache.shape[0]} layers")
    return layer0, nl


def score_workspace_size(cache: KVCache, n_q_heads: int, w: int, n_layers: Optional[int] = None) -> int:
    nl = cache.shape[0] if n_layers is None else n_layers
    return int(load_library().reco_score_workspace_size(cache.ref(), nl, n_q_heads, w))


def select_compact_workspace_size(cache: KVCache, n_layers: Optional[int] = None) -> int:
    nl = cache.shape[0] if n_layers is None else n_layers
    return int(load_library().reco_select_compact_workspace_size(cache.ref(), nl))


def decode_attn_workspace_size(cache: KVCache, n_q_heads: int, n_layers: Optional[int] = None) -> int:
    nl = cache.shape[0] if n_layers is None else n_layers
    return int(load_library().reco_decode_attn_workspace_size(cache.ref(), nl, n_q_heads))


def paged_decode_attn_workspace_size(cache: PagedKVCache, n_q_heads: int, n_layers: Optional[int] = None) -> int:
    nl = cache.shape[0] if n_layers is None else n_layers
    with _on(cache.k):
        return int(load_library().reco_paged_decode_attn_workspace_size(cache.ref(), nl, n_q_heads))


def paged_prefill_attn_workspace_size(cache: PagedKVCache, n_q_heads: int, n_tokens: int,
                                      n_layers: Optional[int] = None) -> int:
    nl = cache.shape[0] if n_layers is None else n_layers
    with _on(cache.k):
        return int(load_library().reco_paged_prefill_attn_workspace_size(cache.ref(), nl, n_q_heads, n_tokens))


def paged_shared_decode_attn_workspace_size(cache: PagedKVCache, n_q_heads: int, n_groups: int,
                                            n_layers: Optional[int] = None) -> int:
    nl = cache.shape[0] if n_layers is None else n_layers
    with _on(cache.k):
        return int(load_library().reco_paged_shared_decode_attn_workspace_size(cache.ref(), nl, n_q_heads, n_groups))


def paged_evict_workspace_size(cache: PagedKVCache, n_layers: Optional[int] = None) -> int:
    nl = cache.shape[0] if n_layers is None else n_layers
    return int(load_library().reco_paged_evict_workspace_size(cache.ref(), nl))


def penalty_sample_workspace_size(rows: int, vocab: int) -> int:
    return int(load_library().reco_penalty_sample_workspace_size(rows, vocab))


def answer_ppl_workspace_size(batch: int, n: int, vocab: int) -> int:
    return int(load_library().reco_answer_ppl_workspace_size(batch, n, vocab))


def _ws(nbytes, device, ws: Optional[torch.Tensor]) -> torch.Tensor:
    """The caller's workspace, else a new one of nbytes() bytes (the library
    checks the size either way)."""
    if ws is not None:
        return ws
    return torch.empty(max(int(nbytes()), 1), dtype=torch.uint8, device=device)


def decode_workspace(cache: "KVCache", n_q_heads: int, n_layers: Optional[int] = None) -> torch.Tensor:
    """A decode workspace (contents need not be initialised).  Do not share
    one between overlapping calls."""
    return _ws(lambda: decode_attn_workspace_size(cache, n_q_heads, n_layers), cache.k.device, None)


def paged_decode_workspace(cache: PagedKVCache, n_q_heads: int, n_layers: Optional[int] = None) -> torch.Tensor:
    """A workspace for reco_paged_decode_attn (contents need not be initialised).
    Do not share one between overlapping calls."""
    return _ws(lambda: paged_decode_attn_workspace_size(cache, n_q_heads, n_layers), cache.k.device, None)


def paged_shared_decode_workspace(cache: PagedKVCache, n_q_heads: int, n_groups: int,
                                  n_layers: Optional[int] = None) -> torch.Tensor:
    """A workspace for reco_paged_shared_decode_attn (contents need not be
    initialised).  Do not share one between overlapping calls."""
    return _ws(lambda: paged_shared_decode_attn_workspace_size(cache, n_q_heads, n_groups, n_layers), cache.k.device, None)


def _score_shapes(cache: KVCache, nl: int, q_win: torch.Tensor, w: int, scores, row_stats):
    NL, B, H, Cap, D = cache.shape
    if q_win.dim() != 5 or q_win.shape[0] != nl or q_win.shape[1] != B or q_win.shape[3] != w or q_win.shape[4] != D:
        raise ValueError("q_win must be [n_layers][B][Hq][w][D]")
    if q_win.dtype != cache.k.dtype:
        raise ValueError("q_win must have the cache dtype")
    hq = q_win.shape[2]
    _expect(scores, "scores", (nl, B, H, Cap), torch.float32)
    _expect(row_stats, "row_stats", (nl, B, hq, w, 2), torch.float32)
    return hq


def reco_score(cache: KVCache, q_win: torch.Tensor, w: int, scale: Optional[float] = None, causal: bool = True,
               scores: Optional[torch.Tensor] = None, layer0: int = 0, n_layers: Optional[int] = None,
               ws: Optional[torch.Tensor] = None, dev_err: Optional[torch.Tensor] = None,
               row_stats: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Eq. 2 window attention mass; returns scores [n_layers][B][H][Cap] fp32.
    ``row_stats`` ([n_layers][B][Hq][w][2], from the window tokens' decode
    steps) replaces the normaliser pass over K."""
    layer0, nl = _layers(cache, layer0, n_layers)
    hq = _score_shapes(cache, nl, q_win, w, scores, row_stats)
    _expect_dev_err(dev_err)
    NL, B, H, Cap, D = cache.shape
    _need_cuda(cache.k, q_win, scores, ws, dev_err, row_stats)
    if scores is None:
        scores = torch.zeros((nl, B, H, Cap), dtype=torch.float32, device=cache.k.device)
    ws = _ws(lambda: score_workspace_size(cache, hq, w, nl), cache.k.device, ws)
    scale = 1.0 / math.sqrt(D) if scale is None else float(scale)
    st = load_library().reco_score(cache.ref(), layer0, nl, _ptr(q_win), hq, w, scale,
                                   RECO_SCORE_CAUSAL if causal else 0, _ptr(row_stats), _ptr(scores), _ptr(ws),
                                   _nbytes(ws), _ptr(dev_err), _stream(cache.k.device))
    _check(st, "reco_score")
    return scores


def _select_shapes(cache: KVCache, nl: int, scores: torch.Tensor, retention: torch.Tensor, kept_idx):
    NL, Bsz, H, Cap, D = cache.shape
    if retention.dtype != torch.float64:
        raise ValueError("retention must be float64")
    if tuple(retention.shape) == (Bsz,):
        stride = 0
    elif tuple(retention.shape) == (nl, Bsz):
        stride = Bsz
    else:
        raise ValueError("retention must be [B] or [n_layers][B]")
    _expect(scores, "scores", (nl, Bsz, H, Cap), torch.float32)
    _expect(kept_idx, "kept_idx", (nl, Bsz, H, Cap), torch.int32)
    return stride


def reco_select_compact(cache: KVCache, scores: torch.Tensor, retention: torch.Tensor, w: int,
                        kept_idx: Optional[torch.Tensor] = None, layer0: int = 0, n_layers: Optional[int] = None,
                        ws: Optional[torch.Tensor] = None, dev_err: Optional[torch.Tensor] = None):
    """Select the reward budget per unit and compact K/V in place (len <- m).
    ``retention`` is float64 [B] (one level per sequence) or [n_layers][B]
    (per-layer budgets)."""
    layer0, nl = _layers(cache, layer0, n_layers)
    stride = _select_shapes(cache, nl, scores, retention, kept_idx)
    _expect_dev_err(dev_err)
    _need_cuda(cache.k, scores, retention, kept_idx, ws, dev_err)
    ws = _ws(lambda: select_compact_workspace_size(cache, nl), cache.k.device, ws)
    st = load_library().reco_select_compact(cache.ref(), layer0, nl, _ptr(scores), _ptr(retention), stride, w,
                                            _ptr(kept_idx), _ptr(ws), _nbytes(ws), _ptr(dev_err),
                                            _stream(cache.k.device))
    _check(st, "reco_select_compact")
    return kept_idx


def reco_pool_scores(cache: KVCache, scores: torch.Tensor, w: int, kernel: int, mode: str = "max",
                     pooled: Optional[torch.Tensor] = None, layer0: int = 0, n_layers: Optional[int] = None,
                     dev_err: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Max / mean pooling of the prefix scores (window scores copied); returns
    pooled [n_layers][B][H][Cap] fp32 (entries at or beyond len unwritten)."""
    layer0, nl = _layers(cache, layer0, n_layers)
    NL, Bsz, H, Cap, D = cache.shape
    if mode not in ("max", "mean"):
        raise ValueError("mode must be 'max' or 'mean'")
    _expect(scores, "scores", (nl, Bsz, H, Cap), torch.float32)
    _expect(pooled, "pooled", (nl, Bsz, H, Cap), torch.float32)
    _expect_dev_err(dev_err)
    _need_cuda(cache.k, scores, pooled, dev_err)
    if pooled is None:
        pooled = torch.zeros_like(scores)
    st = load_library().reco_pool_scores(cache.ref(), layer0, nl, w, _ptr(scores), _ptr(pooled), kernel,
                                         RECO_POOL_MAX if mode == "max" else RECO_POOL_MEAN, _ptr(dev_err),
                                         _stream(cache.k.device))
    _check(st, "reco_pool_scores")
    return pooled


def _decode_shapes(cache: KVCache, nl: int, q: torch.Tensor, k_new, v_new, out, lse, row_stats):
    NL, B, H, Cap, D = cache.shape
    if q.dim() != 4 or q.shape[0] != nl or q.shape[1] != B or q.shape[3] != D or q.dtype != cache.k.dtype:
        raise ValueError("q must be [n_layers][B][Hq][D] in the cache dtype")
    hq = q.shape[2]
    if (k_new is None) != (v_new is None):
        raise ValueError("k_new and v_new must be given together")
    _expect(k_new, "k_new", (nl, B, H, D), cache.k.dtype)
    _expect(v_new, "v_new", (nl, B, H, D), cache.k.dtype)
    _expect(out, "out", (nl, B, hq, D), cache.k.dtype)
    _expect(lse, "lse", (nl, B, hq), torch.float32)
    _expect(row_stats, "row_stats", (nl, B, hq, 2), torch.float32)
    return hq


def reco_decode_attn(cache: KVCache, q: torch.Tensor, k_new: Optional[torch.Tensor] = None,
                     v_new: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                     out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, want_lse: bool = True,
                     layer0: int = 0, n_layers: Optional[int] = None, ws: Optional[torch.Tensor] = None,
                     dev_err: Optional[torch.Tensor] = None, row_stats: Optional[torch.Tensor] = None):
    """GQA decode attention (optionally appending the new token); returns (out, lse).
    ``row_stats`` ([n_layers][B][Hq][2] fp32) optionally receives each query's
    (max, sum) of the log2-domain logits."""
    layer0, nl = _layers(cache, layer0, n_layers)
    hq = _decode_shapes(cache, nl, q, k_new, v_new, out, lse, row_stats)
    _expect_dev_err(dev_err)
    _need_cuda(cache.k, q, k_new, v_new, out, lse, ws, dev_err, row_stats)
    NL, B, H, Cap, D = cache.shape
    if out is None:
        out = torch.empty_like(q)
    if lse is None and want_lse:
        lse = torch.empty((nl, B, hq), dtype=torch.float32, device=q.device)
    ws = _ws(lambda: decode_attn_workspace_size(cache, hq, nl), q.device, ws)
    scale = 1.0 / math.sqrt(D) if scale is None else float(scale)
    st = load_library().reco_decode_attn(cache.ref(), layer0, nl, _ptr(q), hq, scale, _ptr(k_new), _ptr(v_new),
                                         _ptr(out), _ptr(lse), _ptr(row_stats), _ptr(ws), _nbytes(ws),
                                         _ptr(dev_err), _stream(q.device))
    _check(st, "reco_decode_attn")
    return out, lse


def reco_decode_attn_noalloc(cache: KVCache, q: torch.Tensor, out: torch.Tensor, lse: Optional[torch.Tensor] = None,
                             k_new: Optional[torch.Tensor] = None, v_new: Optional[torch.Tensor] = None,
                             scale: Optional[float] = None, layer0: int = 0, n_layers: Optional[int] = None,
                             dev_err: Optional[torch.Tensor] = None, row_stats: Optional[torch.Tensor] = None):
    """reco_decode_attn without a workspace and without any allocation: the
    caller passes ``out`` (and optionally ``lse``); the split partials live in
    the library's static per-device array.  Calls overlapping on one GPU race."""
    layer0, nl = _layers(cache, layer0, n_layers)
    if out is None:
        raise ValueError("out must be given (this entry point allocates nothing)")
    _decode_shapes(cache, nl, q, k_new, v_new, out, lse, row_stats)
    _expect_dev_err(dev_err)
    _need_cuda(cache.k, q, k_new, v_new, out, lse, dev_err, row_stats)
    D = cache.shape[4]
    scale = 1.0 / math.sqrt(D) if scale is None else float(scale)
    st = load_library().reco_decode_attn_noalloc(cache.ref(), layer0, nl, _ptr(q), q.shape[2], scale, _ptr(k_new),
                                                 _ptr(v_new), _ptr(out), _ptr(lse), _ptr(row_stats), _ptr(dev_err),
                                                 _stream(q.device))
    _check(st, "reco_decode_attn_noalloc")
    return out, lse


class PreparedDecode:
    """reco_decode_attn for a loop that calls it again and again with the same
    cache, outputs, workspace and error word (a decoder's per-token call):
    those are checked once here, and each call checks only the tensors that
    change from token to token (query, new K/V rows, statistics slot) against
    the shapes fixed at construction before passing their pointers on.  The
    library computes exactly what reco_decode_attn computes."""

    def __init__(self, cache: KVCache, n_q_heads: int, out: torch.Tensor, lse: Optional[torch.Tensor],
                 ws: torch.Tensor, dev_err: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                 layer0: int = 0, n_layers: Optional[int] = None):
        layer0, nl = _layers(cache, layer0, n_layers)
        NL, Bsz, H, Cap, D = cache.shape
        hq = int(n_q_heads)
        if out is None or ws is None:
            raise ValueError("out and ws must be given")
        _expect(out, "out", (nl, Bsz, hq, D), cache.k.dtype)
        _expect(lse, "lse", (nl, Bsz, hq), torch.float32)
        _expect_dev_err(dev_err)
        _need_cuda(cache.k, out, lse, ws, dev_err)
        _same_gpu(out, cache.k)
        if _nbytes(ws) < decode_attn_workspace_size(cache, hq, nl):
            raise ValueError("ws is smaller than reco_decode_attn_workspace_size")
        self.cache, self.out, self.lse, self.ws, self.dev_err = cache, out, lse, ws, dev_err
        self._fn = load_library().reco_decode_attn
        self._dev = cache.k.device
        self._dt = cache.k.dtype
        self._q_shape = (nl, Bsz, hq, D)
        self._kv_shape = (nl, Bsz, H, D)
        self._st_shape = (nl, Bsz, hq, 2)
        self._fixed_head = (cache.ref(), layer0, nl)
        self._hq = hq
        self._scale = 1.0 / math.sqrt(D) if scale is None else float(scale)
        self._fixed_tail = (_ptr(out), _ptr(lse))
        self._ws = (_ptr(ws), _nbytes(ws), _ptr(dev_err))

    def _check_t(self, t: torch.Tensor, what: str, shape, dtype: torch.dtype):
        if (tuple(t.shape) != shape or t.dtype != dtype or t.device != self._dev or not t.is_contiguous()):
            raise ValueError(f"{what} must be a contiguous {_DT.get(dtype, dtype)} {list(shape)} tensor on "
                             f"{self._dev}")

    def __call__(self, q: torch.Tensor, k_new: Optional[torch.Tensor] = None, v_new: Optional[torch.Tensor] = None,
                 row_stats: Optional[torch.Tensor] = None):
        self._check_t(q, "q", self._q_shape, self._dt)
        if (k_new is None) != (v_new is None):
            raise ValueError("k_new and v_new must be given together")
        if k_new is not None:
            self._check_t(k_new, "k_new", self._kv_shape, self._dt)
            self._check_t(v_new, "v_new", self._kv_shape, self._dt)
        if row_stats is not None:
            self._check_t(row_stats, "row_stats", self._st_shape, torch.float32)
        cref, layer0, nl = self._fixed_head
        st = self._fn(cref, layer0, nl, _ptr(q), self._hq, self._scale, _ptr(k_new), _ptr(v_new),
                      *self._fixed_tail, _ptr(row_stats), *self._ws, _stream(self._dev))
        if st != RECO_OK:
            _check(st, "reco_decode_attn")
        return self.out, self.lse


def _row_count(n, what: str) -> int:
    """A count of rows as the C ABI takes it; a larger one would lose its upper bits on
    the way (2**32 + 5 rows of window would be five)."""
    n = int(n)
    if not -0x80000000 <= n <= 0x7fffffff:
        raise ValueError(f"{what} must fit 32 bits, got {n}")
    return n


def _paged_decode_shapes(cache: PagedKVCache, nl: int, q: torch.Tensor, k_new, v_new, out, lse):
    NL, B, H, Cap, D = cache.shape
    if q.dim() != 4 or q.shape[0] != nl or q.shape[1] != B or q.shape[3] != D or q.dtype != cache.k.dtype:
        raise ValueError("q must be [n_layers][B][Hq][D] in the cache dtype")
    hq = q.shape[2]
    if (k_new is None) != (v_new is None):
        raise ValueError("k_new and v_new must be given together")
    _expect(k_new, "k_new", (nl, B, H, D), cache.k.dtype)
    _expect(v_new, "v_new", (nl, B, H, D), cache.k.dtype)
    _expect(out, "out", (nl, B, hq, D), cache.k.dtype)
    _expect(lse, "lse", (nl, B, hq), torch.float32)
    return hq


def reco_paged_decode_attn(cache: PagedKVCache, q: torch.Tensor, k_new: Optional[torch.Tensor] = None,
                           v_new: Optional[torch.Tensor] = None, sinks: int = 0, window: int = 0,
                           scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                           lse: Optional[torch.Tensor] = None, want_lse: bool = True, layer0: int = 0,
                           n_layers: Optional[int] = None, ws: Optional[torch.Tensor] = None,
                           dev_err: Optional[torch.Tensor] = None):
    """GQA decode attention over a paged cache (optionally appending the new
    token); returns (out, lse).  ``window`` > 0: the token sees its last
    ``window`` rows (its own among them) and the first ``sinks``.  A cache with
    weights accumulates them."""
    layer0, nl = _layers(cache, layer0, n_layers)
    sinks, window = _row_count(sinks, "sinks"), _row_count(window, "window")
    hq = _paged_decode_shapes(cache, nl, q, k_new, v_new, out, lse)
    _expect_dev_err(dev_err)
    _need_cuda(cache.k, q, k_new, v_new, out, lse, ws, dev_err)
    NL, B, H, Cap, D = cache.shape
    if out is None:
        out = torch.empty_like(q)
    if lse is None and want_lse:
        lse = torch.empty((nl, B, hq), dtype=torch.float32, device=q.device)
    ws = _ws(lambda: paged_decode_attn_workspace_size(cache, hq, nl), q.device, ws)
    scale = 1.0 / math.sqrt(D) if scale is None else float(scale)
    with _on(q):
        st = load_library().reco_paged_decode_attn(cache.ref(), layer0, nl, _ptr(q), hq, scale, sinks,
                                                   window, _ptr(k_new), _ptr(v_new), _ptr(out), _ptr(lse),
                                                   _ptr(ws), _nbytes(ws), _ptr(dev_err), _stream(q.device))
    _check(st, "reco_paged_decode_attn")
    return out, lse


class PreparedPagedDecode:
    """reco_paged_decode_attn for a loop that calls it again and again with the
    same cache, outputs, workspace and error word, as PreparedDecode is for
    reco_decode_attn: those are checked once here, each call checks the tensors
    that change from token to token."""

    def __init__(self, cache: PagedKVCache, n_q_heads: int, out: torch.Tensor, lse: Optional[torch.Tensor],
                 ws: torch.Tensor, dev_err: Optional[torch.Tensor] = None, sinks: int = 0, window: int = 0,
                 scale: Optional[float] = None, layer0: int = 0, n_layers: Optional[int] = None):
        layer0, nl = _layers(cache, layer0, n_layers)
        NL, Bsz, H, Cap, D = cache.shape
        sinks, window = _row_count(sinks, "sinks"), _row_count(window, "window")
        hq = int(n_q_heads)
        if out is None or ws is None:
            raise ValueError("out and ws must be given")
        _expect(out, "out", (nl, Bsz, hq, D), cache.k.dtype)
        _expect(lse, "lse", (nl, Bsz, hq), torch.float32)
        _expect_dev_err(dev_err)
        _need_cuda(cache.k, out, lse, ws, dev_err)
        if _nbytes(ws) < paged_decode_attn_workspace_size(cache, hq, nl):
            raise ValueError("ws is smaller than reco_paged_decode_attn_workspace_size")
        self.cache, self.out, self.lse = cache, out, lse
        self._keep = (ws, dev_err)
        self._fn = load_library().reco_paged_decode_attn
        self._dev, self._dt = cache.k.device, cache.k.dtype
        self._q_shape, self._kv_shape = (nl, Bsz, hq, D), (nl, Bsz, H, D)
        scale = 1.0 / math.sqrt(D) if scale is None else float(scale)
        self._head = (cache.ref(), layer0, nl)
        self._mid = (hq, scale, sinks, window)
        self._tail = (_ptr(out), _ptr(lse), _ptr(ws), _nbytes(ws), _ptr(dev_err))

    def _check_t(self, t: torch.Tensor, what: str, shape):
        if tuple(t.shape) != shape or t.dtype != self._dt or t.device != self._dev or not t.is_contiguous():
            raise ValueError(f"{what} must be a contiguous {_DT[self._dt]} {list(shape)} tensor on {self._dev}")

    def __call__(self, q: torch.Tensor, k_new: Optional[torch.Tensor] = None, v_new: Optional[torch.Tensor] = None):
        self._check_t(q, "q", self._q_shape)
        if (k_new is None) != (v_new is None):
            raise ValueError("k_new and v_new must be given together")
        if k_new is not None:
            self._check_t(k_new, "k_new", self._kv_shape)
            self._check_t(v_new, "v_new", self._kv_shape)
        with _on(q):
            st = self._fn(*self._head, _ptr(q), *self._mid, _ptr(k_new), _ptr(v_new), *self._tail, _stream(self._dev))
        if st != RECO_OK:
            _check(st, "reco_paged_decode_attn")
        return self.out, self.lse


class PreparedPagedSharedDecode:
    """reco_paged_shared_decode_attn for a loop that calls it again and again with the same
    cache, groups, outputs, workspace and error word (whose contents may change): those are
    checked once here, each call checks the tensors that change from token to token."""

    def __init__(self, cache: PagedKVCache, n_q_heads: int, first: torch.Tensor, shared: torch.Tensor,
                 out: torch.Tensor, lse: Optional[torch.Tensor], ws: torch.Tensor,
                 dev_err: Optional[torch.Tensor] = None, sinks: int = 0, window: int = 0,
                 scale: Optional[float] = None, layer0: int = 0, n_layers: Optional[int] = None):
        layer0, nl = _layers(cache, layer0, n_layers)
        NL, Bsz, H, Cap, D = cache.shape
        sinks, window = _row_count(sinks, "sinks"), _row_count(window, "window")
        hq = int(n_q_heads)
        if out is None or ws is None:
            raise ValueError("out and ws must be given")
        if cache.weight is not None:
            raise ValueError("rows that sequences share have no weight of one: the cache must be without weights")
        if first.dtype != torch.int32 or first.dim() != 1 or not 2 <= first.numel() <= Bsz + 1:
            raise ValueError(f"first must be int32 [n_groups + 1], of 1 to {Bsz} groups")
        groups = first.numel() - 1
        if shared.dtype != torch.int32 or tuple(shared.shape) not in ((groups,), (nl, groups)):
            raise ValueError("shared must be int32 [n_groups] or [n_layers][n_groups]")
        _expect(out, "out", (nl, Bsz, hq, D), cache.k.dtype)
        _expect(lse, "lse", (nl, Bsz, hq), torch.float32)
        _expect_dev_err(dev_err)
        _need_cuda(cache.k, first, shared, out, lse, ws, dev_err)
        if _nbytes(ws) < paged_shared_decode_attn_workspace_size(cache, hq, groups, nl):
            raise ValueError("ws is smaller than reco_paged_shared_decode_attn_workspace_size")
        self.cache, self.out, self.lse = cache, out, lse
        self._keep = (first, shared, ws, dev_err)
        self._fn = load_library().reco_paged_shared_decode_attn
        self._dev, self._dt, self._index = cache.k.device, cache.k.dtype, cache.k.get_device()
        self._q_shape, self._kv_shape = (nl, Bsz, hq, D), (nl, Bsz, H, D)
        scale = 1.0 / math.sqrt(D) if scale is None else float(scale)
        self._head = (cache.ref(), layer0, nl)
        self._mid = (hq, scale, sinks, window, _ptr(first), groups, _ptr(shared), 0 if shared.dim() == 1 else groups)
        self._tail = (_ptr(out), _ptr(lse), _ptr(ws), _nbytes(ws), _ptr(dev_err))

    def _check_t(self, t: torch.Tensor, what: str, shape):
        if t.shape != shape or t.dtype != self._dt or t.get_device() != self._index or not t.is_contiguous():
            raise ValueError(f"{what} must be a contiguous {_DT[self._dt]} {list(shape)} tensor on {self._dev}")

    def __call__(self, q: torch.Tensor, k_new: Optional[torch.Tensor] = None, v_new: Optional[torch.Tensor] = None):
        self._check_t(q, "q", self._q_shape)
        if (k_new is None) != (v_new is None):
            raise ValueError("k_new and v_new must be given together")
        if k_new is not None:
            self._check_t(k_new, "k_new", self._kv_shape)
            self._check_t(v_new, "v_new", self._kv_shape)
        st = _launch(self._index, self._fn, *self._head, q.data_ptr(), *self._mid, None if k_new is None else k_new.data_ptr(),
                     None if v_new is None else v_new.data_ptr(), *self._tail)
        if st != RECO_OK:
            _check(st, "reco_paged_shared_decode_attn")
        return self.out, self.lse


def reco_paged_shared_decode_attn(cache: PagedKVCache, q: torch.Tensor, first: torch.Tensor, shared: torch.Tensor,
                                  k_new: Optional[torch.Tensor] = None, v_new: Optional[torch.Tensor] = None,
                                  sinks: int = 0, window: int = 0, scale: Optional[float] = None,
                                  out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                                  want_lse: bool = True, layer0: int = 0, n_layers: Optional[int] = None,
                                  ws: Optional[torch.Tensor] = None, dev_err: Optional[torch.Tensor] = None):
    """reco_paged_decode_attn for groups of sequences whose first rows are the same ones,
    which are read once for all; returns (out, lse).  ``first`` int32 [n_groups + 1]: group
    g is the sequences first[g] to first[g + 1] - 1, ``shared`` int32 [n_groups] or
    [n_layers][n_groups] its shared rows, taken from its first sequence's pages."""
    _, nl = _layers(cache, layer0, n_layers)
    if q.dim() != 4:
        raise ValueError("q must be [n_layers][B][Hq][D] in the cache dtype")
    hq = q.shape[2]
    if out is None:
        out = torch.empty_like(q)
    if lse is None and want_lse:
        lse = torch.empty((nl, cache.shape[1], hq), dtype=torch.float32, device=q.device)
    ws = _ws(lambda: paged_shared_decode_attn_workspace_size(cache, hq, first.numel() - 1, nl), q.device, ws)
    call = PreparedPagedSharedDecode(cache, hq, first, shared, out, lse, ws, dev_err, sinks, window, scale, layer0, nl)
    return call(q, k_new, v_new)


def reco_paged_prefill_attn(cache: PagedKVCache, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor,
                            n_new: Optional[torch.Tensor] = None, sinks: int = 0, window: int = 0,
                            scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                            lse: Optional[torch.Tensor] = None, want_lse: bool = True, layer0: int = 0,
                            n_layers: Optional[int] = None, ws: Optional[torch.Tensor] = None,
                            dev_err: Optional[torch.Tensor] = None):
    """Causal attention of T new tokens per sequence ([n_layers][B][Hq][T][D]) over a
    paged cache, whose rows they then become; returns (out, lse).  ``n_new`` int32
    [B]: the real tokens of each sequence (the first ones; places past them are not
    written).  ``window`` > 0: a token sees its last ``window`` rows (its own among
    them) and the first ``sinks``."""
    layer0, nl = _layers(cache, layer0, n_layers)
    sinks, window = _row_count(sinks, "sinks"), _row_count(window, "window")
    NL, B, H, Cap, D = cache.shape
    if q.dim() != 5 or q.shape[0] != nl or q.shape[1] != B or q.shape[4] != D or q.dtype != cache.k.dtype:
        raise ValueError("q must be [n_layers][B][Hq][T][D] in the cache dtype")
    hq, T = q.shape[2], q.shape[3]
    if k_new is None or v_new is None:
        raise ValueError("k_new and v_new must be given")
    _expect(k_new, "k_new", (nl, B, H, T, D), cache.k.dtype)
    _expect(v_new, "v_new", (nl, B, H, T, D), cache.k.dtype)
    _expect(n_new, "n_new", (B,), torch.int32)
    _expect(out, "out", (nl, B, hq, T, D), cache.k.dtype)
    _expect(lse, "lse", (nl, B, hq, T), torch.float32)
    _expect_dev_err(dev_err)
    _need_cuda(cache.k, q, k_new, v_new, n_new, out, lse, ws, dev_err)
    if out is None:
        out = torch.zeros_like(q)
    if lse is None and want_lse:
        lse = torch.full((nl, B, hq, T), -math.inf, dtype=torch.float32, device=q.device)
    ws = _ws(lambda: paged_prefill_attn_workspace_size(cache, hq, T, nl), q.device, ws)
    scale = 1.0 / math.sqrt(D) if scale is None else float(scale)
    with _on(q):
        st = load_library().reco_paged_prefill_attn(cache.ref(), layer0, nl, _ptr(q), hq, T, _ptr(n_new), scale,
                                                    sinks, window, _ptr(k_new), _ptr(v_new), _ptr(out),
                                                    _ptr(lse), _ptr(ws), _nbytes(ws), _ptr(dev_err),
                                                    _stream(q.device))
    _check(st, "reco_paged_prefill_attn")
    return out, lse


def reco_paged_evict(cache: PagedKVCache, budget: torch.Tensor, sinks: int = 0, recent: int = 0,
                     kept_idx: Optional[torch.Tensor] = None, layer0: int = 0, n_layers: Optional[int] = None,
                     ws: Optional[torch.Tensor] = None, dev_err: Optional[torch.Tensor] = None):
    """Keep ``budget`` rows of every longer unit, by accumulated weight, the first
    ``sinks`` and the last ``recent`` always; compact K, V and the weights in
    their pages (len <- budget).  ``budget`` is int32 [B] or [n_layers][B]."""
    layer0, nl = _layers(cache, layer0, n_layers)
    sinks, recent = _row_count(sinks, "sinks"), _row_count(recent, "recent")
    NL, Bsz, H, Cap, D = cache.shape
    if cache.weight is None:
        raise ValueError("eviction needs a cache with weights")
    if budget.dtype != torch.int32 or tuple(budget.shape) not in ((Bsz,), (nl, Bsz)):
        raise ValueError("budget must be int32 [B] or [n_layers][B]")
    _expect(kept_idx, "kept_idx", (nl, Bsz, H, Cap), torch.int32)
    _expect_dev_err(dev_err)
    _need_cuda(cache.k, budget, kept_idx, ws, dev_err)
    ws = _ws(lambda: paged_evict_workspace_size(cache, nl), cache.k.device, ws)
    with _on(cache.k):
        st = load_library().reco_paged_evict(cache.ref(), layer0, nl, _ptr(budget), 0 if budget.dim() == 1 else Bsz,
                                             sinks, recent, _ptr(kept_idx), _ptr(ws), _nbytes(ws),
                                             _ptr(dev_err), _stream(cache.k.device))
    _check(st, "reco_paged_evict")
    return kept_idx


class Rope:
    """A rotation by positions: ``inv_freq`` fp32 [rot_dim / 2] on the GPU, radians per
    position of each pair, and the axis of each pair (``axes``, of 0 to 3; none: all
    pairs turn by axis 0).  Pair i is the elements (i, i + rot_dim / 2) of a row, or
    (2 i, 2 i + 1) where ``interleaved``."""

    def __init__(self, inv_freq: torch.Tensor, axes: Optional[Sequence[int]] = None, interleaved: bool = False):
        if inv_freq.dtype != torch.float32 or inv_freq.dim() != 1 or inv_freq.numel() < 1:
            raise ValueError("inv_freq must be float32 [rot_dim / 2]")
        _need_cuda(inv_freq)
        n = inv_freq.numel()
        axes = None if axes is None else [int(a) for a in axes]
        if axes is not None and (len(axes) != n or min(axes) < 0 or max(axes) > 3):
            raise ValueError(f"axes must give each of the {n} pairs an axis of 0 to 3")
        self.inv_freq, self.rot_dim, self.interleaved = inv_freq, 2 * n, bool(interleaved)
        self.n_axes = 1 if axes is None else max(axes) + 1
        self._axes = None if axes is None else (ctypes.c_int32 * n)(*axes)

    def _struct(self, pos: torch.Tensor) -> RecoRope:
        return RecoRope(self.inv_freq.data_ptr(), pos.data_ptr(), self._axes, self.n_axes, self.rot_dim,
                        int(self.interleaved))

    def _check_pos(self, pos: torch.Tensor, batch: int, T: int):
        shapes = [(self.n_axes, batch, T)] + ([(batch, T)] if self.n_axes == 1 else [])
        if T == 1:
            shapes += [x[:-1] for x in shapes]
        if pos is None or pos.dtype != torch.int32 or tuple(pos.shape) not in shapes:
            raise ValueError(f"pos must be int32 [{self.n_axes}][B={batch}][T={T}]")
        _need_cuda(pos, self.inv_freq)


class _Rows:
    """A tensor's rows as the C ABI takes them: [n_layers][B][heads][T][D], or without T
    for one token, in any order of memory whose rows are contiguous and 16-byte aligned."""

    __slots__ = ("what", "shape", "dtype", "index", "struct", "ref", "at", "extent", "_strides",
                 "_piece", "_write")

    def __init__(self, what: str, shape, dtype: torch.dtype, device, write: bool = False):
        self.what, self.shape, self.dtype, self._write = what, tuple(shape), dtype, write
        self.index = device.index if device.type == "cuda" else -1
        self._piece = 4 if dtype == torch.float32 else 8
        self._strides = None
        self.struct = RecoRows()
        self.ref = ctypes.byref(self.struct)

    def take(self, t: torch.Tensor):
        if t.shape != self.shape or t.dtype != self.dtype or t.get_device() != self.index:
            raise ValueError(f"{self.what} must be {_DT.get(self.dtype, self.dtype)} {list(self.shape)} on GPU {self.index}, "
                             f"got {_DT.get(t.dtype, t.dtype)} {list(t.shape)} on {t.device}")
        st = t.stride()
        if st != self._strides:
            self._take_strides(st)
        p = t.data_ptr()
        if p & 15:
            raise ValueError(f"{self.what} must be 16-byte aligned")
        self.at = self.struct.data = p
        return self.ref

    def meets(self, span) -> bool:
        """Whether the rows taken may lie in ``span`` (addresses)."""
        return self.at < span[1] and span[0] < self.at + self.extent

    def _take_strides(self, st):
        if st[-1] != 1 or any(n > 1 and x % self._piece for n, x in zip(self.shape[:-1], st[:-1])):
            raise ValueError(f"{self.what}: rows must be contiguous and multiples of 16 bytes apart")
        used = [x if n > 1 else 0 for n, x in zip(self.shape[:-1], st[:-1])]      # those of one are not used
        if self._write:
            end = self.shape[-1]
            for x, n in sorted((x, n) for n, x in zip(self.shape[:-1], used) if n > 1):
                if x < end:
                    raise ValueError(f"{self.what}: rows must not overlap")
                end = x * (n - 1) + end
        s = self.struct
        self.extent = (16 // self._piece) * (1 + sum((n - 1) * x for n, x in zip(self.shape, st)))
        s.layer, s.seq, s.head = used[:3]
        s.token = used[3] if len(used) == 4 else 0
        self._strides = st


def _launch(index: int, fn, *args) -> int:
    """fn's status, with its GPU as the current one and that one's stream behind the arguments."""
    if torch.cuda.current_device() == index:
        return fn(*args, _stream_of(index))
    with torch.cuda.device(index):
        return fn(*args, _stream_of(index))


def _stream_of(index: int) -> int:
    return _raw_stream(index) if _raw_stream is not None else torch.cuda.current_stream(index).cuda_stream


def _span(t: torch.Tensor):
    at = t.data_ptr()
    return at, at + t.element_size() * (1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride())))


def _no_partial_overlap(x: torch.Tensor, out: torch.Tensor, what: str, same: bool = True):
    """``out`` is x itself (where that is ``same``), or none of its rows meet x's."""
    (a, a1), (b, b1) = _span(x), _span(out)
    if a1 <= b or b1 <= a:
        return
    if same and a == b and x.shape == out.shape and all(n == 1 or s == t for n, s, t in zip(x.shape, x.stride(), out.stride())):
        return
    # heads beside each other, of the same tokens
    d, e, i = b - a, x.element_size(), 2
    others = [j for j in range(x.dim() - 1) if j != i]
    if all(x.shape[j] == out.shape[j] and (x.shape[j] == 1 or x.stride(j) == out.stride(j)) for j in others):
        x1, o1 = (e * ((t.shape[i] - 1) * t.stride(i) + t.shape[-1]) for t in (x, out))
        low, high = (x1, d + o1) if d >= 0 else (o1, x1 - d)      # the lower one's end, the higher one's from the lower's start
        nested = low <= abs(d)
        for st, n in sorted((x.stride(j) * e, x.shape[j]) for j in others if x.shape[j] > 1):
            nested, high = nested and high <= st, st * (n - 1) + high
        if nested:
            return
    raise ValueError(f"{what} must be the same rows as its input or meet none of them" if same else
                     f"{what} must not meet k_new or v_new")


class PreparedRope:
    """reco_rope for a loop that calls it again and again with the same positions
    tensor, output and counts (whose contents may change): those are checked once
    here, each call checks its input.  Calls of several threads take their turns."""

    def __init__(self, rope: Rope, pos: torch.Tensor, out: torch.Tensor, n_new: Optional[torch.Tensor] = None,
                 dev_err: Optional[torch.Tensor] = None):
        if out.dim() not in (4, 5) or out.dtype not in (torch.float32, torch.bfloat16) or out.numel() == 0:
            raise ValueError("rows must be float32 or bfloat16 [NL][B][H][T][D], or without T for one token")
        NL, Bsz, H, *T, D = out.shape
        T = T[0] if T else 1
        if rope.rot_dim > D:
            raise ValueError(f"rot_dim {rope.rot_dim} is larger than a row of {D}")
        rope._check_pos(pos, Bsz, T)
        _expect(n_new, "n_new", (Bsz,), torch.int32)
        _expect_dev_err(dev_err)
        _need_cuda(pos, n_new, dev_err)
        _same_gpu(out, pos)
        self.out = out
        self._keep = (rope, pos, n_new, dev_err)
        self._fn = load_library().reco_rope
        self._struct = rope._struct(pos)
        self._in = _Rows("x", out.shape, out.dtype, out.device)
        self._span = _span(out)
        self._head = ctypes.byref(self._struct)
        self._out = _Rows("out", out.shape, out.dtype, out.device, write=True).take(out)
        self._tail = (NL, Bsz, H, T, D, RECO_F32 if out.dtype == torch.float32 else RECO_BF16, _ptr(n_new),
                      _ptr(dev_err))
        self._lock = threading.Lock()      # of _in, which the library reads without Python's own

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        with self._lock:
            xr = self._in.take(x)
            if self._in.meets(self._span):
                _no_partial_overlap(x, self.out, "out")
            st = _launch(self._in.index, self._fn, self._head, xr, self._out, *self._tail)
        if st != RECO_OK:
            _check(st, "reco_rope")
        return self.out


def reco_rope(rope: Rope, x: torch.Tensor, pos: torch.Tensor, n_new: Optional[torch.Tensor] = None,
              out: Optional[torch.Tensor] = None, dev_err: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Rows x ([NL][B][H][T][D], or [NL][B][H][D] for one token, of any strides whose rows
    are contiguous) rotated by ``pos`` (int32 [B][T], or [n_axes][B][T]); returns ``out``
    (contiguous where none is given; x itself rotates in place).  ``n_new`` int32 [B]: the
    real tokens of each sequence, the first ones; places past them are not written."""
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device) if n_new is None else \
            torch.zeros(x.shape, dtype=x.dtype, device=x.device)
    return PreparedRope(rope, pos, out, n_new, dev_err)(x)


class PreparedPagedAppend:
    """reco_paged_append for a loop that calls it again and again with the same cache,
    positions tensor, rotated queries and counts (whose contents may change): those are
    checked once here, each call checks the new rows.  ``n_tokens`` None: rows without
    the dimension T, one token each.  Calls of several threads take their turns."""

    def __init__(self, cache: PagedKVCache, n_tokens: Optional[int] = None, rope: Optional[Rope] = None,
                 pos: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                 n_new: Optional[torch.Tensor] = None, layer0: int = 0, n_layers: Optional[int] = None,
                 dev_err: Optional[torch.Tensor] = None):
        layer0, nl = _layers(cache, layer0, n_layers)
        NL, Bsz, H, Cap, D = cache.shape
        run = () if n_tokens is None else (_row_count(n_tokens, "n_tokens"),)
        T = run[0] if run else 1
        if T < 1:
            raise ValueError("n_tokens must be 1 or more")
        if (rope is None) != (pos is None):
            raise ValueError("rope and pos must be given together")
        if rope is not None:
            if rope.rot_dim > D:
                raise ValueError(f"rot_dim {rope.rot_dim} is larger than a row of {D}")
            rope._check_pos(pos, Bsz, T)
        dt, dev = cache.k.dtype, cache.k.device
        hq = 0
        if q_out is not None:
            if q_out.dim() != 4 + len(run):
                raise ValueError("q_out must be [n_layers][B][Hq][T][D] (without T for one token)")
            hq = q_out.shape[2]
        _expect(n_new, "n_new", (Bsz,), torch.int32)
        _expect_dev_err(dev_err)
        _need_cuda(cache.k, pos, n_new, dev_err)
        self.cache, self.q_out = cache, q_out
        self._keep = (rope, pos, n_new, dev_err)
        self._fn = load_library().reco_paged_append
        self._k, self._v = (_Rows(what, (nl, Bsz, H, *run, D), dt, dev) for what in ("k_new", "v_new"))
        self._q = self._qo = None
        if q_out is not None:
            shape = (nl, Bsz, hq, *run, D)
            self._q = _Rows("q", shape, dt, dev)
            self._qo = _Rows("q_out", shape, dt, dev, write=True).take(q_out)
            self._span = _span(q_out)
        self._struct = None if rope is None else rope._struct(pos)
        self._head = (cache.ref(), layer0, nl, None if rope is None else ctypes.byref(self._struct), T, _ptr(n_new))
        self._tail = (hq, _ptr(dev_err))
        self._lock = threading.Lock()      # of _k, _v and _q, which the library reads without Python's own

    def __call__(self, k_new: torch.Tensor, v_new: torch.Tensor, q: Optional[torch.Tensor] = None):
        if (q is None) != (self._q is None):
            raise ValueError("q and q_out must be given together")
        with self._lock:
            k, v = self._k.take(k_new), self._v.take(v_new)
            qr = None
            if q is not None:
                qr = self._q.take(q)
                if self._q.meets(self._span):
                    _no_partial_overlap(q, self.q_out, "q_out")
                if self._k.meets(self._span):
                    _no_partial_overlap(k_new, self.q_out, "q_out", same=False)
                if self._v.meets(self._span):
                    _no_partial_overlap(v_new, self.q_out, "q_out", same=False)
            st = _launch(self._k.index, self._fn, *self._head, k, v, qr, self._qo, *self._tail)
        if st != RECO_OK:
            _check(st, "reco_paged_append")
        return self.q_out


def reco_paged_append(cache: PagedKVCache, k_new: torch.Tensor, v_new: torch.Tensor, rope: Optional[Rope] = None,
                      pos: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
                      n_new: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None, layer0: int = 0,
                      n_layers: Optional[int] = None, dev_err: Optional[torch.Tensor] = None):
    """Append rows k_new, v_new ([n_layers][B][H][T][D], or [n_layers][B][H][D] for one
    token, of any strides whose rows are contiguous) to every unit, keys rotated by
    ``rope`` at ``pos`` (int32 [B][T], or [n_axes][B][T]); returns the queries q
    ([n_layers][B][Hq][T][D]) rotated with them (``q_out``, contiguous where none is
    given), or None.  ``n_new`` int32 [B]: the real tokens of each sequence, the first
    ones.  Decode attention without k_new then sees the rows."""
    if k_new.dim() not in (4, 5):
        raise ValueError("k_new must be [n_layers][B][H][T][D] (without T for one token)")
    if q is not None and q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if n_new is None else \
            torch.zeros(q.shape, dtype=q.dtype, device=q.device)
    call = PreparedPagedAppend(cache, k_new.shape[3] if k_new.dim() == 5 else None, rope, pos, q_out, n_new, layer0,
                               n_layers, dev_err)
    return call(k_new, v_new, q)


def _logit_rows(logits: torch.Tensor):
    if logits.dtype != torch.float32 or logits.dim() != 2 or logits.stride(1) != 1 or \
            logits.stride(0) < logits.shape[1]:
        raise ValueError("logits must be fp32 [rows][vocab] with unit column stride and row stride >= vocab")
    return logits.shape


def reco_logit_penalty(logits: torch.Tensor, refl_ids: torch.Tensor, reward: torch.Tensor, tau_lo: float,
                       tau_hi: float, beta_lo: float, beta_mid: float, beta_hi: float,
                       dev_err: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Eq. 3-4 in place on fp32 logits [rows][vocab] (row stride may exceed vocab)."""
    rows, vocab = _logit_rows(logits)
    if refl_ids.dtype != torch.int32 or refl_ids.dim() != 1:
        raise ValueError("refl_ids must be a 1-D int32 tensor")
    _expect(reward, "reward", (rows,), torch.float32)
    _expect_dev_err(dev_err)
    _need_cuda(refl_ids, reward, dev_err)
    _same_gpu(logits, reward)
    st = load_library().reco_logit_penalty(_ptr(logits), rows, vocab, logits.stride(0), _ptr(refl_ids),
                                           refl_ids.numel(), _ptr(reward), tau_lo, tau_hi, beta_lo, beta_mid,
                                           beta_hi, _ptr(dev_err), _stream(logits.device))
    _check(st, "reco_logit_penalty")
    return logits


def reco_penalty_sample(logits: torch.Tensor, refl_ids: Optional[torch.Tensor], reward: torch.Tensor, tau_lo: float,
                        tau_hi: float, beta_lo: float, beta_mid: float, beta_hi: float, temperature: float,
                        seed: int, offset: int, tokens: Optional[torch.Tensor] = None,
                        ws: Optional[torch.Tensor] = None, dev_err: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Eq. 3-4 in place on fp32 logits [rows][vocab], then the next token of
    each row from softmax(z~ / T) (greedy when T = 0); returns tokens [rows] int32."""
    rows, vocab = _logit_rows(logits)
    if refl_ids is not None and (refl_ids.dtype != torch.int32 or refl_ids.dim() != 1):
        raise ValueError("refl_ids must be a 1-D int32 tensor")
    _expect(reward, "reward", (rows,), torch.float32)
    _expect(tokens, "tokens", (rows,), torch.int32)
    _expect_dev_err(dev_err)
    _need_cuda(reward, refl_ids, tokens, ws, dev_err)
    _same_gpu(logits, reward)
    if tokens is None:
        tokens = torch.empty(rows, dtype=torch.int32, device=logits.device)
    ws = _ws(lambda: penalty_sample_workspace_size(rows, vocab), logits.device, ws)
    n_refl = 0 if refl_ids is None else refl_ids.numel()
    st = load_library().reco_penalty_sample(_ptr(logits), rows, vocab, logits.stride(0), _ptr(refl_ids), n_refl,
                                            _ptr(reward), tau_lo, tau_hi, beta_lo, beta_mid, beta_hi,
                                            float(temperature), int(seed) & (2 ** 64 - 1),
                                            int(offset) & (2 ** 64 - 1), _ptr(tokens), _ptr(ws), _nbytes(ws),
                                            _ptr(dev_err), _stream(logits.device))
    _check(st, "reco_penalty_sample")
    return tokens


class PreparedPenaltySample:
    """reco_penalty_sample for a loop over logit rows of one shape (a
    decoder's per-token draw): the reflection ids, the per-row rewards, the
    token output, the workspace and the error word are checked once, and each
    call checks only the logit rows before passing their pointer on, with
    the temperature, seed and draw offset of that call."""

    def __init__(self, rows: int, vocab: int, refl_ids: Optional[torch.Tensor], reward: torch.Tensor,
                 tokens: torch.Tensor, ws: torch.Tensor, dev_err: Optional[torch.Tensor] = None):
        rows, vocab = int(rows), int(vocab)
        if refl_ids is not None and (refl_ids.dtype != torch.int32 or refl_ids.dim() != 1):
            raise ValueError("refl_ids must be a 1-D int32 tensor")
        if tokens is None or ws is None:
            raise ValueError("tokens and ws must be given")
        _expect(reward, "reward", (rows,), torch.float32)
        _expect(tokens, "tokens", (rows,), torch.int32)
        _expect_dev_err(dev_err)
        _need_cuda(reward, refl_ids, tokens, ws, dev_err)
        _same_gpu(tokens, reward)
        if _nbytes(ws) < penalty_sample_workspace_size(rows, vocab):
            raise ValueError("ws is smaller than reco_penalty_sample_workspace_size")
        self.tokens = tokens
        self._keep = (refl_ids, reward, ws, dev_err)
        self._fn = load_library().reco_penalty_sample
        self._dev = reward.device
        self._rows, self._vocab = rows, vocab
        self._ids = (_ptr(refl_ids), 0 if refl_ids is None else refl_ids.numel(), _ptr(reward))
        self._tail = (_ptr(tokens), _ptr(ws), _nbytes(ws), _ptr(dev_err))

    def __call__(self, logits: torch.Tensor, tau_lo: float, tau_hi: float, beta_lo: float, beta_mid: float,
                 beta_hi: float, temperature: float, seed: int, offset: int) -> torch.Tensor:
        if (logits.dtype != torch.float32 or logits.dim() != 2 or tuple(logits.shape) != (self._rows, self._vocab)
                or logits.stride(1) != 1 or logits.stride(0) < self._vocab or logits.device != self._dev):
            raise ValueError(f"logits must be fp32 [{self._rows}][{self._vocab}] with unit column stride on "
                             f"{self._dev}")
        st = self._fn(_ptr(logits), self._rows, self._vocab, logits.stride(0), *self._ids, tau_lo, tau_hi, beta_lo,
                      beta_mid, beta_hi, float(temperature), int(seed) & (2 ** 64 - 1), int(offset) & (2 ** 64 - 1),
                      *self._tail, _stream(self._dev))
        if st != RECO_OK:
            _check(st, "reco_penalty_sample")
        return self.tokens


def reco_answer_ppl(logits: torch.Tensor, tokens: torch.Tensor, tau_p: float, ppl: Optional[torch.Tensor] = None,
                    stop: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                    dev_err: Optional[torch.Tensor] = None):
    """Eq. 5-6: returns (ppl [B] fp32, stop [B] int32)."""
    if logits.dtype != torch.float32 or logits.dim() != 3:
        raise ValueError("logits must be fp32 [B][n][V]")
    B, n, V = logits.shape
    _expect(tokens, "tokens", (B, n), torch.int32)
    _expect(ppl, "ppl", (B,), torch.float32)
    _expect(stop, "stop", (B,), torch.int32)
    _expect_dev_err(dev_err)
    _need_cuda(logits, tokens, ppl, stop, ws, dev_err)
    if ppl is None:
        ppl = torch.empty(B, dtype=torch.float32, device=logits.device)
    if stop is None:
        stop = torch.empty(B, dtype=torch.int32, device=logits.device)
    ws = _ws(lambda: answer_ppl_workspace_size(B, n, V), logits.device, ws)
    st = load_library().reco_answer_ppl(_ptr(logits), _ptr(tokens), B, n, V, tau_p, _ptr(ppl), _ptr(stop),
                                        _ptr(ws), _nbytes(ws), _ptr(dev_err), _stream(logits.device))
    _check(st, "reco_answer_ppl")
    return ppl, stop


def reco_retention_from_reward(v: float, lo: float = 0.3, hi: float = 1.0) -> float:
    return float(load_library().reco_retention_from_reward(float(v), float(lo), float(hi)))


def reco_retention_eq1(v_hist: Sequence[float], lam: float = 0.25, delta: float = 0.1) -> float:
    arr = (ctypes.c_double * len(v_hist))(*[float(x) for x in v_hist])
    return float(load_library().reco_retention_eq1(arr, len(v_hist), float(lam), float(delta)))


def reco_layer_retention(r: float, layer: int, n_layers: int, spread: float) -> float:
    return float(load_library().reco_layer_retention(float(r), int(layer), int(n_layers), float(spread)))


def reco_kept_count(L: int, w: int, r: float) -> int:
    return int(load_library().reco_kept_count(int(L), int(w), float(r)))


def reco_abi_version() -> int:
    return int(load_library().reco_abi_version())
