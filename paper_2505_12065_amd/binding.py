"""ctypes binding of libann.so: the same entry points as include/ann.h, taking
torch device tensors.  Argument marshalling only — shapes, pointers, the current
HIP stream; every step of the search runs in the library's kernels.  There is no
fallback: if the library is missing or a call fails, an exception is raised.

Calls of the usual form are marshalled in native code (csrc/marshal.cpp), which hands every other one back."""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("ANN_LIBRARY_PATH", os.path.join(_HERE, "libann.so"))

ANN_OK, ANN_ERR_INVALID, ANN_ERR_ALIGNMENT, ANN_ERR_UNKNOWN_CORPUS, ANN_ERR_LAUNCH, ANN_ERR_NOMEM = 0, -1, -2, -3, -4, -5
ANN_F16, ANN_BF16, ANN_F32 = 0, 1, 2
ANN_K_MAX, ANN_EF_MAX, ANN_R_MAX, ANN_D_MAX = 16, 16384, 256, 4096
ANN_ENTRIES_MAX = 32
ANN_PAGE_MAX, ANN_HEAD_MAX, ANN_HISTORY_MAX, ANN_BIAS_MAX = 1024, 256, 16777215, 4096

ROTATIONS = {"none": 0, "linear": 1, "base": 2, "ramp": 3, "smooth": 4}      # ANN_ROTATION_* of include/ann.h

_DTYPES = {torch.float16: ANN_F16, torch.bfloat16: ANN_BF16, torch.float32: ANN_F32}

EXPORTS = ("ann_version", "ann_last_error", "ann_flat_search_typed", "ann_flat_search",
           "ann_graph_search_typed", "ann_graph_search", "ann_register_corpus", "ann_unregister_corpus",
           "ann_set_default_dtype", "ann_flat_workspace_bytes", "ann_release_workspace",
           "ann_graph_search_nonstall_typed", "ann_graph_nonstall_workspace_bytes",
           "ann_graph_search_entries_typed", "ann_gather_ids", "ann_timing_enable", "ann_timing_read",
           "ann_measure_mfma_rate", "ann_priority_order", "ann_flat_search_static",
           "ann_graph_search_multi_typed", "ann_timing_read_each",
           "ann_set_workspace", "ann_flat_search_after_typed",
           "ann_qk_norm_rotate", "ann_paged_attention", "ann_paged_attention_workspace_bytes", "ann_cache_evict", "ann_logit_rules",
           "ann_rotation_frequencies", "ann_rotate_append", "ann_chunk_attention", "ann_chunk_attention_workspace_bytes",
           "ann_shared_attention", "ann_shared_attention_workspace_bytes")


class PagedCache(ctypes.Structure):
    """ann_paged_cache of include/ann.h."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p)] + \
        [(name, ctypes.c_int64) for name in ("k_page", "k_head", "k_slot", "v_page", "v_head", "v_slot")] + \
        [(name, ctypes.c_int32) for name in ("pages", "heads", "slots", "d", "dtype")]


class AnnError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"libann error {code}: {message}")
        self.code = code


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2505_12065_amd.build` "
                "(or __graft_entry__.build()); there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        c = ctypes
        vp, i32, i64 = c.c_void_p, c.c_int32, c.c_int64
        L.ann_version.restype = c.c_int
        L.ann_last_error.restype = c.c_char_p
        L.ann_flat_search_typed.argtypes = [vp, i64, i32, i32, vp, i32, i32, vp, vp, vp]
        L.ann_flat_search.argtypes = [vp, i64, i32, vp, i32, i32, vp, vp, vp]
        L.ann_flat_search_after_typed.argtypes = [vp, i64, i32, i32, vp, i32, i32, vp, vp, vp, vp, vp]
        L.ann_flat_search_static.argtypes = [vp, i64, i32, i32, vp, i32, i32, vp, vp, vp]
        L.ann_graph_search_typed.argtypes = [vp, i64, i32, i32, vp, i32, i32, vp, i32, i32, i32, vp, vp, vp]
        L.ann_graph_search.argtypes = [vp, vp, i32, i32, vp, i32, i32, i32, vp, vp, vp]
        L.ann_register_corpus.argtypes = [vp, i64, i32, i32]
        L.ann_unregister_corpus.argtypes = [vp]
        L.ann_set_default_dtype.argtypes = [i32]
        L.ann_flat_workspace_bytes.argtypes = [i64, i32, i32, i32, i32]
        L.ann_flat_workspace_bytes.restype = i64
        L.ann_graph_search_nonstall_typed.argtypes = [vp, i64, i32, i32, vp, i32, i32, vp, i32, i32, i32, vp, i32,
                                                      c.c_float, i32, vp, vp, vp, vp, vp, vp]
        L.ann_graph_search_multi_typed.argtypes = [vp, i64, i32, i32, vp, i32, vp, i32, vp, i32, i32, i32, vp, vp, vp]
        L.ann_graph_search_entries_typed.argtypes = [vp, i64, i32, i32, vp, i32, vp, vp, i32, i32, i32, vp, vp, vp]
        L.ann_gather_ids.argtypes = [vp, i64, vp, i64, vp, vp]
        L.ann_measure_mfma_rate.argtypes = [i32, i32, c.POINTER(c.c_double)]
        L.ann_priority_order.argtypes = [vp, vp, vp, vp, i32, i32, vp, vp, vp]
        L.ann_set_workspace.argtypes = [vp, i64]
        L.ann_timing_enable.argtypes = [i32]
        L.ann_timing_read.argtypes = [i32, c.POINTER(i32), c.POINTER(c.c_double)]
        L.ann_timing_read_each.argtypes = [i32, i32, c.POINTER(i32), c.POINTER(c.c_float)]
        L.ann_graph_nonstall_workspace_bytes.argtypes = [i64, i32]
        L.ann_graph_nonstall_workspace_bytes.restype = i64
        f32, cache = c.c_float, c.POINTER(PagedCache)
        L.ann_qk_norm_rotate.argtypes = [vp, i64, i64, i32, i32, vp, vp, f32, vp, vp, i32, i32, i32, vp, cache, vp, vp]
        L.ann_paged_attention.argtypes = [vp, i64, i64, i32, i32, cache, vp, i32, vp, i32, f32, i32, vp, vp, vp, i64, vp]
        L.ann_paged_attention_workspace_bytes.argtypes = [i32] * 7
        L.ann_paged_attention_workspace_bytes.restype = i64
        L.ann_cache_evict.argtypes = [cache, vp, i32, vp, i32, vp, i64, vp, i32, i32, i32, i32, vp, vp, vp, i64, vp]
        L.ann_logit_rules.argtypes = [vp, i64, i32, i32, i32, vp, i32, vp, vp, vp, vp, vp, vp, vp, i32, vp, i32, vp, vp, i64, vp]
        f64 = c.c_double
        L.ann_rotation_frequencies.argtypes = [i32, f64, i32, f64, i32, f64, f64, vp, vp]
        L.ann_rotate_append.argtypes = [vp, i64, i64, i32, i32, vp, i32, vp, vp, i32, vp, vp, i32, f32, i32, cache, vp, vp]
        L.ann_chunk_attention.argtypes = [vp, i64, i64, i32, i32, vp, i32, cache, vp, i32, vp, i32, f32, i32, vp, vp, vp]
        L.ann_chunk_attention_workspace_bytes.argtypes = [i32] * 8
        L.ann_chunk_attention_workspace_bytes.restype = i64
        L.ann_shared_attention.argtypes = [vp, i64, i64, i32, i32, cache, vp, i32, vp, vp, vp, i32, i32, i32, f32, vp, vp, vp]
        L.ann_shared_attention_workspace_bytes.argtypes = [i32] * 8
        L.ann_shared_attention_workspace_bytes.restype = i64
        for name in EXPORTS:
            if name not in ("ann_last_error", "ann_flat_workspace_bytes", "ann_graph_nonstall_workspace_bytes",
                            "ann_paged_attention_workspace_bytes", "ann_chunk_attention_workspace_bytes", "ann_shared_attention_workspace_bytes"):
                getattr(L, name).restype = c.c_int
        _lib = L
        _load_marshal(L)
    return _lib


_marshal = None


def _load_marshal(L: ctypes.CDLL) -> None:
    """csrc/marshal.cpp is built against one torch and one Python; where it is not there, does not load or was built for others, every
    call is marshalled here."""
    global _marshal
    from . import build                                  # (here: the package does not import what `python -m` runs)
    path = os.path.join(_HERE, "_marshal.so")
    try:
        loader = importlib.machinery.ExtensionFileLoader("_marshal", path)
        module = importlib.util.module_from_spec(importlib.util.spec_from_file_location("_marshal", path, loader=loader))
        loader.exec_module(module)
    except ImportError:
        return
    if getattr(module, "built_for", None) != build.marshal_target():
        return
    module.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in
                  (L.ann_flat_search_typed, L.ann_flat_search_after_typed, L.ann_graph_search_typed, L.ann_graph_search_entries_typed,
                   L.ann_graph_search_nonstall_typed, L.ann_gather_ids, L.ann_priority_order)))
    module.bind_many(*(ctypes.cast(f, ctypes.c_void_p).value for f in (L.ann_rotate_append, L.ann_chunk_attention, L.ann_shared_attention)))
    module.bind_decode(*(ctypes.cast(f, ctypes.c_void_p).value for f in
                         (L.ann_qk_norm_rotate, L.ann_paged_attention, L.ann_cache_evict, L.ann_logit_rules)))
    _marshal = module


def _check(rc: int) -> None:
    if rc != ANN_OK:
        raise AnnError(rc, lib().ann_last_error().decode())


# The stream's handle without a Stream object around it (2.5 us), where this torch has the call for it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _usual(function: str, first, *rest):
    """What csrc/marshal.cpp answers to a call on the current device and stream; None: it is not of the usual form."""
    if not getattr(first, "is_cuda", False):
        return None
    lib()
    if _marshal is None:
        return None
    device = _current_device()
    out = getattr(_marshal, function)(first, *rest, device, _raw_stream(device))
    if type(out) is int:
        _check(out)
    return out


def _stream(stream, index: int) -> int:
    if stream is None:
        return _raw_stream(index)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _call(device: torch.device, stream, entry_point, *args) -> None:
    """entry_point(*args, stream) with `device` current.  (A torch.cuda.device block costs 1.2 us even where it
    changes nothing, and small searches are bound by what runs here, so it is entered only where it does.)"""
    index = device.index
    if torch.cuda.current_device() == index:
        rc = entry_point(*args, _stream(stream, index))
    else:
        with torch.cuda.device(device):
            rc = entry_point(*args, _stream(stream, index))
    if rc != ANN_OK:
        _check(rc)


def _outputs(B: int, k: int, device, ids, scores):
    if ids is None:
        ids = torch.empty(B, k, dtype=torch.int32, device=device)
    elif ids.shape != (B, k) or ids.dtype != torch.int32 or not ids.is_contiguous() or not ids.is_cuda:
        raise ValueError("ids must be a contiguous int32 [B, k] device tensor")
    if scores is None:
        scores = torch.empty(B, k, dtype=torch.float32, device=device)
    elif scores.shape != (B, k) or scores.dtype != torch.float32 or not scores.is_contiguous() or not scores.is_cuda:
        raise ValueError("scores must be a contiguous float32 [B, k] device tensor")
    return ids, scores


def _matrix(t: torch.Tensor, name: str) -> torch.Tensor:
    if t.dim() != 2 or not t.is_cuda or not t.is_contiguous() or t.dtype not in _DTYPES:
        raise ValueError(f"{name} must be a contiguous 2-D fp16/bf16/fp32 device tensor")
    return t


def ann_version() -> int:
    return lib().ann_version()


def ann_last_error() -> str:
    return lib().ann_last_error().decode()


def ann_flat_search_typed(corpus: torch.Tensor, queries: torch.Tensor, k: int, *, after=None, ids=None, scores=None,
                          stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Exact top-k of every query over the corpus; element type taken from the tensors.
    after = (scores float32 [B], ids int32 [B]) device tensors: the continuation entry point, the k best rows
    that come strictly after that pair in the order."""
    if ids is None and scores is None and stream is None:
        out = None
        if after is None:
            out = _usual("flat", corpus, queries, k, None, None)
        elif type(after) is tuple and len(after) == 2 and after[0] is not None:
            out = _usual("flat", corpus, queries, k, *after)
        if out is not None:
            return out
    _matrix(corpus, "corpus"), _matrix(queries, "queries")
    if queries.dtype != corpus.dtype or queries.shape[1] != corpus.shape[1]:
        raise ValueError("queries must have the corpus' element type and dimension")
    (N, d), B = corpus.shape, queries.shape[0]
    ids, scores = _outputs(B, k, corpus.device, ids, scores)
    if after is None:
        _call(corpus.device, stream, lib().ann_flat_search_typed, corpus.data_ptr(), N, d, _DTYPES[corpus.dtype],
              queries.data_ptr(), B, k, ids.data_ptr(), scores.data_ptr())
    else:
        a_s, a_i = after
        if a_s.dtype != torch.float32 or a_i.dtype != torch.int32 or tuple(a_s.shape) != (B,) or tuple(a_i.shape) != (B,) \
                or not (a_s.is_cuda and a_i.is_cuda and a_s.is_contiguous() and a_i.is_contiguous()):
            raise ValueError("after must be (float32 [B], int32 [B]) contiguous device tensors")
        _call(corpus.device, stream, lib().ann_flat_search_after_typed, corpus.data_ptr(), N, d, _DTYPES[corpus.dtype],
              queries.data_ptr(), B, k, a_s.data_ptr(), a_i.data_ptr(), ids.data_ptr(), scores.data_ptr())
    return ids, scores


ANN_STATIC_WORKSPACE_BYTES = 8 * 1024 * 1024


def ann_flat_search_static(corpus: torch.Tensor, queries: torch.Tensor, k: int, *, ids: torch.Tensor,
                           scores: torch.Tensor, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Exact top-k through the entry point that allocates nothing: the caller brings ids and
    scores, the workspace is the library's static array."""
    _matrix(corpus, "corpus"), _matrix(queries, "queries")
    if queries.dtype != corpus.dtype or queries.shape[1] != corpus.shape[1]:
        raise ValueError("queries must have the corpus' element type and dimension")
    (N, d), B = corpus.shape, queries.shape[0]
    ids, scores = _outputs(B, k, corpus.device, ids, scores)
    _call(corpus.device, stream, lib().ann_flat_search_static, corpus.data_ptr(), N, d, _DTYPES[corpus.dtype],
          queries.data_ptr(), B, k, ids.data_ptr(), scores.data_ptr())
    return ids, scores


def ann_flat_search(corpus: torch.Tensor, queries: torch.Tensor, k: int, *, ids=None, scores=None,
                    stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Exact top-k through the short entry point, which assumes the library's default
    element type (fp16 unless ann_set_default_dtype changed it)."""
    _matrix(corpus, "corpus"), _matrix(queries, "queries")
    if queries.dtype != corpus.dtype or queries.shape[1] != corpus.shape[1]:
        raise ValueError("queries must have the corpus' element type and dimension")
    (N, d), B = corpus.shape, queries.shape[0]
    ids, scores = _outputs(B, k, corpus.device, ids, scores)
    _call(corpus.device, stream, lib().ann_flat_search, corpus.data_ptr(), N, d, queries.data_ptr(), B, k, ids.data_ptr(),
          scores.data_ptr())
    return ids, scores


def _graph(graph: torch.Tensor, N: int) -> torch.Tensor:
    if graph.dim() != 2 or graph.dtype != torch.int32 or not graph.is_cuda or not graph.is_contiguous() \
            or graph.shape[0] != N:
        raise ValueError("graph must be a contiguous int32 [N, R] device tensor")
    return graph


def ann_graph_search_typed(corpus: torch.Tensor, graph: torch.Tensor, entry: int, queries: torch.Tensor, k: int,
                           ef: int, *, ids=None, scores=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Best-first graph search with a candidate list of ef entries."""
    if ids is None and scores is None and stream is None:
        out = _usual("graph", corpus, graph, entry, queries, k, ef)
        if out is not None:
            return out
    _matrix(corpus, "corpus"), _matrix(queries, "queries")
    if queries.dtype != corpus.dtype or queries.shape[1] != corpus.shape[1]:
        raise ValueError("queries must have the corpus' element type and dimension")
    (N, d), B = corpus.shape, queries.shape[0]
    _graph(graph, N)
    ids, scores = _outputs(B, k, corpus.device, ids, scores)
    _call(corpus.device, stream, lib().ann_graph_search_typed, corpus.data_ptr(), N, d, _DTYPES[corpus.dtype],
          graph.data_ptr(), graph.shape[1], int(entry), queries.data_ptr(), B, k, ef, ids.data_ptr(), scores.data_ptr())
    return ids, scores


def ann_graph_search_nonstall_typed(corpus: torch.Tensor, graph: torch.Tensor, entry: int, queries: torch.Tensor,
                                    k: int, ef: int, *, entries: Optional[torch.Tensor] = None, tau: float = 0.9,
                                    window: int = 500, engine_ready: Optional[torch.Tensor] = None, ids=None, scores=None,
                                    stats=None, ema=None, stream=None):
    """Graph search with the maturity (non-stall) exit.  `engine_ready` is an int32 tensor of one
    element on the device or in pinned host memory (None = always ready).  Returns
    (ids, scores, stats [B,3] = (early, scored, expansions), ema [B])."""
    if engine_ready is None and ids is None and scores is None and stats is None and ema is None and stream is None:
        out = _usual("nonstall", corpus, graph, entry, queries, k, ef, entries, tau, window)
        if out is not None:
            return out
    _matrix(corpus, "corpus"), _matrix(queries, "queries")
    if queries.dtype != corpus.dtype or queries.shape[1] != corpus.shape[1]:
        raise ValueError("queries must have the corpus' element type and dimension")
    (N, d), B = corpus.shape, queries.shape[0]
    _graph(graph, N)
    ids, scores = _outputs(B, k, corpus.device, ids, scores)
    if stats is None:
        stats = torch.empty(B, 3, dtype=torch.int32, device=corpus.device)
    if ema is None:
        ema = torch.empty(B, dtype=torch.float32, device=corpus.device)
    if stats.dtype != torch.int32 or tuple(stats.shape) != (B, 3) or not stats.is_contiguous() or not stats.is_cuda:
        raise ValueError("stats must be a contiguous int32 [B, 3] device tensor")
    if ema.dtype != torch.float32 or tuple(ema.shape) != (B,) or not ema.is_contiguous() or not ema.is_cuda:
        raise ValueError("ema must be a contiguous float32 [B] device tensor")
    entries_ptr, n_entries = 0, 0
    if entries is not None:
        entries_ptr, n_entries = _entries(entries, B).data_ptr(), (1 if entries.dim() == 1 else entries.shape[1])
    ready_ptr = 0
    if engine_ready is not None:
        if engine_ready.dtype != torch.int32 or engine_ready.numel() != 1 or \
                not (engine_ready.is_cuda or engine_ready.is_pinned()):
            raise ValueError("engine_ready must be one int32 on the device or in pinned host memory")
        ready_ptr = engine_ready.data_ptr()
    _call(corpus.device, stream, lib().ann_graph_search_nonstall_typed, corpus.data_ptr(), N, d, _DTYPES[corpus.dtype],
          graph.data_ptr(), graph.shape[1], int(entry), queries.data_ptr(), B, k, ef, entries_ptr, n_entries, float(tau),
          int(window), ready_ptr, ids.data_ptr(), scores.data_ptr(), stats.data_ptr(), ema.data_ptr())
    return ids, scores, stats, ema


def _entries(entries: torch.Tensor, B: int) -> torch.Tensor:
    ok_shape = tuple(entries.shape) == (B,) or (entries.dim() == 2 and entries.shape[0] == B and entries.shape[1] >= 1)
    if entries.dtype != torch.int32 or not ok_shape or not entries.is_contiguous() or not entries.is_cuda:
        raise ValueError("entries must be a contiguous int32 [B] or [B, E] device tensor")
    return entries


def ann_graph_search_multi_typed(corpus: torch.Tensor, graph: torch.Tensor, entries: torch.Tensor,
                                 queries: torch.Tensor, k: int, ef: int, *, ids=None, scores=None,
                                 stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Graph search with entries[B, E] entry nodes per query."""
    _matrix(corpus, "corpus"), _matrix(queries, "queries")
    if queries.dtype != corpus.dtype or queries.shape[1] != corpus.shape[1]:
        raise ValueError("queries must have the corpus' element type and dimension")
    (N, d), B = corpus.shape, queries.shape[0]
    _graph(graph, N)
    _entries(entries, B)
    if entries.dim() != 2:
        raise ValueError("entries must be [B, E]")
    ids, scores = _outputs(B, k, corpus.device, ids, scores)
    _call(corpus.device, stream, lib().ann_graph_search_multi_typed, corpus.data_ptr(), N, d, _DTYPES[corpus.dtype],
          graph.data_ptr(), graph.shape[1], entries.data_ptr(), entries.shape[1], queries.data_ptr(), B, k, ef,
          ids.data_ptr(), scores.data_ptr())
    return ids, scores


def ann_graph_search_entries_typed(corpus: torch.Tensor, graph: torch.Tensor, entries: torch.Tensor,
                                   queries: torch.Tensor, k: int, ef: int, *, ids=None, scores=None,
                                   stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Graph search with one entry node per query."""
    if ids is None and scores is None and stream is None:
        out = _usual("graph_entries", corpus, graph, entries, queries, k, ef)
        if out is not None:
            return out
    _matrix(corpus, "corpus"), _matrix(queries, "queries")
    if queries.dtype != corpus.dtype or queries.shape[1] != corpus.shape[1]:
        raise ValueError("queries must have the corpus' element type and dimension")
    (N, d), B = corpus.shape, queries.shape[0]
    _graph(graph, N)
    if _entries(entries, B).dim() != 1:
        raise ValueError("entries must be [B]")
    ids, scores = _outputs(B, k, corpus.device, ids, scores)
    _call(corpus.device, stream, lib().ann_graph_search_entries_typed, corpus.data_ptr(), N, d, _DTYPES[corpus.dtype],
          graph.data_ptr(), graph.shape[1], entries.data_ptr(), queries.data_ptr(), B, k, ef, ids.data_ptr(),
          scores.data_ptr())
    return ids, scores


def ann_gather_ids(table: torch.Tensor, idx: torch.Tensor, *, out=None, stream=None) -> torch.Tensor:
    """out[i] = table[idx[i]] (-1 where idx[i] is out of range); int32 device tensors."""
    if out is None and stream is None:
        usual = _usual("gather", table, idx)
        if usual is not None:
            return usual[0]
    for t in (table, idx):
        if t.dtype != torch.int32 or not t.is_contiguous() or not t.is_cuda:
            raise ValueError("table and idx must be contiguous int32 device tensors")
    if out is None:
        out = torch.empty_like(idx)
    if out.dtype != torch.int32 or out.shape != idx.shape or not out.is_contiguous() or not out.is_cuda:
        raise ValueError("out must be a contiguous int32 device tensor shaped like idx")
    _call(table.device, stream, lib().ann_gather_ids, table.data_ptr(), table.numel(), idx.data_ptr(), idx.numel(),
          out.data_ptr())
    return out


KERNEL_FLAT_STREAM, KERNEL_FLAT_WIDE, KERNEL_FLAT_F32, KERNEL_GRAPH = 0, 1, 2, 3


def ann_priority_order(R: torch.Tensor, W: torch.Tensor, C: torch.Tensor, Wcur: torch.Tensor, G: int = 6, *,
                       stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Scheduler priority levels and execution order.  R, C int32 [n]; W, Wcur float64 [n]; device tensors."""
    if stream is None:
        out = _usual("order", R, W, C, Wcur, G)
        if out is not None:
            return out
    n = R.numel()
    for t, dt in ((R, torch.int32), (C, torch.int32), (W, torch.float64), (Wcur, torch.float64)):
        if t.dtype != dt or t.numel() != n or not t.is_contiguous() or not t.is_cuda:
            raise ValueError("R, C must be int32 and W, Wcur float64 contiguous device tensors of one length")
    level = torch.empty(n, dtype=torch.int32, device=R.device)
    order = torch.empty(n, dtype=torch.int32, device=R.device)
    _call(R.device, stream, lib().ann_priority_order, R.data_ptr(), W.data_ptr(), C.data_ptr(), Wcur.data_ptr(), n, int(G),
          level.data_ptr(), order.data_ptr())
    return level, order


def ann_measure_mfma_rate(random_operands: bool, iters: int = 100000) -> float:
    """Dense fp16 MFMA rate (TFLOP/s) the current device sustains on register operands."""
    out = ctypes.c_double(0.0)
    _check(lib().ann_measure_mfma_rate(1 if random_operands else 0, int(iters), ctypes.byref(out)))
    return out.value


def ann_timing_enable(on: bool) -> None:
    _check(lib().ann_timing_enable(1 if on else 0))


def ann_timing_read(kernel: int) -> Tuple[int, float]:
    """(launches, total milliseconds) of the main kernel `kernel` since timing was switched on."""
    n, ms = ctypes.c_int32(0), ctypes.c_double(0.0)
    _check(lib().ann_timing_read(kernel, ctypes.byref(n), ctypes.byref(ms)))
    return n.value, ms.value


def ann_timing_read_each(kernel: int):
    """Durations (ms) of the recorded launches of the main kernel `kernel`, in call order."""
    n = ctypes.c_int32(0)
    _check(lib().ann_timing_read_each(kernel, 0, ctypes.byref(n), None))
    buf = (ctypes.c_float * max(1, n.value))()
    _check(lib().ann_timing_read_each(kernel, n.value, ctypes.byref(n), buf))
    return [buf[i] for i in range(n.value)]


def ann_graph_nonstall_workspace_bytes(N: int, B: int) -> int:
    return int(lib().ann_graph_nonstall_workspace_bytes(N, B))


def ann_graph_search(corpus: torch.Tensor, graph: torch.Tensor, entry: int, queries: torch.Tensor, k: int, ef: int,
                     *, ids=None, scores=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Graph search through the short entry point: the corpus must have been registered."""
    _matrix(queries, "queries")
    B = queries.shape[0]
    ids, scores = _outputs(B, k, queries.device, ids, scores)
    _call(queries.device, stream, lib().ann_graph_search, corpus.data_ptr(), graph.data_ptr(), graph.shape[1], int(entry),
          queries.data_ptr(), B, k, ef, ids.data_ptr(), scores.data_ptr())
    return ids, scores


def ann_register_corpus(corpus: torch.Tensor) -> None:
    _matrix(corpus, "corpus")
    _check(lib().ann_register_corpus(corpus.data_ptr(), corpus.shape[0], corpus.shape[1], _DTYPES[corpus.dtype]))


def ann_unregister_corpus(corpus: torch.Tensor) -> None:
    _check(lib().ann_unregister_corpus(corpus.data_ptr()))


def ann_set_default_dtype(dtype: torch.dtype) -> None:
    _check(lib().ann_set_default_dtype(_DTYPES[dtype]))


def ann_flat_workspace_bytes(N: int, d: int, dtype: torch.dtype, B: int, k: int) -> int:
    return int(lib().ann_flat_workspace_bytes(N, d, _DTYPES[dtype], B, k))


def ann_set_workspace(buf: Optional[torch.Tensor]) -> None:
    """Use `buf` (a contiguous uint8 device tensor the caller keeps alive) as the workspace of its device;
    None hands the workspace back to the library.  An exact search that wants more (ann_flat_workspace_bytes) runs in parts,
    down to parts of 8192 rows; what does not fit even so raises."""
    if buf is None:
        _check(lib().ann_set_workspace(None, 0))
        return
    if buf.dtype != torch.uint8 or not buf.is_cuda or not buf.is_contiguous():
        raise ValueError("the workspace must be a contiguous uint8 device tensor")
    with torch.cuda.device(buf.device):
        _check(lib().ann_set_workspace(buf.data_ptr(), buf.numel()))


def ann_release_workspace() -> None:
    _check(lib().ann_release_workspace())


# ---- the step between two retrievals ---------------------------------------------------------

def _array(t: torch.Tensor, name: str, dtype: torch.dtype, shape) -> torch.Tensor:
    """A contiguous device tensor of that type and shape (-1: any size)."""
    if t.dtype != dtype or not t.is_cuda or not t.is_contiguous() or t.dim() != len(shape) or \
            any(w not in (-1, n) for w, n in zip(shape, t.shape)):
        raise ValueError(f"{name} must be a contiguous {str(dtype).replace('torch.', '')} device tensor of shape "
                         f"{['any' if w == -1 else w for w in shape]}")
    return t


def _rows(t: torch.Tensor, name: str, dtype: torch.dtype, shape) -> torch.Tensor:
    """A device tensor of that type and shape whose last dimension is contiguous."""
    if t.dtype != dtype or not t.is_cuda or t.dim() != len(shape) or any(w not in (-1, n) for w, n in zip(shape, t.shape)) or \
            (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name} must be a {str(dtype).replace('torch.', '')} device tensor of shape "
                         f"{['any' if w == -1 else w for w in shape]} whose rows are contiguous")
    return t


def _strides(t: torch.Tensor):
    """Strides of all dimensions but the last, 0 for those of size 1, which torch leaves anything."""
    return [s if n > 1 else 0 for s, n in zip(t.stride()[:-1], t.shape)]


def _int32(x, name: str) -> int:
    """x as an int that the C call takes as it is (ctypes keeps the low 32 bits of a larger one, without a word)."""
    x = int(x)
    if not -2 ** 31 <= x < 2 ** 31:
        raise ValueError(f"{name} = {x} does not fit 32 bits")
    return x


def _cache(k_cache: torch.Tensor, v_cache: torch.Tensor) -> PagedCache:
    for t, name in ((k_cache, "k_cache"), (v_cache, "v_cache")):
        if t.dim() != 4 or not t.is_cuda or t.dtype not in _DTYPES or (t.shape[3] > 1 and t.stride(3) != 1):
            raise ValueError(f"{name} must be an fp16/bf16/fp32 device tensor [pages, heads, slots, d] whose rows are contiguous")
    if k_cache.shape != v_cache.shape or k_cache.dtype != v_cache.dtype or k_cache.device != v_cache.device:
        raise ValueError("k_cache and v_cache must have one shape and element type and be on one device")
    pages, heads, slots, d = k_cache.shape
    return PagedCache(k_cache.data_ptr(), v_cache.data_ptr(), *_strides(k_cache), *_strides(v_cache),
                      pages, heads, slots, d, _DTYPES[k_cache.dtype])


def _same_device(first: torch.Tensor, *others) -> None:
    if any(t is not None and t.device != first.device for t in others):
        raise ValueError("all tensors must be on one device")


def ann_qk_norm_rotate(qkv: torch.Tensor, q_weight: torch.Tensor, k_weight: torch.Tensor, positions: torch.Tensor,
                       cos_sin: torch.Tensor, slots: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, *,
                       eps: float = 1e-6, interleaved: bool = False, q=None, stream=None) -> torch.Tensor:
    """Norms of queries and keys for each head, the rotation by position, and the write of keys and values into the paged
    cache [pages, heads, slots, d].  qkv is [T, query heads + 2 heads, d], cos_sin float32 [positions, rot], cosines before
    sines; positions and slots int32 [T].  Returns the queries [T, query heads, d]."""
    if q is None and stream is None:
        usual = _usual("rotate", qkv, q_weight, k_weight, positions, cos_sin, slots, k_cache, v_cache, eps, interleaved)
        if usual is not None:
            return usual[0]
    cache = _cache(k_cache, v_cache)
    dtype, heads, d = k_cache.dtype, cache.heads, cache.d
    _rows(qkv, "qkv", dtype, (-1, -1, d))
    T, q_heads = qkv.shape[0], qkv.shape[1] - 2 * heads
    if q_heads < 1:
        raise ValueError("qkv must have query heads and the cache's heads twice")
    _array(q_weight, "q_weight", dtype, (d,)), _array(k_weight, "k_weight", dtype, (d,))
    _array(positions, "positions", torch.int32, (T,)), _array(slots, "slots", torch.int32, (T,))
    _array(cos_sin, "cos_sin", torch.float32, (-1, -1))
    if q is None:
        q = torch.empty(T, q_heads, d, dtype=dtype, device=qkv.device)
    _array(q, "q", dtype, (T, q_heads, d))
    _same_device(k_cache, qkv, q_weight, k_weight, positions, cos_sin, slots, q)
    _call(qkv.device, stream, lib().ann_qk_norm_rotate, qkv.data_ptr(), *_strides(qkv), T, q_heads, q_weight.data_ptr(),
          k_weight.data_ptr(), float(eps), positions.data_ptr(), cos_sin.data_ptr(), cos_sin.shape[0], cos_sin.shape[1],
          1 if interleaved else 0, slots.data_ptr(), ctypes.byref(cache), q.data_ptr())
    return q


def ann_paged_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, page_table: torch.Tensor,
                        lengths: torch.Tensor, *, scale: Optional[float] = None, window: int = 0, max_length: Optional[int] = None,
                        mass: Optional[torch.Tensor] = None, out=None, lse=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention of one new token per request over its paged cache.  q [B, query heads, d], page_table int32 [B, pages of a
    request], lengths int32 [B]; scale 1 / sqrt(d) unless given; max_length: the largest length, or a bound as close as
    is known, which decides how the work is divided (else all that the page table holds, which costs time where contexts are much shorter).  mass
    float32 [B, heads, slots]: the weight of every slot is added to it.  Long contexts and weights use the device's one workspace, as some searches do: such
    calls on several streams have to be ordered (ann_set_workspace).  Returns (out [B, query heads, d], lse float32 [B, query heads])."""
    if out is None and lse is None and stream is None:
        usual = _usual("attend", q, k_cache, v_cache, page_table, lengths, scale, window, max_length, mass)
        if usual is not None:
            return usual
    cache = _cache(k_cache, v_cache)
    d = cache.d
    _rows(q, "q", k_cache.dtype, (-1, -1, d))
    B, q_heads = q.shape[:2]
    _array(page_table, "page_table", torch.int32, (B, -1)), _array(lengths, "lengths", torch.int32, (B,))
    if mass is not None:
        _array(mass, "mass", torch.float32, (B, cache.heads, -1))
    width = page_table.shape[1]
    out = torch.empty(B, q_heads, d, dtype=q.dtype, device=q.device) if out is None else _array(out, "out", q.dtype, (B, q_heads, d))
    lse = torch.empty(B, q_heads, dtype=torch.float32, device=q.device) if lse is None else _array(lse, "lse", torch.float32, (B, q_heads))
    _same_device(k_cache, q, page_table, lengths, mass, out, lse)
    _call(q.device, stream, lib().ann_paged_attention, q.data_ptr(), *_strides(q), B, q_heads, ctypes.byref(cache),
          page_table.data_ptr(), width, lengths.data_ptr(), width * cache.slots if max_length is None else _int32(max_length, "max_length"),
          d ** -0.5 if scale is None else float(scale), _int32(window, "window"), out.data_ptr(), lse.data_ptr(),
          0 if mass is None else mass.data_ptr(), 0 if mass is None else mass.shape[2])
    return out, lse


def ann_paged_attention_workspace_bytes(B: int, q_heads: int, heads: int, d: int, dtype: torch.dtype, max_length: int,
                                        with_mass: bool = False) -> int:
    sizes = [_int32(x, name) for x, name in ((B, "B"), (q_heads, "q_heads"), (heads, "heads"), (d, "d"))]
    return int(lib().ann_paged_attention_workspace_bytes(*sizes, _DTYPES[dtype], _int32(max_length, "max_length"), 1 if with_mass else 0))


def ann_cache_evict(k_cache: torch.Tensor, v_cache: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor,
                    mass: torch.Tensor, new_page_table: torch.Tensor, budget: int, *, first: int = 0, recent: int = 0,
                    stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """The `budget` slots of every request and cache head that had the most attention (mass float32 [B, heads, slots]), its first
    `first` and last `recent` among them, copied to the pages of new_page_table.  Returns (kept int32 [B, heads, budget], -1 behind
    the last; new lengths int32 [B]; the kept slots' mass float32 [B, heads, new slots], 0 behind them)."""
    if stream is None:
        usual = _usual("evict", k_cache, v_cache, page_table, lengths, mass, new_page_table, budget, first, recent)
        if usual is not None:
            return usual
    cache = _cache(k_cache, v_cache)
    _array(page_table, "page_table", torch.int32, (-1, -1))
    B, device, budget = page_table.shape[0], k_cache.device, _int32(budget, "budget")
    _array(lengths, "lengths", torch.int32, (B,)), _array(mass, "mass", torch.float32, (B, cache.heads, -1))
    _array(new_page_table, "new_page_table", torch.int32, (B, -1))
    _same_device(k_cache, page_table, lengths, mass, new_page_table)
    new_slots = new_page_table.shape[1] * cache.slots
    kept = torch.empty(B, cache.heads, max(0, budget), dtype=torch.int32, device=device)
    new_lengths = torch.empty(B, dtype=torch.int32, device=device)
    new_mass = torch.empty(B, cache.heads, new_slots, dtype=torch.float32, device=device)
    _call(device, stream, lib().ann_cache_evict, ctypes.byref(cache), page_table.data_ptr(), page_table.shape[1], lengths.data_ptr(), B,
          mass.data_ptr(), mass.shape[2], new_page_table.data_ptr(), new_page_table.shape[1], budget, _int32(first, "first"), _int32(recent, "recent"),
          kept.data_ptr(), new_lengths.data_ptr(), new_mass.data_ptr(), new_slots)
    return kept, new_lengths, new_mass


def ann_logit_rules(logits: torch.Tensor, tokens: torch.Tensor, lengths: torch.Tensor, prompt_lengths: torch.Tensor,
                    repetition: torch.Tensor, presence: torch.Tensor, frequency: torch.Tensor, *,
                    bias_tokens: Optional[torch.Tensor] = None, bias_values: Optional[torch.Tensor] = None,
                    masks: Optional[torch.Tensor] = None, mask_rows: Optional[torch.Tensor] = None, out=None,
                    stream=None) -> torch.Tensor:
    """Penalties for repeated tokens, biases and grammar masks on logits [B, V] (fp16, bf16 or fp32).  tokens int32 [B, T], of which
    lengths[b] count, the first prompt_lengths[b] of them as given (prompt and retrieved passages) and not chosen; repetition, presence, frequency float32 [B]; bias_tokens int32
    and bias_values float32 [B, K]; masks int32 [M, ceil(V / 32)], a bit for each token, 1: allowed, and mask_rows int32 [B] into it,
    -1: no mask.  out may be logits.  Returns out."""
    if out is None and stream is None:
        usual = _usual("rules", logits, tokens, lengths, prompt_lengths, repetition, presence, frequency, bias_tokens, bias_values,
                       masks, mask_rows)
        if usual is not None:
            return usual[0]
    if logits.dtype not in _DTYPES:
        raise ValueError("logits must be an fp16/bf16/fp32 device tensor")
    _rows(logits, "logits", logits.dtype, (-1, -1))
    B, V = logits.shape
    _array(tokens, "tokens", torch.int32, (B, -1)), _array(lengths, "lengths", torch.int32, (B,))
    _array(prompt_lengths, "prompt_lengths", torch.int32, (B,))
    for t, name in ((repetition, "repetition"), (presence, "presence"), (frequency, "frequency")):
        _array(t, name, torch.float32, (B,))
    K, M = 0, 0
    if bias_tokens is not None or bias_values is not None:
        if bias_tokens is None or bias_values is None:
            raise ValueError("bias_tokens and bias_values go together")
        K = _array(bias_tokens, "bias_tokens", torch.int32, (B, -1)).shape[1]
        _array(bias_values, "bias_values", torch.float32, (B, K))
    if masks is not None or mask_rows is not None:
        if masks is None or mask_rows is None:
            raise ValueError("masks and mask_rows go together")
        M = _array(masks, "masks", torch.int32, (-1, (V + 31) // 32)).shape[0]
        _array(mask_rows, "mask_rows", torch.int32, (B,))
    out = torch.empty(B, V, dtype=logits.dtype, device=logits.device) if out is None else _rows(out, "out", logits.dtype, (B, V))
    _same_device(logits, tokens, lengths, prompt_lengths, repetition, presence, frequency, bias_tokens, bias_values, masks, mask_rows, out)
    _call(logits.device, stream, lib().ann_logit_rules, logits.data_ptr(), logits.stride(0) if B > 1 else V, B, V, _DTYPES[logits.dtype],
          tokens.data_ptr(), tokens.shape[1], lengths.data_ptr(), prompt_lengths.data_ptr(), repetition.data_ptr(),
          presence.data_ptr(), frequency.data_ptr(), bias_tokens.data_ptr() if K else 0, bias_values.data_ptr() if K else 0, K,
          masks.data_ptr() if M else 0, M, mask_rows.data_ptr() if M else 0, out.data_ptr(), out.stride(0) if B > 1 else V)
    return out


# ---- many tokens at once ---------------------------------------------------------------------

def ann_rotation_frequencies(rot: int, base: float = 10_000.0, *, scaling: str = "none", factor: float = 1.0, original: int = 0,
                             low: float = 1.0, high: float = 32.0, device=None) -> Tuple[torch.Tensor, float]:
    """(frequencies float64 [rot / 2], amplitude) of a rotation, as ann_rotate_append takes them; scaling for contexts longer than the
    `original` length: "none", "linear", "base", "ramp" (by the pair's number, between those that turn `high` and `low` times in the original context) or "smooth" (by
    the turns themselves).  On the CPU unless a device is given."""
    if scaling not in ROTATIONS:
        raise ValueError(f"scaling must be one of {list(ROTATIONS)}")
    frequencies, amplitude = torch.empty(max(0, _int32(rot, "rot") // 2), dtype=torch.float64), ctypes.c_double(1.0)
    _check(lib().ann_rotation_frequencies(rot, float(base), ROTATIONS[scaling], float(factor), _int32(original, "original"), float(low), float(high),
                                          frequencies.data_ptr(), ctypes.byref(amplitude)))
    return (frequencies if device is None else frequencies.to(device)), amplitude.value


def ann_rotate_append(qkv: torch.Tensor, starts: torch.Tensor, lengths: torch.Tensor, page_table: torch.Tensor, frequencies: Optional[torch.Tensor],
                      k_cache: torch.Tensor, v_cache: torch.Tensor, *, positions: Optional[torch.Tensor] = None, amplitude: float = 1.0,
                      interleaved: bool = False, q=None, stream=None) -> torch.Tensor:
    """The rotation of queries and keys by position and the write of keys and values behind what each request holds in the paged cache
    [pages, heads, slots, d].  qkv is [T, query heads + 2 heads, d], request b's tokens being starts[b] to starts[b + 1] - 1 (int32 [B + 1]) and the last of the
    lengths[b] slots that it then has; page_table int32 [B, pages of a request]; frequencies float64 [rot / 2] on the device (None: nothing is rotated); positions int32 [T]
    where they are not the slots.  Returns the queries [T, query heads, d]; rows of tokens that are no request's are left as they were."""
    if q is None and stream is None:
        usual = _usual("append", qkv, starts, lengths, page_table, frequencies, k_cache, v_cache, positions, amplitude, interleaved)
        if usual is not None:
            return usual[0]
    cache = _cache(k_cache, v_cache)
    dtype, heads, d = k_cache.dtype, cache.heads, cache.d
    _rows(qkv, "qkv", dtype, (-1, -1, d))
    T, q_heads = qkv.shape[0], qkv.shape[1] - 2 * heads
    if q_heads < 1:
        raise ValueError("qkv must have query heads and the cache's heads twice")
    B = _array(lengths, "lengths", torch.int32, (-1,)).shape[0]
    _array(starts, "starts", torch.int32, (B + 1,)), _array(page_table, "page_table", torch.int32, (B, -1))
    if positions is not None:
        _array(positions, "positions", torch.int32, (T,))
    if frequencies is not None:
        _array(frequencies, "frequencies", torch.float64, (-1,))
    if q is None:
        q = torch.empty(T, q_heads, d, dtype=dtype, device=qkv.device)
    _array(q, "q", dtype, (T, q_heads, d))
    _same_device(k_cache, qkv, starts, lengths, page_table, frequencies, positions, q)
    _call(qkv.device, stream, lib().ann_rotate_append, qkv.data_ptr(), *_strides(qkv), T, q_heads, starts.data_ptr(), B, lengths.data_ptr(),
          page_table.data_ptr(), page_table.shape[1], 0 if positions is None else positions.data_ptr(), 0 if frequencies is None else frequencies.data_ptr(),
          0 if frequencies is None else 2 * frequencies.shape[0], float(amplitude), 1 if interleaved else 0, ctypes.byref(cache), q.data_ptr())
    return q


def ann_chunk_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor,
                        starts: torch.Tensor, *, scale: Optional[float] = None, window: int = 0, max_length: Optional[int] = None, out=None, lse=None,
                        stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention of every request's new tokens over its paged cache, each up to its own slot.  q [T, query heads, d], request b's tokens being starts[b] to
    starts[b + 1] - 1 (int32 [B + 1]) and the last of its lengths[b] slots; page_table int32 [B, pages of a request]; scale 1 / sqrt(d) unless given; max_length: the
    largest length, or a bound as close as is known (else all that the page table holds).  Few tokens of long contexts use the device's one workspace, as some searches do: such calls on
    several streams have to be ordered (ann_set_workspace).  Returns (out [T, query heads, d], lse float32 [T, query heads]); rows of tokens that are no request's are left
    as they were."""
    if out is None and lse is None and stream is None:
        usual = _usual("chunk", q, k_cache, v_cache, page_table, lengths, starts, scale, window, max_length)
        if usual is not None:
            return usual
    cache = _cache(k_cache, v_cache)
    d = cache.d
    _rows(q, "q", k_cache.dtype, (-1, -1, d))
    T, q_heads = q.shape[:2]
    B = _array(lengths, "lengths", torch.int32, (-1,)).shape[0]
    _array(page_table, "page_table", torch.int32, (B, -1)), _array(starts, "starts", torch.int32, (B + 1,))
    width = page_table.shape[1]
    out = torch.empty(T, q_heads, d, dtype=q.dtype, device=q.device) if out is None else _array(out, "out", q.dtype, (T, q_heads, d))
    lse = torch.empty(T, q_heads, dtype=torch.float32, device=q.device) if lse is None else _array(lse, "lse", torch.float32, (T, q_heads))
    _same_device(k_cache, q, page_table, lengths, starts, out, lse)
    _call(q.device, stream, lib().ann_chunk_attention, q.data_ptr(), *_strides(q), T, q_heads, starts.data_ptr(), B, ctypes.byref(cache), page_table.data_ptr(),
          width, lengths.data_ptr(), width * cache.slots if max_length is None else _int32(max_length, "max_length"), d ** -0.5 if scale is None else float(scale),
          _int32(window, "window"), out.data_ptr(), lse.data_ptr())
    return out, lse


def ann_chunk_attention_workspace_bytes(T: int, B: int, q_heads: int, heads: int, d: int, dtype: torch.dtype, max_length: int, window: int = 0) -> int:
    sizes = [_int32(x, name) for x, name in ((T, "T"), (B, "B"), (q_heads, "q_heads"), (heads, "heads"), (d, "d"))]
    return int(lib().ann_chunk_attention_workspace_bytes(*sizes, _DTYPES[dtype], _int32(max_length, "max_length"), _int32(window, "window")))


def ann_shared_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor,
                         group_starts: torch.Tensor, shared: torch.Tensor, *, max_shared: Optional[int] = None, max_own: Optional[int] = None,
                         scale: Optional[float] = None, out=None, lse=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention of one new token per request over its paged cache, where the requests group_starts[g] to group_starts[g + 1] - 1 (int32 [groups + 1]) have their first shared[g] (int32
    [groups]) slots in common, which are then read once for the group.  q [B, query heads, d], page_table int32 [B, pages of a request], lengths int32 [B]; max_shared and max_own: the
    largest numbers of shared and of own slots, or bounds as close as are known (else all that the page table holds).  Uses the device's one workspace: such calls on several
    streams have to be ordered (ann_set_workspace).  Returns (out [B, query heads, d], lse float32 [B, query heads])."""
    if out is None and lse is None and stream is None:
        usual = _usual("shared", q, k_cache, v_cache, page_table, lengths, group_starts, shared, max_shared, max_own, scale)
        if usual is not None:
            return usual
    cache = _cache(k_cache, v_cache)
    d = cache.d
    _rows(q, "q", k_cache.dtype, (-1, -1, d))
    B, q_heads = q.shape[:2]
    _array(page_table, "page_table", torch.int32, (B, -1)), _array(lengths, "lengths", torch.int32, (B,))
    groups = _array(shared, "shared", torch.int32, (-1,)).shape[0]
    _array(group_starts, "group_starts", torch.int32, (groups + 1,))
    width = page_table.shape[1]
    out = torch.empty(B, q_heads, d, dtype=q.dtype, device=q.device) if out is None else _array(out, "out", q.dtype, (B, q_heads, d))
    lse = torch.empty(B, q_heads, dtype=torch.float32, device=q.device) if lse is None else _array(lse, "lse", torch.float32, (B, q_heads))
    _same_device(k_cache, q, page_table, lengths, group_starts, shared, out, lse)
    bounds = [width * cache.slots if x is None else _int32(x, name) for x, name in ((max_shared, "max_shared"), (max_own, "max_own"))]
    _call(q.device, stream, lib().ann_shared_attention, q.data_ptr(), *_strides(q), B, q_heads, ctypes.byref(cache), page_table.data_ptr(), width,
          lengths.data_ptr(), group_starts.data_ptr(), shared.data_ptr(), groups, *bounds, d ** -0.5 if scale is None else float(scale), out.data_ptr(), lse.data_ptr())
    return out, lse


def ann_shared_attention_workspace_bytes(B: int, groups: int, q_heads: int, heads: int, d: int, dtype: torch.dtype, max_shared: int, max_own: int) -> int:
    sizes = [_int32(x, name) for x, name in ((B, "B"), (groups, "groups"), (q_heads, "q_heads"), (heads, "heads"), (d, "d"))]
    return int(lib().ann_shared_attention_workspace_bytes(*sizes, _DTYPES[dtype], _int32(max_shared, "max_shared"), _int32(max_own, "max_own")))
