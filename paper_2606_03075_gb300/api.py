"""Python binding of the TGV-KV C ABI (include/tgvkv.h).

Argument marshalling only: each function checks that the torch tensors have
the dtype, device, contiguity and size the C call expects, passes their device
pointers and the current CUDA stream, and raises on a non-zero return code.
Every step of the computation runs in the library's CUDA kernels.  PyTorch
provides device memory and streams.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import math
from dataclasses import dataclass

import torch

from . import _lib

Desc = _lib.Desc

_BF16_LIKE = (torch.bfloat16, torch.int16, torch.uint16)


class TgvkvError(RuntimeError):
    def __init__(self, code, fn):
        msg = _lib.load().tgvkv_last_error().decode()
        super().__init__(f"{fn} failed with code {code}: {msg}")
        self.code = code


BASIS = {"vision": _lib.BASIS_VISION, "all": _lib.BASIS_ALL}
WEIGHTS = {"given": _lib.WEIGHTS_GIVEN, "eq7": _lib.WEIGHTS_EQ7}
STAT = {"tv": _lib.STAT_TV, "tt": _lib.STAT_TT, "uniform": _lib.STAT_UNIFORM}


def make_desc(L, H_q, H_kv, d, N, N_v, n_win, softmax_scale=0.0, w_layer_stride=None,
              basis="vision", weights="given", keep_first=0, keep_last=0, stat="tv",
              head_budgets=False) -> Desc:
    """A problem descriptor; w_layer_stride defaults to n_win (one weight row per layer).

    basis: "vision" (r counts vision KV, every text KV kept) or "all" (r counts
    every KV, both cases of Eq. 10); weights: "given" (the caller's w~) or
    "eq7" (tgvkv_evict derives w~ by Eq. 7); keep_first / keep_last: sinks;
    stat: the statistic the layer budgets follow, "tv" / "tt" / "uniform";
    head_budgets: one budget per (layer, KV head) (tvb_stat and budgets then
    hold L * H_kv entries)."""
    return Desc(L=L, H_q=H_q, H_kv=H_kv, d=d, N=N, N_v=N_v, n_win=n_win,
                softmax_scale=float(softmax_scale),
                w_layer_stride=n_win if w_layer_stride is None else w_layer_stride,
                budget_basis=BASIS[basis], weight_mode=WEIGHTS[weights],
                keep_first=keep_first, keep_last=keep_last, budget_stat=STAT[stat],
                head_budgets=int(bool(head_budgets)))


def budget_units(desc: Desc) -> int:
    """Entries of tvb_stat and budgets: L, or L * H_kv with head budgets."""
    return desc.L * desc.H_kv if desc.head_budgets else desc.L


def desc_for_workload(wl, softmax_scale=0.0, **options) -> Desc:
    return make_desc(wl.L, wl.H_q, wl.H_kv, wl.d, wl.N, wl.N_v, wl.n_win, softmax_scale,
                     **options)


# The current stream's handle without a Stream object around it (which costs 5 us a
# call).  Not public names: where a torch lacks them, the public way is taken.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is None or _raw_device is None:
            return torch.cuda.current_stream().cuda_stream
        return _raw_stream(_raw_device())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _ptr(t, dtypes, numel, name):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}, expected one of {dtypes}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.numel() < numel:
        raise ValueError(f"{name} holds {t.numel()} elements, needs {numel}")
    return t.data_ptr()


def _check(code, fn):
    if code != 0:
        raise TgvkvError(code, fn)


def tgvkv_workspace_size(desc: Desc) -> int:
    n = _lib.load().tgvkv_workspace_size(ctypes.byref(desc))
    if n == 0:
        raise TgvkvError(-1, "tgvkv_workspace_size")
    return int(n)


def tgvkv_vision_budget_total(desc: Desc, ratio: float) -> int:
    n = _lib.load().tgvkv_vision_budget_total(ctypes.byref(desc), float(ratio))
    if n < 0:
        raise TgvkvError(-1, "tgvkv_vision_budget_total")
    return int(n)


def tgvkv_budget_total(desc: Desc, ratio: float) -> int:
    n = _lib.load().tgvkv_budget_total(ctypes.byref(desc), float(ratio))
    if n < 0:
        raise TgvkvError(-1, "tgvkv_budget_total")
    return int(n)


def tgvkv_retained_rows(desc: Desc, ratio: float) -> int:
    n = _lib.load().tgvkv_retained_rows(ctypes.byref(desc), float(ratio))
    if n < 0:
        raise TgvkvError(-1, "tgvkv_retained_rows")
    return int(n)


def tgvkv_workspace_init(desc: Desc, ws: torch.Tensor, stream=None):
    p = _ptr(ws, (torch.uint8,), tgvkv_workspace_size(desc), "workspace")
    _check(_lib.load().tgvkv_workspace_init(ctypes.byref(desc), p, _stream(stream)),
           "tgvkv_workspace_init")


def _named(device):
    """The device of an allocating call: the current one where none is named."""
    return "cuda" if device is None else device


def _on(t):
    """The tensor's device made the current one: what a call starts runs on the current
    device and its stream."""
    return torch.cuda.device(t.device) if t.is_cuda else contextlib.nullcontext()


def new_workspace(desc: Desc, device=None) -> torch.Tensor:
    """A zeroed workspace tensor (uint8) for this problem."""
    ws = torch.empty(tgvkv_workspace_size(desc), dtype=torch.uint8, device=_named(device))
    with _on(ws):
        tgvkv_workspace_init(desc, ws)
    return ws


def tgvkv_score(desc, q_text, k, modality, text_pos, w, scores, tvb_stat, ws, stream=None):
    L, Hq, Hkv, d, N, Nv, nw = desc.L, desc.H_q, desc.H_kv, desc.d, desc.N, desc.N_v, desc.n_win
    wrows = (L - 1) * desc.w_layer_stride + nw if nw else 0
    _check(_lib.load().tgvkv_score(
        ctypes.byref(desc),
        _ptr(q_text, _BF16_LIKE, L * Hq * nw * d, "q_text"),
        _ptr(k, _BF16_LIKE, L * Hkv * N * d, "k"),
        _ptr(modality, (torch.uint8,), N, "modality"),
        _ptr(text_pos, (torch.int32,), nw, "text_pos"),
        _ptr(w, (torch.float32,), wrows, "w"),
        _ptr(scores, (torch.float32,), L * Hkv * Nv, "scores"),
        _ptr(tvb_stat, (torch.float32,), budget_units(desc), "tvb_stat"),
        _ptr(ws, (torch.uint8,), tgvkv_workspace_size(desc), "workspace"),
        _stream(stream)), "tgvkv_score")


def tgvkv_text_scores(desc, q_text, k, modality, text_pos, text_scores, weights, ws, stream=None):
    L, Hq, Hkv, d, N, nw = desc.L, desc.H_q, desc.H_kv, desc.d, desc.N, desc.n_win
    _check(_lib.load().tgvkv_text_scores(
        ctypes.byref(desc),
        _ptr(q_text, _BF16_LIKE, L * Hq * nw * d, "q_text"),
        _ptr(k, _BF16_LIKE, L * Hkv * N * d, "k"),
        _ptr(modality, (torch.uint8,), N, "modality"),
        _ptr(text_pos, (torch.int32,), nw, "text_pos"),
        _ptr(text_scores, (torch.float32,), L * Hkv * (N - desc.N_v), "text_scores"),
        _ptr(weights, (torch.float32,), L * nw, "weights"),
        _ptr(ws, (torch.uint8,), tgvkv_workspace_size(desc), "workspace"),
        _stream(stream)), "tgvkv_text_scores")


def tgvkv_budget(desc, tvb_stat, ratio, budgets, ws, stream=None):
    _check(_lib.load().tgvkv_budget(
        ctypes.byref(desc),
        _ptr(tvb_stat, (torch.float32,), budget_units(desc), "tvb_stat"), float(ratio),
        _ptr(budgets, (torch.int32,), budget_units(desc), "budgets"),
        _ptr(ws, (torch.uint8,), tgvkv_workspace_size(desc), "workspace"),
        _stream(stream)), "tgvkv_budget")


def tgvkv_select(desc, scores, budgets, modality, offsets, idx, ws, stream=None):
    LH = desc.L * desc.H_kv
    _check(_lib.load().tgvkv_select(
        ctypes.byref(desc),
        _ptr(scores, (torch.float32,), LH * desc.N_v, "scores"),
        _ptr(budgets, (torch.int32,), budget_units(desc), "budgets"),
        _ptr(modality, (torch.uint8,), desc.N, "modality"),
        _ptr(offsets, (torch.int64,), LH + 1, "offsets"),
        _ptr(idx, (torch.int32,), 0, "idx"),
        _ptr(ws, (torch.uint8,), tgvkv_workspace_size(desc), "workspace"),
        _stream(stream)), "tgvkv_select")


def tgvkv_select_tpr(desc, scores, text_scores, budgets, modality, offsets, idx, ws, stream=None):
    LH = desc.L * desc.H_kv
    _check(_lib.load().tgvkv_select_tpr(
        ctypes.byref(desc),
        _ptr(scores, (torch.float32,), LH * desc.N_v, "scores"),
        _ptr(text_scores, (torch.float32,), LH * (desc.N - desc.N_v), "text_scores"),
        _ptr(budgets, (torch.int32,), budget_units(desc), "budgets"),
        _ptr(modality, (torch.uint8,), desc.N, "modality"),
        _ptr(offsets, (torch.int64,), LH + 1, "offsets"),
        _ptr(idx, (torch.int32,), 0, "idx"),
        _ptr(ws, (torch.uint8,), tgvkv_workspace_size(desc), "workspace"),
        _stream(stream)), "tgvkv_select_tpr")


def tgvkv_compact(desc, k, v, offsets, idx, k_out, v_out, ws, stream=None):
    n = desc.L * desc.H_kv * desc.N * desc.d
    capacity = min(k_out.numel(), v_out.numel()) // desc.d   # rows of the outputs
    _check(_lib.load().tgvkv_compact(
        ctypes.byref(desc),
        _ptr(k, _BF16_LIKE, n, "k"), _ptr(v, _BF16_LIKE, n, "v"),
        _ptr(offsets, (torch.int64,), desc.L * desc.H_kv + 1, "offsets"),
        _ptr(idx, (torch.int32,), 0, "idx"),
        _ptr(k_out, _BF16_LIKE, 0, "k_out"), _ptr(v_out, _BF16_LIKE, 0, "v_out"),
        capacity,
        _ptr(ws, (torch.uint8,), tgvkv_workspace_size(desc), "workspace"),
        _stream(stream)), "tgvkv_compact")


def tgvkv_select_compact(desc, scores, text_scores, budgets, modality, k, v, offsets, idx,
                         k_out, v_out, ws, stream=None):
    LH = desc.L * desc.H_kv
    n = LH * desc.N * desc.d
    # rows every output holds: k_out, v_out and idx alike
    capacity = min(k_out.numel() // desc.d, v_out.numel() // desc.d, idx.numel())
    _check(_lib.load().tgvkv_select_compact(
        ctypes.byref(desc),
        _ptr(scores, (torch.float32,), LH * desc.N_v, "scores"),
        _ptr(text_scores, (torch.float32,), LH * (desc.N - desc.N_v), "text_scores"),
        _ptr(budgets, (torch.int32,), budget_units(desc), "budgets"),
        _ptr(modality, (torch.uint8,), desc.N, "modality"),
        _ptr(k, _BF16_LIKE, n, "k"), _ptr(v, _BF16_LIKE, n, "v"),
        _ptr(offsets, (torch.int64,), LH + 1, "offsets"),
        _ptr(idx, (torch.int32,), 0, "idx"),
        _ptr(k_out, _BF16_LIKE, 0, "k_out"), _ptr(v_out, _BF16_LIKE, 0, "v_out"),
        capacity,
        _ptr(ws, (torch.uint8,), tgvkv_workspace_size(desc), "workspace"),
        _stream(stream)), "tgvkv_select_compact")


def tgvkv_select_compact_launches(desc: Desc) -> int:
    return int(_lib.load().tgvkv_select_compact_launches(ctypes.byref(desc)))


@dataclass
class EvictOutputs:
    scores: torch.Tensor     # fp32 [L, H_kv, N_v]
    tvb_stat: torch.Tensor   # fp32 [L]
    budgets: torch.Tensor    # int32 [L]
    offsets: torch.Tensor    # int64 [L*H_kv + 1]
    idx: torch.Tensor        # int32 [retained rows]
    k_out: torch.Tensor      # bf16 [retained rows, d]
    v_out: torch.Tensor      # bf16 [retained rows, d]


def alloc_outputs(desc: Desc, ratio: float, device=None) -> EvictOutputs:
    dev = _named(device)
    rows = tgvkv_retained_rows(desc, ratio)
    L, Hkv = desc.L, desc.H_kv
    return EvictOutputs(
        scores=torch.empty((L, Hkv, desc.N_v), dtype=torch.float32, device=dev),
        tvb_stat=torch.empty(budget_units(desc), dtype=torch.float32, device=dev),
        budgets=torch.empty(budget_units(desc), dtype=torch.int32, device=dev),
        offsets=torch.empty(L * Hkv + 1, dtype=torch.int64, device=dev),
        idx=torch.empty(max(rows, 1), dtype=torch.int32, device=dev),
        k_out=torch.empty((max(rows, 1), desc.d), dtype=torch.bfloat16, device=dev),
        v_out=torch.empty((max(rows, 1), desc.d), dtype=torch.bfloat16, device=dev))


def tgvkv_evict(desc, q_text, k, v, modality, text_pos, w, ratio, out: EvictOutputs, ws,
                stream=None):
    L, Hq, Hkv, d, N, Nv, nw = desc.L, desc.H_q, desc.H_kv, desc.d, desc.N, desc.N_v, desc.n_win
    rows = tgvkv_retained_rows(desc, ratio)
    wrows = (L - 1) * desc.w_layer_stride + nw if nw else 0
    _check(_lib.load().tgvkv_evict(
        ctypes.byref(desc),
        _ptr(q_text, _BF16_LIKE, L * Hq * nw * d, "q_text"),
        _ptr(k, _BF16_LIKE, L * Hkv * N * d, "k"),
        _ptr(v, _BF16_LIKE, L * Hkv * N * d, "v"),
        _ptr(modality, (torch.uint8,), N, "modality"),
        _ptr(text_pos, (torch.int32,), nw, "text_pos"),
        _ptr(w, (torch.float32,), wrows, "w"),
        float(ratio),
        _ptr(out.scores, (torch.float32,), L * Hkv * Nv, "scores"),
        _ptr(out.tvb_stat, (torch.float32,), budget_units(desc), "tvb_stat"),
        _ptr(out.budgets, (torch.int32,), budget_units(desc), "budgets"),
        _ptr(out.offsets, (torch.int64,), L * Hkv + 1, "offsets"),
        _ptr(out.idx, (torch.int32,), rows, "idx"),
        _ptr(out.k_out, _BF16_LIKE, rows * d, "k_out"),
        _ptr(out.v_out, _BF16_LIKE, rows * d, "v_out"),
        _ptr(ws, (torch.uint8,), tgvkv_workspace_size(desc), "workspace"),
        _stream(stream)), "tgvkv_evict")


def tgvkv_evict_with_stats(desc, q_text, k, v, modality, text_pos, w, ratio, row_stats,
                           out: EvictOutputs, ws, stream=None):
    """tgvkv_evict with the query rows' (m, Z, vision mass) from tgvkv_prefill."""
    L, Hq, Hkv, d, N, Nv, nw = desc.L, desc.H_q, desc.H_kv, desc.d, desc.N, desc.N_v, desc.n_win
    rows = tgvkv_retained_rows(desc, ratio)
    wrows = (L - 1) * desc.w_layer_stride + nw if nw else 0
    _check(_lib.load().tgvkv_evict_with_stats(
        ctypes.byref(desc),
        _ptr(q_text, _BF16_LIKE, L * Hq * nw * d, "q_text"),
        _ptr(k, _BF16_LIKE, L * Hkv * N * d, "k"),
        _ptr(v, _BF16_LIKE, L * Hkv * N * d, "v"),
        _ptr(modality, (torch.uint8,), N, "modality"),
        _ptr(text_pos, (torch.int32,), nw, "text_pos"),
        _ptr(w, (torch.float32,), wrows, "w"),
        float(ratio),
        _ptr(row_stats, (torch.float32,), 3 * L * Hq * nw, "row_stats"),
        _ptr(out.scores, (torch.float32,), L * Hkv * Nv, "scores"),
        _ptr(out.tvb_stat, (torch.float32,), budget_units(desc), "tvb_stat"),
        _ptr(out.budgets, (torch.int32,), budget_units(desc), "budgets"),
        _ptr(out.offsets, (torch.int64,), L * Hkv + 1, "offsets"),
        _ptr(out.idx, (torch.int32,), rows, "idx"),
        _ptr(out.k_out, _BF16_LIKE, rows * d, "k_out"),
        _ptr(out.v_out, _BF16_LIKE, rows * d, "v_out"),
        _ptr(ws, (torch.uint8,), tgvkv_workspace_size(desc), "workspace"),
        _stream(stream)), "tgvkv_evict_with_stats")


def tgvkv_prefill(desc, q, k, v, modality, text_pos, o, q_text, row_stats, ws, stream=None):
    """Causal prefill attention over every token, plus the eviction step's query
    rows (q_text) and their (m, Z, vision mass) (see include/tgvkv.h)."""
    L, Hq, Hkv, d, N, nw = desc.L, desc.H_q, desc.H_kv, desc.d, desc.N, desc.n_win
    _check(_lib.load().tgvkv_prefill(
        ctypes.byref(desc),
        _ptr(q, _BF16_LIKE, L * Hq * N * d, "q"),
        _ptr(k, _BF16_LIKE, L * Hkv * N * d, "k"),
        _ptr(v, _BF16_LIKE, L * Hkv * N * d, "v"),
        _ptr(modality, (torch.uint8,), N, "modality"),
        _ptr(text_pos, (torch.int32,), nw, "text_pos"),
        _ptr(o, _BF16_LIKE, L * Hq * N * d, "o"),
        _ptr(q_text, _BF16_LIKE, L * Hq * nw * d, "q_text"),
        _ptr(row_stats, (torch.float32,), 3 * L * Hq * nw, "row_stats"),
        _ptr(ws, (torch.uint8,), tgvkv_workspace_size(desc), "workspace"),
        _stream(stream)), "tgvkv_prefill")


def tgvkv_check_wait_timeout(ws: torch.Tensor, stream=None):
    """Launch the failure-detection self-test: a bounded wait that runs out and
    sets TGVKV_STATUS_TIMEOUT in the workspace's status word."""
    _check(_lib.load().tgvkv_check_wait_timeout(_ptr(ws, (torch.uint8,), 4, "workspace"),
                                                _stream(stream)), "tgvkv_check_wait_timeout")


def tgvkv_status(ws: torch.Tensor, stream=None) -> int:
    """Synchronise the stream, return and clear the device status bits."""
    rc = _lib.load().tgvkv_status(_ptr(ws, (torch.uint8,), 4, "workspace"), _stream(stream))
    if rc < 0:
        raise TgvkvError(-rc, "tgvkv_status")
    return rc


def tgvkv_decode(desc, q, k_rows, v_rows, offsets, out, ws, stream=None):
    """One decode step of every layer over a CSR cache (see include/tgvkv.h)."""
    L, Hq, Hkv, d = desc.L, desc.H_q, desc.H_kv, desc.d
    capacity = min(k_rows.numel(), v_rows.numel()) // d
    _check(_lib.load().tgvkv_decode(
        ctypes.byref(desc),
        _ptr(q, _BF16_LIKE, L * Hq * d, "q"),
        _ptr(k_rows, _BF16_LIKE, 0, "k_rows"),
        _ptr(v_rows, _BF16_LIKE, 0, "v_rows"),
        capacity,
        _ptr(offsets, (torch.int64,), L * Hkv + 1, "offsets"),
        _ptr(out, (torch.float32,), L * Hq * d, "out"),
        _ptr(ws, (torch.uint8,), tgvkv_workspace_size(desc), "workspace"),
        _stream(stream)), "tgvkv_decode")


def tgvkv_decode_launches(desc: Desc) -> int:
    return int(_lib.load().tgvkv_decode_launches(ctypes.byref(desc)))


def tgvkv_evict_launches(desc: Desc) -> int:
    """Kernels one tgvkv_evict call launches for this problem."""
    n = _lib.load().tgvkv_evict_launches(ctypes.byref(desc))
    if n < 0:
        raise TgvkvError(-1, "tgvkv_evict_launches")
    return int(n)


# ---- the paged cache ---------------------------------------------------------

CacheDesc = _lib.CacheDesc
CACHE_FORMAT = {"bf16": _lib.CACHE_BF16, "int8": _lib.CACHE_INT8, "int4": _lib.CACHE_INT4,
                "fp4": _lib.CACHE_FP4}
CACHE_GROUP = 32   # values that share a scale

# format -> (dtypes a pool may have, pool elements per row of d values)
_POOL = {_lib.CACHE_BF16: (_BF16_LIKE, lambda d: d),
         _lib.CACHE_INT8: ((torch.int8, torch.uint8), lambda d: d),
         _lib.CACHE_INT4: ((torch.uint8,), lambda d: d // 2),
         _lib.CACHE_FP4: ((torch.uint8,), lambda d: d // 2)}


def make_cache_desc(B, H_q, H_kv, d, page_size, n_pages, max_pages, format="bf16",
                    softmax_scale=0.0) -> CacheDesc:
    """A paged cache's descriptor (include/tgvkv.h).

    B: sequences (the requests of a batch, or the layers of one); page_size:
    slots per page (16 to 256, a power of two); n_pages: pages of the pool;
    max_pages: page-table entries of a set; format: "bf16", "int8", "int4" or "fp4"
    (4-bit floats)."""
    return CacheDesc(B=B, H_q=H_q, H_kv=H_kv, d=d, page_size=page_size, n_pages=n_pages,
                     max_pages=max_pages, format=CACHE_FORMAT[format],
                     softmax_scale=float(softmax_scale))


@dataclass
class PagedCache:
    k: torch.Tensor                      # [n_pages, page_size, d] (int4, fp4: d / 2)
    v: torch.Tensor
    k_scale: torch.Tensor | None = None  # uint8 [n_pages, page_size, d / 32]; None for bf16
    v_scale: torch.Tensor | None = None


def alloc_cache(desc: CacheDesc, device=None) -> PagedCache:
    """Pools of this descriptor's geometry and format (uninitialised)."""
    dev = _named(device)
    dtypes, row = _POOL[desc.format]
    pool = (desc.n_pages, desc.page_size, row(desc.d))
    scale = (desc.n_pages, desc.page_size, desc.d // CACHE_GROUP)
    quantised = desc.format != _lib.CACHE_BF16
    new = [torch.empty(pool, dtype=dtypes[0], device=dev) for _ in range(2)]
    new += [torch.empty(scale, dtype=torch.uint8, device=dev) if quantised else None
            for _ in range(2)]
    return PagedCache(*new)


@functools.lru_cache(maxsize=256)
def _cache_geometry(fields: bytes):
    """Of a descriptor (its bytes): workspace bytes (0: rejected), sets, page-table
    entries, elements of a pool and of a scale pool (0: none)."""
    d = CacheDesc.from_buffer_copy(fields)
    ws = int(_lib.load().tgvkv_cache_workspace_size(ctypes.byref(d)))
    if ws == 0:
        return 0, 0, 0, 0, 0
    slots, sets = d.n_pages * d.page_size, d.B * d.H_kv
    scale = 0 if d.format == _lib.CACHE_BF16 else slots * (d.d // CACHE_GROUP)
    return ws, sets, sets * d.max_pages, slots * _POOL[d.format][1](d.d), scale


def _geometry(desc, fn):
    geo = _cache_geometry(bytes(desc))
    if geo[0] == 0:
        # asked again, as the library's message is that of its last call
        _lib.load().tgvkv_cache_workspace_size(ctypes.byref(desc))
        raise TgvkvError(-1, fn)
    return geo


def tgvkv_cache_workspace_size(desc: CacheDesc) -> int:
    return _geometry(desc, "tgvkv_cache_workspace_size")[0]


def tgvkv_cache_workspace_init(desc: CacheDesc, ws: torch.Tensor, stream=None):
    p = _ptr(ws, (torch.uint8,), tgvkv_cache_workspace_size(desc), "workspace")
    _check(_lib.load().tgvkv_cache_workspace_init(ctypes.byref(desc), p, _stream(stream)),
           "tgvkv_cache_workspace_init")


def new_cache_workspace(desc: CacheDesc, device=None) -> torch.Tensor:
    """A workspace tensor (uint8) for the paged-cache calls, its status clear."""
    ws = torch.empty(tgvkv_cache_workspace_size(desc), dtype=torch.uint8, device=_named(device))
    with _on(ws):
        tgvkv_cache_workspace_init(desc, ws)
    return ws


def _dev(t, dtype, numel, name):
    """_ptr for one dtype; these calls are short, so the checks are one expression."""
    try:
        if t.is_cuda and t.dtype is dtype and t.is_contiguous() and t.numel() >= numel:
            return t.data_ptr()
    except AttributeError:       # not a tensor
        pass
    if t is None:
        raise TypeError(f"{name} must be a torch.Tensor")
    return _ptr(t, (dtype,), numel, name)


def _table(desc, t, geo):
    """The page table: flat, or with max_pages as its last dimension (another width would
    be read with the wrong row length)."""
    if isinstance(t, torch.Tensor) and t.dim() > 1 and t.shape[-1] != desc.max_pages:
        raise ValueError(f"page_table has shape {tuple(t.shape)}, expected max_pages = {desc.max_pages} columns")
    return _dev(t, torch.int32, geo[2], "page_table")


def _pools(desc, cache: PagedCache, geo):
    dtypes = _POOL[desc.format][0]
    k, v = cache.k, cache.v
    try:
        fine = (k.is_cuda and v.is_cuda and k.dtype in dtypes and v.dtype in dtypes and k.is_contiguous()
                and v.is_contiguous() and k.numel() >= geo[3] and v.numel() >= geo[3])
    except AttributeError:       # not a tensor
        fine = False
    if fine:
        k, v = k.data_ptr(), v.data_ptr()
    else:
        k, v = _ptr(k, dtypes, geo[3], "cache.k"), _ptr(v, dtypes, geo[3], "cache.v")
    if not geo[4]:
        return ctypes.byref(_lib.CachePools(k, v))
    if cache.k_scale is None or cache.v_scale is None:
        raise ValueError("a quantised cache needs k_scale and v_scale")
    return ctypes.byref(_lib.CachePools(k, v, _dev(cache.k_scale, torch.uint8, geo[4], "cache.k_scale"),
                                        _dev(cache.v_scale, torch.uint8, geo[4], "cache.v_scale")))


def _tokens(t, heads, d, name):
    """Pointer, (token, head) strides and tokens of a token-major tensor [T, heads, d]."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dtype not in _BF16_LIKE:
        raise TypeError(f"{name} has dtype {t.dtype}, expected one of {_BF16_LIKE}")
    shape = t.shape
    if len(shape) != 3 or shape[1] != heads or shape[2] != d:
        raise ValueError(f"{name} has shape {tuple(shape)}, expected (tokens, {heads}, {d})")
    n = shape[0]
    if n == 0:
        return t.data_ptr(), heads * d, d, 0
    tok, head, last = t.stride()
    if last != 1:
        raise ValueError(f"{name}'s last dimension must be contiguous")
    # the stride of a dimension with one entry never matters
    return t.data_ptr(), tok if n > 1 else heads * d, head if heads > 1 else d, n


def tgvkv_cache_write(desc, cache: PagedCache, page_table, lens, k_new, v_new, tok_offsets,
                      lens_out, ws, stream=None):
    """Append new tokens, k_new and v_new bf16 [T, H_kv, d] (any token and head
    strides), to the cache, quantised to its format; lens_out receives the new
    lengths (see include/tgvkv.h)."""
    geo = _geometry(desc, "tgvkv_cache_write")
    heads, d, sets = desc.H_kv, desc.d, geo[1]
    kp, kt, kh, n = _tokens(k_new, heads, d, "k_new")
    vp, vt, vh, nv = _tokens(v_new, heads, d, "v_new")
    if n != nv:
        raise ValueError(f"k_new has {n} tokens, v_new {nv}")
    _check(_lib.load().tgvkv_cache_write(
        ctypes.byref(desc), _pools(desc, cache, geo),
        _table(desc, page_table, geo), _dev(lens, torch.int32, sets, "lens"),
        kp, kt, kh, vp, vt, vh, n, _dev(tok_offsets, torch.int32, desc.B + 1, "tok_offsets"),
        _dev(lens_out, torch.int32, sets, "lens_out"), _dev(ws, torch.uint8, geo[0], "workspace"),
        _stream(stream)), "tgvkv_cache_write")


def tgvkv_cache_write_rows(desc, cache: PagedCache, page_table, lens, k_rows, v_rows, offsets,
                           lens_out, ws, stream=None):
    """Append the rows of a CSR cache (tgvkv_evict's k_out, v_out and offsets)."""
    geo = _geometry(desc, "tgvkv_cache_write_rows")
    sets = geo[1]
    kp, vp = _ptr(k_rows, _BF16_LIKE, 0, "k_rows"), _ptr(v_rows, _BF16_LIKE, 0, "v_rows")
    rows = min(k_rows.numel(), v_rows.numel()) // desc.d if kp is not None and vp is not None else 0
    _check(_lib.load().tgvkv_cache_write_rows(
        ctypes.byref(desc), _pools(desc, cache, geo),
        _table(desc, page_table, geo), _dev(lens, torch.int32, sets, "lens"),
        kp, vp, rows, _dev(offsets, torch.int64, sets + 1, "offsets"),
        _dev(lens_out, torch.int32, sets, "lens_out"), _dev(ws, torch.uint8, geo[0], "workspace"),
        _stream(stream)), "tgvkv_cache_write_rows")


def tgvkv_cache_read(desc, cache: PagedCache, page_table, first, offsets, k_out, v_out, ws,
                     stream=None):
    """Read rows offsets[s] .. offsets[s+1] of k_out and v_out (bf16) back from
    the slots first[s] on of every set s (first None: from slot 0)."""
    geo = _geometry(desc, "tgvkv_cache_read")
    sets = geo[1]
    kp, vp = _ptr(k_out, _BF16_LIKE, 0, "k_out"), _ptr(v_out, _BF16_LIKE, 0, "v_out")
    rows = min(k_out.numel(), v_out.numel()) // desc.d if kp is not None and vp is not None else 0
    _check(_lib.load().tgvkv_cache_read(
        ctypes.byref(desc), _pools(desc, cache, geo),
        _table(desc, page_table, geo),
        None if first is None else _dev(first, torch.int32, sets, "first"),
        _dev(offsets, torch.int64, sets + 1, "offsets"), kp, vp, rows,
        _dev(ws, torch.uint8, geo[0], "workspace"), _stream(stream)), "tgvkv_cache_read")


def tgvkv_chunk_attention(desc, cache: PagedCache, page_table, lens, q, tok_offsets, max_q, out, ws,
                          stream=None):
    """Attention of each sequence's new tokens (the last of lens slots) over the
    paged cache: q bf16 [T, H_q, d] (any token and head strides), out bf16
    [T, H_q, d] contiguous (see include/tgvkv.h)."""
    geo = _geometry(desc, "tgvkv_chunk_attention")
    heads, d = desc.H_q, desc.d
    qp, qt, qh, n = _tokens(q, heads, d, "q")
    _check(_lib.load().tgvkv_chunk_attention(
        ctypes.byref(desc), _pools(desc, cache, geo),
        _table(desc, page_table, geo), _dev(lens, torch.int32, geo[1], "lens"),
        qp, qt, qh, n, _dev(tok_offsets, torch.int32, desc.B + 1, "tok_offsets"), max_q,
        _ptr(out, _BF16_LIKE, n * heads * d, "out"), _dev(ws, torch.uint8, geo[0], "workspace"),
        _stream(stream)), "tgvkv_chunk_attention")


# ---- pages of the cache, handed out on the GPU ---------------------------------
#
# These calls and the rotary ones take a few microseconds on the GPU, so what the binding
# does for a call is kept short (structures are passed as they are, ctypes takes their
# addresses; one look at each attribute of a tensor).

_I32, _U8, _BF16 = torch.int32, torch.uint8, torch.bfloat16


@dataclass
class PageList:
    page_table: torch.Tensor   # int32 [B * H_kv, max_pages]; -1: no page
    free: torch.Tensor         # int32 [n_pages]: a stack, of which n_free are left
    n_free: torch.Tensor       # int32 [1]


def alloc_pages(desc: CacheDesc, device=None) -> PageList:
    """A descriptor's page list: an empty table, every page of the pool free."""
    _geometry(desc, "alloc_pages")
    new = dict(dtype=torch.int32, device=_named(device))
    pages = PageList(torch.empty((desc.B * desc.H_kv, desc.max_pages), **new),
                     torch.empty(desc.n_pages, **new), torch.empty(1, **new))
    if pages.free.is_cuda:
        with _on(pages.free):
            tgvkv_pages_init(desc, pages)
    return pages


def _page_list(desc, pages: PageList, geo):
    table = pages.page_table
    try:
        shape = table.shape
        if len(shape) == 2 and shape[0] * shape[1] >= geo[2] and shape[1] == desc.max_pages and \
                table.is_cuda and table.dtype is _I32 and table.is_contiguous():
            tp = table.data_ptr()
        else:
            tp = _table(desc, table, geo)
    except AttributeError:       # not a tensor
        tp = _table(desc, table, geo)
    return _lib.PageListPointers(tp, _dev(pages.free, _I32, desc.n_pages, "pages.free"),
                                 _dev(pages.n_free, _I32, 1, "pages.n_free"))


def tgvkv_pages_init(desc, pages: PageList, stream=None):
    """An empty table and every page free (see include/tgvkv.h)."""
    geo = _geometry(desc, "tgvkv_pages_init")
    rc = _lib.load().tgvkv_pages_init(desc, _page_list(desc, pages, geo), _stream(stream))
    if rc:
        raise TgvkvError(rc, "tgvkv_pages_init")


def _resize(fn, desc, pages, lens, lens_new, ws, stream):
    geo = _geometry(desc, fn)
    sets = geo[1]
    rc = getattr(_lib.load(), fn)(
        desc, _page_list(desc, pages, geo), _dev(lens, _I32, sets, "lens"),
        _dev(lens_new, _I32, sets, "lens_new"), _dev(ws, _U8, geo[0], "workspace"),
        _stream(stream))
    if rc:
        raise TgvkvError(rc, fn)


def tgvkv_pages_grow(desc, pages: PageList, lens, lens_new, ws, stream=None):
    """Pages for sets that go from lens to lens_new slots (those that get longer)."""
    _resize("tgvkv_pages_grow", desc, pages, lens, lens_new, ws, stream)


def tgvkv_pages_shrink(desc, pages: PageList, lens, lens_new, ws, stream=None):
    """Pages back from sets that go from lens to lens_new slots (those that get shorter)."""
    _resize("tgvkv_pages_shrink", desc, pages, lens, lens_new, ws, stream)


def _slot_map(desc, slots):
    """Pointer and tokens of a slot map, int32 [T, H_kv]."""
    try:
        shape = slots.shape
        if (len(shape) == 2 and shape[1] == desc.H_kv and slots.is_cuda and slots.dtype is _I32
                and slots.is_contiguous()):
            return slots.data_ptr(), shape[0]
    except AttributeError:       # not a tensor
        pass
    if not isinstance(slots, torch.Tensor):
        raise TypeError("slots must be a torch.Tensor")
    if len(shape) != 2 or shape[1] != desc.H_kv:
        raise ValueError(f"slots has shape {tuple(shape)}, expected (tokens, {desc.H_kv})")
    return _dev(slots, _I32, 0, "slots"), shape[0]


def tgvkv_pages_append(desc, pages: PageList, lens, tok_offsets, slots, lens_out, ws, n_tokens=None,
                       stream=None):
    """Room for new tokens: pages taken, slots int32 [T, H_kv] (the pool row of every token
    and KV head) and the new lengths written.  slots None: no map, n_tokens says how many
    tokens tok_offsets may count (see include/tgvkv.h)."""
    geo = _geometry(desc, "tgvkv_pages_append")
    sets = geo[1]
    if slots is None:
        if n_tokens is None:
            raise TypeError("n_tokens is needed where slots is None")
        sp, n = None, int(n_tokens)
    else:
        sp, n = _slot_map(desc, slots)
        if n_tokens is not None and n_tokens != n:
            raise ValueError(f"slots has {n} tokens, n_tokens is {n_tokens}")
        sp = sp or None
    rc = _lib.load().tgvkv_pages_append(
        desc, _page_list(desc, pages, geo), _dev(lens, _I32, sets, "lens"),
        _dev(tok_offsets, _I32, desc.B + 1, "tok_offsets"), n, sp,
        _dev(lens_out, _I32, sets, "lens_out"), _dev(ws, _U8, geo[0], "workspace"),
        _stream(stream))
    if rc:
        raise TgvkvError(rc, "tgvkv_pages_append")


def tgvkv_page_slots(desc, page_table, lens, tok_offsets, slots, ws, stream=None):
    """The slots of new tokens whose sets hold their pages already."""
    geo = _geometry(desc, "tgvkv_page_slots")
    sp, n = _slot_map(desc, slots)
    rc = _lib.load().tgvkv_page_slots(
        desc, _table(desc, page_table, geo), _dev(lens, _I32, geo[1], "lens"),
        _dev(tok_offsets, _I32, desc.B + 1, "tok_offsets"), n, sp,
        _dev(ws, _U8, geo[0], "workspace"), _stream(stream))
    if rc:
        raise TgvkvError(rc, "tgvkv_page_slots")


# ---- rotary positions ----------------------------------------------------------

RopePlan = _lib.RopePlan
ROPE_LAYOUT = {"half": _lib.ROPE_HALF, "interleaved": _lib.ROPE_INTERLEAVED}
ROPE_SCALING = {"none": _lib.ROPE_NONE, "linear": _lib.ROPE_LINEAR, "base": _lib.ROPE_BASE,
                "parts": _lib.ROPE_PARTS}
ROPE_MODE = {"forward": _lib.ROPE_FORWARD, "gradient": _lib.ROPE_GRADIENT, "move": _lib.ROPE_MOVE}


def make_rope(d, rot_dim=None, base=10000.0, layout="half", sections=None, scaling="none",
              factor=1.0, original=0, low=1.0, high=32.0, attention=1.0, freqs=None) -> RopePlan:
    """A rotary plan (include/tgvkv.h): host data, made once for a model.

    d: values of a row; rot_dim: how many turn (default: all); layout: "half" or
    "interleaved"; sections: pairs of every position axis (default: one axis); scaling:
    "none", "linear" (factor), "base" (factor) or "parts" (factor, original, low, high);
    attention: the factor of turned values; freqs: rot_dim / 2 frequencies, radians a
    position, in the place of base and scaling."""
    rot_dim = d if rot_dim is None else rot_dim
    sections = [rot_dim // 2] if sections is None else [int(n) for n in sections]
    if not 1 <= len(sections) <= 4:
        raise ValueError(f"{len(sections)} position axes, expected 1 to 4")
    if len(sections) == 1 and sections[0] != rot_dim // 2:
        raise ValueError(f"sections {sections} are not the {rot_dim // 2} pairs")
    if attention == 0:
        raise ValueError("attention is 0")
    values = None
    if freqs is not None:
        values = [float(f) for f in freqs]
        if len(values) != rot_dim // 2:
            raise ValueError(f"{len(values)} frequencies, expected {rot_dim // 2}")
        values = (ctypes.c_double * max(len(values), 1))(*values)
    desc = _lib.RopeDesc(d=d, rot_dim=rot_dim, layout=ROPE_LAYOUT[layout], axes=len(sections),
                         sections=(ctypes.c_int32 * 4)(*sections), scaling=ROPE_SCALING[scaling],
                         original=original, base=base, factor=factor, low=low, high=high,
                         attention=attention, freqs=values)
    plan = RopePlan()
    _check(_lib.load().tgvkv_rope_init(ctypes.byref(plan), ctypes.byref(desc)), "tgvkv_rope_init")
    return plan


def _positions(plan, t, n):
    """Pointer and axis stride of positions, int32 [n] (one axis) or [axes, n]."""
    try:
        shape = t.shape
        if (n and t.is_cuda and t.dtype is _I32 and 1 <= len(shape) <= 2 and shape[-1] == n
                and t.is_contiguous() and t.numel() == n * plan.axes):
            return t.data_ptr(), n
    except AttributeError:       # not a tensor
        pass
    if not isinstance(t, torch.Tensor):
        raise TypeError("positions must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError("positions must be a CUDA tensor")
    if t.dtype is not _I32:
        raise TypeError(f"positions has dtype {t.dtype}, expected torch.int32")
    shape, axes = t.shape, plan.axes
    if not (shape == (axes, n) or (axes == 1 and shape == (n,))):
        raise ValueError(f"positions has shape {tuple(shape)}, expected ({axes}, {n})")
    if axes == 1:
        if n > 1 and t.stride(-1) != 1:
            raise ValueError("positions' last dimension must be contiguous")
        return t.data_ptr(), n
    strides = t.stride()
    if n > 1 and strides[1] != 1:
        raise ValueError("positions' last dimension must be contiguous")
    return t.data_ptr(), strides[0]


def _rows(t, d, name):
    """Pointer, (token, head) strides, and the shape of a tensor [T, heads, d]."""
    try:
        if t.is_cuda and t.dtype is _BF16:
            shape = t.shape
            n, heads, last = shape
            if last == d:
                tok, head, last = t.stride()
                if last == 1 and n > 1 and heads > 1:
                    return t.data_ptr(), tok, head, shape
                if n > 0 and last == 1:    # the stride of a dimension with one entry never matters
                    return t.data_ptr(), tok if n > 1 else heads * d, head if heads > 1 else d, shape
    except (AttributeError, ValueError):   # not a tensor, or not of three dimensions
        pass
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dim() != 3:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected (tokens, heads, {d})")
    p, tok, head, _ = _tokens(t, t.shape[1], d, name)
    return p, tok, head, t.shape


def tgvkv_rope(plan, positions, q, q_out, k=None, k_out=None, mode="forward", stream=None):
    """q_out (and k_out) receive the rows of q (and k), bf16 [T, heads, d] with any token
    and head strides, turned by their tokens' positions, int32 [T] or [axes, T]; an output
    may be its input.  mode: "forward", "gradient" (q, k: the gradients of turned rows) or
    "move" (positions: differences) (see include/tgvkv.h)."""
    d = plan.d
    qp, qt, qh, q_shape = _rows(q, d, "q")
    op, ot, oh, shape = _rows(q_out, d, "q_out")
    if shape != q_shape:
        raise ValueError(f"q_out has shape {tuple(shape)}, q {tuple(q_shape)}")
    n, H_q, _ = q_shape
    kp, kt, kh, H_k, lp, lt, lh = None, 0, 0, 0, None, 0, 0
    if k is not None and k_out is not None:
        kp, kt, kh, k_shape = _rows(k, d, "k")
        lp, lt, lh, shape = _rows(k_out, d, "k_out")
        if shape != k_shape or k_shape[0] != n:
            raise ValueError(f"k has shape {tuple(k_shape)}, k_out {tuple(shape)}, q {tuple(q_shape)}")
        H_k = k_shape[1]
    elif k is not None or k_out is not None:
        raise TypeError("k and k_out go together")
    pp, ps = _positions(plan, positions, n)
    rc = _lib.load().tgvkv_rope(plan, ROPE_MODE[mode], pp, ps, n, qp, qt, qh, H_q, op, ot, oh,
                                kp, kt, kh, H_k, lp, lt, lh, _stream(stream))
    if rc:
        raise TgvkvError(rc, "tgvkv_rope")


def tgvkv_rope_write(desc, cache: PagedCache, plan, positions, slots, q, k_new, v_new, q_out, ws,
                     stream=None):
    """A serving step's tokens in one pass: q bf16 [T, H_q, d] turned into q_out, k_new turned
    and v_new stored in the cache's format at the pool rows of slots, int32 [T, H_kv] (any
    token and head strides; q and q_out None: keys and values only) (see include/tgvkv.h)."""
    geo = _geometry(desc, "tgvkv_rope_write")
    d, heads = desc.d, desc.H_kv
    kp, kt, kh, shape = _rows(k_new, d, "k_new")
    vp, vt, vh, v_shape = _rows(v_new, d, "v_new")
    n = shape[0]
    if shape[1] != heads or v_shape != shape:
        raise ValueError(f"k_new has shape {tuple(shape)}, v_new {tuple(v_shape)}, "
                         f"expected (tokens, {heads}, {d})")
    sp, ns = _slot_map(desc, slots)
    qp, qt, qh, op, ot, oh = None, 0, 0, None, 0, 0
    if q is not None and q_out is not None:
        qp, qt, qh, shape = _rows(q, d, "q")
        op, ot, oh, o_shape = _rows(q_out, d, "q_out")
        if shape[1] != desc.H_q or o_shape != shape:
            raise ValueError(f"q has shape {tuple(shape)}, q_out {tuple(o_shape)}, "
                             f"expected (tokens, {desc.H_q}, {d})")
    elif q is not None or q_out is not None:
        raise TypeError("q and q_out go together")
    if ns != n or shape[0] != n:
        raise ValueError(f"tokens: k_new {n}, slots {ns}, q {shape[0]}")
    pp, ps = _positions(plan, positions, n)
    rc = _lib.load().tgvkv_rope_write(
        desc, _pools(desc, cache, geo), plan, pp, ps, sp, n, qp, qt, qh, kp, kt, kh, vp, vt, vh,
        op, ot, oh, _dev(ws, _U8, geo[0], "workspace"), _stream(stream))
    if rc:
        raise TgvkvError(rc, "tgvkv_rope_write")


def default_scale(d: int) -> float:
    return 1.0 / math.sqrt(d)
