"""ctypes binding of libaudiokv.so. Same names as the C entry points (without
the audiokv_ prefix); every function only marshals arguments. Tensors must be
contiguous CUDA(HIP) tensors of the documented dtype; outputs are allocated
here with torch and returned."""
from __future__ import annotations

import ctypes as C
import dataclasses
import os
from dataclasses import dataclass
from typing import Optional, Sequence, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libaudiokv.so")

POOL_AVG, POOL_MAX = 0, 1
LAYOUT_HEAD_MAJOR, LAYOUT_TOKEN_MAJOR = 0, 1
SCOPE_ITEM, SCOPE_GLOBAL = 0, 1
CUTOFF_FRACTION, CUTOFF_ENERGY, CUTOFF_ENERGY_NO_DC = 0, 1, 2


class AudioKVError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"audiokv error {code}: {msg}")
        self.code = code


class _CParams(C.Structure):
    _fields_ = [
        ("size", C.c_uint32),
        ("n_q_heads", C.c_int32),
        ("n_kv_heads", C.c_int32),
        ("head_dim", C.c_int32),
        ("window", C.c_int32),
        ("pool_kernel", C.c_int32),
        ("pool_mode", C.c_int32),
        ("causal", C.c_int32),
        ("kv_layout", C.c_int32),
        ("softmax_scale", C.c_float),
        ("floor_frac", C.c_float),
        ("cutoff_mode", C.c_int32),
        ("taper_bins", C.c_int32),
        ("kv_stride_item", C.c_int64),
        ("kv_stride_head", C.c_int64),
        ("kv_stride_tok", C.c_int64),
    ]


class _CSlots(C.Structure):
    _fields_ = [
        ("size", C.c_uint32),
        ("capacity", C.c_int32),
        ("k", C.c_void_p),
        ("v", C.c_void_p),
        ("lengths", C.c_void_p),
        ("weights", C.c_void_p),
        ("positions", C.c_void_p),
    ]


@dataclass
class Params:
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    window: int
    pool_kernel: int = 7
    pool_mode: int = POOL_AVG
    causal: int = 1
    kv_layout: int = LAYOUT_HEAD_MAJOR
    softmax_scale: float = 0.0
    floor_frac: float = 0.1
    cutoff_mode: int = CUTOFF_FRACTION
    taper_bins: int = 0
    kv_stride_item: int = 0       # explicit K/V strides in elements; all 0: the packed layout of kv_layout
    kv_stride_head: int = 0
    kv_stride_tok: int = 0

    def key(self) -> tuple:
        return (self.n_q_heads, self.n_kv_heads, self.head_dim, self.window, self.pool_kernel, self.pool_mode,
                self.causal, self.kv_layout, self.softmax_scale, self.floor_frac, self.cutoff_mode, self.taper_bins,
                self.kv_stride_item, self.kv_stride_head, self.kv_stride_tok)

    def c(self) -> _CParams:
        return _CParams(C.sizeof(_CParams), self.n_q_heads, self.n_kv_heads, self.head_dim, self.window,
                        self.pool_kernel, self.pool_mode, self.causal, self.kv_layout,
                        self.softmax_scale, self.floor_frac, self.cutoff_mode, self.taper_bins,
                        self.kv_stride_item, self.kv_stride_head, self.kv_stride_tok)


_SLOTS_SIZE = C.sizeof(_CSlots)
_BF16, _F32, _I32 = torch.bfloat16, torch.float32, torch.int32


@dataclass
class Slots:
    """Rows that sequences own: device tensors, see audiokv_slots. `weights` and `positions` may be missing."""
    k: torch.Tensor                          # bf16, in the layout of Params with the sequence as the item
    v: torch.Tensor
    lengths: torch.Tensor                    # int32 [n_seqs * n_kv_heads]
    capacity: int
    weights: Optional[torch.Tensor] = None   # fp32 [n_seqs * n_kv_heads, capacity]
    positions: Optional[torch.Tensor] = None # int32, the same

    def _c(self, p: Params, n_seqs: int, at: int) -> _CSlots:
        """The C struct, after a look at types, sizes and the device (in one expression: a step is some twenty microseconds of the host's)."""
        k, v, lengths, w, pos = self.k, self.v, self.lengths, self.weights, self.positions
        heads = n_seqs * p.n_kv_heads
        slots = heads * self.capacity
        if (k.dtype is not _BF16 or v.dtype is not _BF16 or k.get_device() != at or v.get_device() != at
                or p.kv_stride_tok == 0 and (not k.is_contiguous() or not v.is_contiguous() or k.numel() < slots * p.head_dim
                                             or v.numel() < slots * p.head_dim)):
            raise ValueError(f"slots.k and slots.v must be tensors of the current device, {at}, and dtype {_BF16}, and contiguous with "
                             f"{slots * p.head_dim} values where params has no strides")
        if p.kv_stride_tok != 0 and n_seqs > 0:
            end = ((n_seqs - 1) * p.kv_stride_item + (p.n_kv_heads - 1) * p.kv_stride_head + (self.capacity - 1) * p.kv_stride_tok + p.head_dim)
            if _room(p, k) < end or _room(p, v) < end:
                raise ValueError(f"slots.k or slots.v has room for {min(_room(p, k), _room(p, v))} values, {end} needed by the strides")
        if lengths.dtype is not _I32 or lengths.get_device() != at or not lengths.is_contiguous() or lengths.numel() < heads:
            raise ValueError(f"slots.lengths must be a contiguous tensor of {heads} values of dtype {_I32} on the current device, {at}")
        if w is not None and (w.dtype is not _F32 or w.get_device() != at or not w.is_contiguous() or w.numel() < slots):
            raise ValueError(f"slots.weights must be a contiguous tensor of {slots} values of dtype {_F32} on the current device, {at}")
        if pos is not None and (pos.dtype is not _I32 or pos.get_device() != at or not pos.is_contiguous() or pos.numel() < slots):
            raise ValueError(f"slots.positions must be a contiguous tensor of {slots} values of dtype {_I32} on the current device, {at}")
        return _CSlots(_SLOTS_SIZE, self.capacity, k.data_ptr(), v.data_ptr(), lengths.data_ptr(), _ptr(w), _ptr(pos))


def lib_path() -> str:
    return _LIB_PATH


def _load() -> C.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: run `python -m paper_2604_06694_amd.build` "
                          "(there is no fallback path)")
    lib = C.CDLL(_LIB_PATH)
    vp, i32, i64, f64 = C.c_void_p, C.c_int32, C.c_int64, C.c_double
    pp = C.POINTER(_CParams)
    lib.audiokv_version.restype = i32
    lib.audiokv_last_error.restype = C.c_char_p
    lib.audiokv_n_keep.restype = i32
    lib.audiokv_n_keep.argtypes = [f64, i32]
    lib.audiokv_total_kept.argtypes = [pp, i32, vp, f64, C.POINTER(i64)]
    lib.audiokv_workspace_bytes.argtypes = [pp, i32, vp, C.POINTER(C.c_size_t)]
    lib.audiokv_score.argtypes = [pp, vp, vp, vp, vp, i32, vp, vp, C.c_size_t, vp]
    lib.audiokv_score_lse.argtypes = [pp, vp, vp, vp, vp, vp, i32, vp, vp, C.c_size_t, vp]
    lib.audiokv_allocate.argtypes = [pp, vp, i32, i32, i32, vp, vp, f64, vp, vp, vp]
    lib.audiokv_smooth.argtypes = [pp, vp, vp, vp, i32, f64, f64, vp, vp, C.c_size_t, vp]
    lib.audiokv_smooth_cutoffs.argtypes = [pp, vp, vp, vp, i32, f64, vp, vp, C.c_size_t, vp]
    lib.audiokv_select.argtypes = [pp, vp, vp, vp, vp, vp, i32, vp, vp, C.c_size_t, vp]
    lib.audiokv_compact.argtypes = [pp, vp, vp, vp, vp, vp, vp, i32, i64, vp, vp, vp]
    lib.audiokv_evict.argtypes = [pp, vp, vp, vp, vp, i32, vp, vp, i32, f64, f64, f64,
                                  vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    lib.audiokv_evict_lse.argtypes = [pp, vp, vp, vp, vp, vp, i32, vp, vp, i32, f64, f64, f64,
                                  vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    lib.audiokv_evict_noalloc.argtypes = [pp, vp, vp, vp, vp, i32, vp, vp, i32, f64, f64, f64,
                                          vp, vp, vp, vp, vp, vp]
    lib.audiokv_decode_workspace_bytes.argtypes = [pp, i32, i64, C.POINTER(C.c_size_t)]
    lib.audiokv_decode_attend.argtypes = [pp, vp, vp, vp, vp, i32, i64, vp, vp, C.c_size_t, vp]
    lib.audiokv_accumulate_workspace_bytes.argtypes = [pp, i32, vp, vp, C.POINTER(C.c_size_t)]
    lib.audiokv_accumulate.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, i32, vp, i64, vp, C.c_size_t, vp]
    lib.audiokv_decode_shared_workspace_bytes.argtypes = [pp, i32, i64, i32, i32, i32, C.POINTER(C.c_size_t)]
    lib.audiokv_decode_shared.argtypes = [pp, vp, vp, vp, vp, i32, i64, vp, i32, i32, C.POINTER(_CSlots), i32, vp, vp, vp, vp, vp,
                                          C.c_size_t, vp]
    lib.audiokv_evict_accumulated_workspace_bytes.argtypes = [pp, i32, i32, i32, C.POINTER(C.c_size_t)]
    lib.audiokv_evict_accumulated.argtypes = [pp, C.POINTER(_CSlots), i32, i32, vp, i32, i32, vp, C.c_size_t, vp]
    lib.audiokv_profile_enable.argtypes = [i32]
    lib.audiokv_profile_enable.restype = i32
    lib.audiokv_profile_read.argtypes = [C.POINTER(C.c_float)]
    lib.audiokv_profile_read.restype = i32
    for name in ("total_kept", "workspace_bytes", "score", "allocate", "smooth", "smooth_cutoffs", "select", "compact", "evict",
                 "decode_workspace_bytes", "decode_attend", "score_lse", "evict_lse", "evict_noalloc",
                 "accumulate_workspace_bytes", "accumulate", "decode_shared_workspace_bytes", "decode_shared",
                 "evict_accumulated_workspace_bytes", "evict_accumulated"):
        getattr(lib, "audiokv_" + name).restype = i32
    return lib


_lib = _load()


def _check(rc: int) -> None:
    if rc != 0:
        raise AudioKVError(rc, _lib.audiokv_last_error().decode())


# The current device and its current stream's handle without the objects and checks around them. These are no public names of
# torch's, so they may be missing.
_raw_device = getattr(torch._C, "_cuda_getDevice", None)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    """The current stream's handle. (torch.cuda.current_stream() builds an object around it: 2.8 us of a call, this 0.2.)"""
    if _raw_stream is None or _raw_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_raw_device())


_LENS_CACHE: dict = {}


def _host_lens(seqlens: Sequence[int]):
    """ctypes int32 array of the lengths; the arrays of recent length lists are kept (a serving loop passes the
    same few lists over and over, and building the array costs more than the rest of the marshalling)."""
    key = tuple(seqlens)
    arr = _LENS_CACHE.get(key)
    if arr is None:
        if len(_LENS_CACHE) > 256:
            _LENS_CACHE.clear()
        arr = _LENS_CACHE[key] = (C.c_int32 * len(key))(*[int(x) for x in key])
    return arr


def _cu(seqlens: Sequence[int], device) -> torch.Tensor:
    cu = [0]
    for L in seqlens:
        cu.append(cu[-1] + int(L))
    return torch.tensor(cu, dtype=torch.int32, device=device)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _need(t: torch.Tensor, dtype, name: str) -> torch.Tensor:
    if t.dtype is not dtype or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device tensor of dtype {dtype}")
    return t


# Kernels go to the current stream of the current device: tensors of another one, or of the host, are refused.
def _device() -> int:
    return _raw_device() if _raw_device is not None else torch.cuda.current_device()


def _need_at(t: torch.Tensor, dtype, at: int, name: str) -> torch.Tensor:
    if t.dtype is not dtype or t.get_device() != at or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor of dtype {dtype} on the current device, {at}")
    return t


def _workspace_at(t: torch.Tensor, at: int) -> torch.Tensor:
    if t.get_device() != at or not t.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on the current device, {at}")
    return t


def _table(t: Optional[torch.Tensor], n: int, at: int, name: str) -> None:
    """Exclusive prefix sums of n numbers, if given."""
    if t is not None and _need_at(t, _I32, at, name).numel() < n + 1:
        raise ValueError(f"{name} has {t.numel()} values, {n + 1} needed")


def _rows_end(p: Params, lens: Sequence[int]) -> int:
    """Elements from the first of K (or V) to the end of the last row that items of these lengths have."""
    if p.kv_stride_tok == 0:
        return sum(int(x) for x in lens) * p.n_kv_heads * p.head_dim
    last_head = (p.n_kv_heads - 1) * p.kv_stride_head + p.head_dim
    return max((i * p.kv_stride_item + (int(x) - 1) * p.kv_stride_tok + last_head for i, x in enumerate(lens)), default=0)


def _room(p: Params, t: torch.Tensor) -> int:
    """Elements of memory from t's first: a tensor that strides address may be a view of a part of it."""
    if p.kv_stride_tok == 0:
        return t.numel()
    return t.untyped_storage().nbytes() // t.element_size() - t.storage_offset()


def version() -> int:
    return _lib.audiokv_version()


def n_keep(ratio: float, L: int) -> int:
    return _lib.audiokv_n_keep(float(ratio), int(L))


_SIZE_CACHE: dict = {}


def _cached(key, compute):
    v = _SIZE_CACHE.get(key)
    if v is None:
        if len(_SIZE_CACHE) > 1024:
            _SIZE_CACHE.clear()
        v = _SIZE_CACHE[key] = compute()
    return v


def total_kept(p: Params, seqlens: Sequence[int], ratio: float) -> int:
    def compute():
        out = C.c_int64(0)
        cp = p.c()
        _check(_lib.audiokv_total_kept(C.byref(cp), len(seqlens), _host_lens(seqlens), float(ratio), C.byref(out)))
        return out.value
    return _cached(("rows", p.key(), tuple(seqlens), float(ratio)), compute)


def workspace_bytes(p: Params, seqlens: Sequence[int]) -> int:
    def compute():
        out = C.c_size_t(0)
        cp = p.c()
        _check(_lib.audiokv_workspace_bytes(C.byref(cp), len(seqlens), _host_lens(seqlens), C.byref(out)))
        return out.value
    return _cached(("ws", p.key(), tuple(seqlens)), compute)


def _workspace(p: Params, seqlens: Sequence[int], device, workspace: Optional[torch.Tensor]) -> torch.Tensor:
    if workspace is not None:         # (its size is checked by the call that it is handed to)
        return workspace
    return torch.empty(max(workspace_bytes(p, seqlens), 256), dtype=torch.uint8, device=device)


def score(p: Params, q_win: torch.Tensor, k: torch.Tensor, seqlens: Sequence[int], *,
          cu_seqlens: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
          workspace: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None) -> torch.Tensor:
    """`lse` (fp32 [n_items, n_q_heads, window], natural-log softmax denominators of the window rows) selects
    audiokv_score_lse."""
    _need(q_win, torch.bfloat16, "q_win"); _need(k, torch.bfloat16, "k")
    dev = k.device
    cu = cu_seqlens if cu_seqlens is not None else _cu(seqlens, dev)
    total = sum(int(x) for x in seqlens) * p.n_kv_heads
    if out is None:
        out = torch.empty(total, dtype=torch.float32, device=dev)
    ws = _workspace(p, seqlens, dev, workspace)
    cp = p.c()
    if lse is not None:
        _need(lse, torch.float32, "lse")
        _check(_lib.audiokv_score_lse(C.byref(cp), _ptr(q_win), _ptr(k), _ptr(lse), _ptr(cu), _host_lens(seqlens),
                                      len(seqlens), _ptr(out), _ptr(ws), ws.numel(), _stream()))
        return out
    _check(_lib.audiokv_score(C.byref(cp), _ptr(q_win), _ptr(k), _ptr(cu), _host_lens(seqlens), len(seqlens),
                              _ptr(out), _ptr(ws), ws.numel(), _stream()))
    return out


def allocate(p: Params, weights: torch.Tensor, n_segments: int, heads_per_segment: int, seqlens: Sequence[int],
             ratio: float, *, weight_group: int = 1, cu_seqlens: Optional[torch.Tensor] = None
             ) -> Tuple[torch.Tensor, torch.Tensor]:
    _need(weights, torch.float32, "weights")
    dev = weights.device
    cu = cu_seqlens if cu_seqlens is not None else _cu(seqlens, dev)
    n = n_segments * heads_per_segment
    budgets = torch.empty(n, dtype=torch.int32, device=dev)
    cu_b = torch.empty(n + 1, dtype=torch.int32, device=dev)
    cp = p.c()
    _check(_lib.audiokv_allocate(C.byref(cp), _ptr(weights), n_segments, heads_per_segment, weight_group, _ptr(cu),
                                 _host_lens(seqlens), float(ratio), _ptr(budgets), _ptr(cu_b), _stream()))
    return budgets, cu_b


def smooth(p: Params, scores: torch.Tensor, seqlens: Sequence[int], cutoff_frac: float, alpha: float, *,
           cu_seqlens: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
           workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    _need(scores, torch.float32, "scores")
    dev = scores.device
    cu = cu_seqlens if cu_seqlens is not None else _cu(seqlens, dev)
    if out is None:
        out = torch.empty_like(scores)
    ws = workspace if workspace is not None else _workspace(dataclasses.replace(p, window=0), seqlens, dev, None)
    cp = p.c()
    _check(_lib.audiokv_smooth(C.byref(cp), _ptr(scores), _ptr(cu), _host_lens(seqlens), len(seqlens),
                               float(cutoff_frac), float(alpha), _ptr(out), _ptr(ws), ws.numel(), _stream()))
    return out


def smooth_cutoffs(p: Params, scores: torch.Tensor, seqlens: Sequence[int], cutoff_frac: float, *,
                   cu_seqlens: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The cutoff bin k* of every head (int32 [n_items * n_kv_heads])."""
    _need(scores, torch.float32, "scores")
    dev = scores.device
    cu = cu_seqlens if cu_seqlens is not None else _cu(seqlens, dev)
    out = torch.empty(len(seqlens) * p.n_kv_heads, dtype=torch.int32, device=dev)
    ws = workspace if workspace is not None else _workspace(dataclasses.replace(p, window=0), seqlens, dev, None)
    cp = p.c()
    _check(_lib.audiokv_smooth_cutoffs(C.byref(cp), _ptr(scores), _ptr(cu), _host_lens(seqlens), len(seqlens),
                                       float(cutoff_frac), _ptr(out), _ptr(ws), ws.numel(), _stream()))
    return out


def select(p: Params, scores: torch.Tensor, budgets: torch.Tensor, cu_budgets: torch.Tensor,
           seqlens: Sequence[int], total_rows: int, *, cu_seqlens: Optional[torch.Tensor] = None) -> torch.Tensor:
    _need(scores, torch.float32, "scores"); _need(budgets, torch.int32, "budgets"); _need(cu_budgets, torch.int32, "cu_budgets")
    dev = scores.device
    cu = cu_seqlens if cu_seqlens is not None else _cu(seqlens, dev)
    idx = torch.empty(max(int(total_rows), 1), dtype=torch.int32, device=dev)
    cp = p.c()
    _check(_lib.audiokv_select(C.byref(cp), _ptr(scores), _ptr(budgets), _ptr(cu_budgets), _ptr(cu),
                               _host_lens(seqlens), len(seqlens), _ptr(idx), None, 0, _stream()))
    return idx if idx.shape[0] == int(total_rows) else idx[:int(total_rows)]


def compact(p: Params, k: torch.Tensor, v: torch.Tensor, indices: torch.Tensor, cu_budgets: torch.Tensor,
            seqlens: Sequence[int], total_rows: int, *, cu_seqlens: Optional[torch.Tensor] = None
            ) -> Tuple[torch.Tensor, torch.Tensor]:
    _need(k, torch.bfloat16, "k"); _need(v, torch.bfloat16, "v"); _need(indices, torch.int32, "indices")
    dev = k.device
    cu = cu_seqlens if cu_seqlens is not None else _cu(seqlens, dev)
    k_out = torch.empty((max(int(total_rows), 1), p.head_dim), dtype=torch.bfloat16, device=dev)
    v_out = torch.empty_like(k_out)
    cp = p.c()
    _check(_lib.audiokv_compact(C.byref(cp), _ptr(k), _ptr(v), _ptr(indices), _ptr(cu_budgets), _ptr(cu),
                                _host_lens(seqlens), len(seqlens), int(total_rows), _ptr(k_out), _ptr(v_out),
                                _stream()))
    if k_out.shape[0] == int(total_rows):
        return k_out, v_out
    return k_out[:int(total_rows)], v_out[:int(total_rows)]


def evict(p: Params, q_win: torch.Tensor, k: torch.Tensor, v: torch.Tensor, weights: torch.Tensor,
          seqlens: Sequence[int], ratio: float, cutoff_frac: float, alpha: float, *,
          alloc_scope: int = SCOPE_GLOBAL, cu_seqlens: Optional[torch.Tensor] = None,
          workspace: Optional[torch.Tensor] = None, outputs: Optional[dict] = None,
          lse: Optional[torch.Tensor] = None) -> dict:
    """Runs the fused path (audiokv_evict_lse when `lse` is given). `outputs` may carry preallocated k_out, v_out, indices, budgets, cu_budgets
    (used by the benchmark so that the timed region allocates nothing)."""
    _need(q_win, torch.bfloat16, "q_win"); _need(k, torch.bfloat16, "k"); _need(v, torch.bfloat16, "v")
    _need(weights, torch.float32, "weights")
    dev = k.device
    cu = cu_seqlens if cu_seqlens is not None else _cu(seqlens, dev)
    n_heads = len(seqlens) * p.n_kv_heads
    rows = total_kept(p, seqlens, ratio)
    o = outputs if outputs is not None else {}
    if "k_out" not in o:
        o["k_out"] = torch.empty((max(rows, 1), p.head_dim), dtype=torch.bfloat16, device=dev)
        o["v_out"] = torch.empty_like(o["k_out"])
        o["indices"] = torch.empty(max(rows, 1), dtype=torch.int32, device=dev)
        o["budgets"] = torch.empty(n_heads, dtype=torch.int32, device=dev)
        o["cu_budgets"] = torch.empty(n_heads + 1, dtype=torch.int32, device=dev)
    ws = _workspace(p, seqlens, dev, workspace)
    cp = p.c()
    if lse is not None:
        _need(lse, torch.float32, "lse")
        _check(_lib.audiokv_evict_lse(C.byref(cp), _ptr(q_win), _ptr(k), _ptr(v), _ptr(lse), _ptr(weights),
                                      int(alloc_scope), _ptr(cu), _host_lens(seqlens), len(seqlens), float(ratio),
                                      float(cutoff_frac), float(alpha), _ptr(o["k_out"]), _ptr(o["v_out"]),
                                      _ptr(o["indices"]), _ptr(o["budgets"]), _ptr(o["cu_budgets"]), _ptr(ws),
                                      ws.numel(), _stream()))
        o["total_rows"] = rows
        o["workspace"] = ws
        return o
    _check(_lib.audiokv_evict(C.byref(cp), _ptr(q_win), _ptr(k), _ptr(v), _ptr(weights), int(alloc_scope), _ptr(cu),
                              _host_lens(seqlens), len(seqlens), float(ratio), float(cutoff_frac), float(alpha),
                              _ptr(o["k_out"]), _ptr(o["v_out"]), _ptr(o["indices"]), _ptr(o["budgets"]),
                              _ptr(o["cu_budgets"]), _ptr(ws), ws.numel(), _stream()))
    o["total_rows"] = rows
    o["workspace"] = ws
    return o


NOALLOC_SCRATCH_BYTES = 8 << 20


def evict_noalloc(p: Params, q_win: torch.Tensor, k: torch.Tensor, v: torch.Tensor, weights: torch.Tensor,
                  seqlens: Sequence[int], ratio: float, cutoff_frac: float, alpha: float, outputs: dict, *,
                  alloc_scope: int = SCOPE_GLOBAL, cu_seqlens: torch.Tensor) -> dict:
    """audiokv_evict_noalloc: the caller brings every buffer (`outputs` with k_out, v_out, indices, budgets,
    cu_budgets; `cu_seqlens` on the device); neither this function nor the library allocates device memory."""
    cp = p.c()
    o = outputs
    _check(_lib.audiokv_evict_noalloc(C.byref(cp), _ptr(q_win), _ptr(k), _ptr(v), _ptr(weights), int(alloc_scope),
                                      _ptr(cu_seqlens), _host_lens(seqlens), len(seqlens), float(ratio),
                                      float(cutoff_frac), float(alpha), _ptr(o["k_out"]), _ptr(o["v_out"]),
                                      _ptr(o["indices"]), _ptr(o["budgets"]), _ptr(o["cu_budgets"]), _stream()))
    return o


def decode_workspace_bytes(p: Params, n_items: int, total_rows: int) -> int:
    out = C.c_size_t(0)
    cp = p.c()
    _check(_lib.audiokv_decode_workspace_bytes(C.byref(cp), int(n_items), int(total_rows), C.byref(out)))
    return out.value


def decode_attend(p: Params, q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                  cu_budgets: torch.Tensor, n_items: int, total_rows: int, *,
                  out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One decoding step on the compacted cache: fp32 [n_items, n_q_heads, head_dim]."""
    _need(q, torch.bfloat16, "q"); _need(k_cache, torch.bfloat16, "k_cache"); _need(v_cache, torch.bfloat16, "v_cache")
    _need(cu_budgets, torch.int32, "cu_budgets")
    dev = q.device
    if out is None:
        out = torch.empty((n_items, p.n_q_heads, p.head_dim), dtype=torch.float32, device=dev)
    ws = workspace
    if ws is None:
        ws = torch.empty(max(decode_workspace_bytes(p, n_items, total_rows), 256), dtype=torch.uint8, device=dev)
    cp = p.c()
    _check(_lib.audiokv_decode_attend(C.byref(cp), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(cu_budgets),
                                      int(n_items), int(total_rows), _ptr(out), _ptr(ws), ws.numel(), _stream()))
    return out


def accumulate_workspace_bytes(p: Params, seqlens: Sequence[int], queries: Sequence[int]) -> int:
    if len(queries) != len(seqlens):
        raise ValueError(f"{len(queries)} numbers of queries for {len(seqlens)} lengths")

    def compute():
        out = C.c_size_t(0)
        cp = p.c()
        _check(_lib.audiokv_accumulate_workspace_bytes(C.byref(cp), len(seqlens), _host_lens(seqlens), _host_lens(queries),
                                                       C.byref(out)))
        return out.value
    return _cached(("accumulate", p.key(), tuple(seqlens), tuple(queries)), compute)


def accumulate(p: Params, q: torch.Tensor, k: torch.Tensor, seqlens: Sequence[int], queries: Sequence[int], *,
               weights: Optional[torch.Tensor] = None, pitch: int = 0, lse: Optional[torch.Tensor] = None,
               cu_seqlens: Optional[torch.Tensor] = None, cu_queries: Optional[torch.Tensor] = None,
               workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Adds the attention weight that every token receives from the last queries[i] positions of each item to `weights`
    (fp32; zeros of the scores' layout if not given) and returns it. `pitch`: distance between heads of `weights`, 0:
    packed like scores. `lse`: fp32, [n_q_heads][queries[i]] of item after item."""
    at = _device()
    _need_at(q, _BF16, at, "q"); _need_at(k, _BF16, at, "k")
    if len(queries) != len(seqlens):
        raise ValueError(f"{len(queries)} numbers of queries for {len(seqlens)} lengths")
    dev = k.device
    if q.numel() < sum(queries) * p.n_q_heads * p.head_dim:
        raise ValueError("q is smaller than its queries")
    if _room(p, k) < _rows_end(p, seqlens):
        raise ValueError(f"k has room for {_room(p, k)} values, {_rows_end(p, seqlens)} needed")
    _table(cu_seqlens, len(seqlens), at, "cu_seqlens"); _table(cu_queries, len(seqlens), at, "cu_queries")
    cu = cu_seqlens if cu_seqlens is not None else _cu(seqlens, dev)
    cu_q = cu_queries if cu_queries is not None else _cu(queries, dev)
    total = (pitch * len(seqlens) if pitch else sum(int(x) for x in seqlens)) * p.n_kv_heads
    if weights is None:
        weights = torch.zeros(total, dtype=torch.float32, device=dev)
    _need_at(weights, _F32, at, "weights")
    if weights.numel() < total:
        raise ValueError(f"weights has {weights.numel()} values, {total} needed")
    if lse is not None:
        _need_at(lse, _F32, at, "lse")
        if lse.numel() < sum(queries) * p.n_q_heads:
            raise ValueError("lse is smaller than its queries")
    if workspace is not None:
        ws = _workspace_at(workspace, at)
    else:
        ws = torch.empty(max(accumulate_workspace_bytes(p, seqlens, queries), 256), dtype=torch.uint8, device=dev)
    cp = p.c()
    _check(_lib.audiokv_accumulate(C.byref(cp), _ptr(q), _ptr(k), _ptr(lse), _ptr(cu), _host_lens(seqlens), _ptr(cu_q),
                                   _host_lens(queries), len(seqlens), _ptr(weights), int(pitch), _ptr(ws), ws.numel(), _stream()))
    return weights


def decode_shared_workspace_bytes(p: Params, n_items: int, total_rows: int, n_seqs: int, max_seqs: int, max_own: int) -> int:
    out = C.c_size_t(0)
    cp = p.c()
    _check(_lib.audiokv_decode_shared_workspace_bytes(C.byref(cp), int(n_items), int(total_rows), int(n_seqs), int(max_seqs),
                                                      int(max_own), C.byref(out)))
    return out.value


def decode_shared(p: Params, q: torch.Tensor, k_prompt: Optional[torch.Tensor], v_prompt: Optional[torch.Tensor],
                  cu_budgets: Optional[torch.Tensor], total_rows: int, cu_seqs: Optional[torch.Tensor], max_seqs: int, *,
                  slots: Optional[Slots] = None, max_own: int = 0, k_new: Optional[torch.Tensor] = None,
                  v_new: Optional[torch.Tensor] = None, pos_new: Optional[torch.Tensor] = None,
                  out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One decoding step of q.shape[0] sequences (q: bf16 [n_seqs, n_q_heads, head_dim]) on the compacted caches that they
    share (`k_prompt` None: on none) and the rows that they own; bf16 output of q's shape. Updates `slots` in place."""
    at = _device()
    _need_at(q, _BF16, at, "q")
    dev, n_seqs = q.device, q.shape[0]
    if q.numel() != n_seqs * p.n_q_heads * p.head_dim:
        raise ValueError("q must be [n_seqs, n_q_heads, head_dim]")
    n_items = 0
    if k_prompt is not None:
        _need_at(k_prompt, _BF16, at, "k_prompt"); _need_at(v_prompt, _BF16, at, "v_prompt")
        _need_at(cu_budgets, _I32, at, "cu_budgets"); _need_at(cu_seqs, _I32, at, "cu_seqs")
        n_items = cu_seqs.numel() - 1
        if n_items < 1:                       # (the library's call without items lets every sequence take part)
            raise ValueError("cu_seqs must have an entry per item and one more; without prompts, k_prompt is None")
        if cu_budgets.numel() < n_items * p.n_kv_heads + 1:
            raise ValueError(f"cu_budgets has {cu_budgets.numel()} values, {n_items * p.n_kv_heads + 1} needed")
        if min(k_prompt.numel(), v_prompt.numel()) < total_rows * p.head_dim:
            raise ValueError(f"k_prompt or v_prompt holds fewer than {total_rows} rows")
    if k_new is not None:
        rows = n_seqs * p.n_kv_heads * p.head_dim
        if _need_at(k_new, _BF16, at, "k_new").numel() < rows or v_new is None or _need_at(v_new, _BF16, at, "v_new").numel() < rows:
            raise ValueError("k_new and v_new must be [n_seqs, n_kv_heads, head_dim]")
    elif v_new is not None:
        raise ValueError("k_new and v_new come together")
    if pos_new is not None and _need_at(pos_new, _I32, at, "pos_new").numel() < n_seqs:
        raise ValueError("pos_new must have a value per sequence")
    if out is None:
        out = torch.empty(q.shape, dtype=torch.bfloat16, device=dev)
    elif _need_at(out, _BF16, at, "out").numel() < q.numel():
        raise ValueError("out is smaller than q")
    if workspace is not None:
        ws = _workspace_at(workspace, at)
    else:
        ws = torch.empty(max(decode_shared_workspace_bytes(p, n_items, total_rows, n_seqs, max_seqs, max_own if slots else 0), 256),
                         dtype=torch.uint8, device=dev)
    cs = C.byref(slots._c(p, n_seqs, at)) if slots is not None else None
    prompts = (k_prompt.data_ptr(), v_prompt.data_ptr(), cu_budgets.data_ptr()) if n_items > 0 else (None, None, None)
    _check(_lib.audiokv_decode_shared(C.byref(p.c()), q.data_ptr(), *prompts, n_items, int(total_rows),
                                      cu_seqs.data_ptr() if n_items > 0 else None, n_seqs, int(max_seqs), cs, int(max_own),
                                      _ptr(k_new), _ptr(v_new), _ptr(pos_new), out.data_ptr(), ws.data_ptr(), ws.numel(), _stream()))
    return out


def evict_accumulated_workspace_bytes(p: Params, n_seqs: int, max_own: int, budget: int) -> int:
    out = C.c_size_t(0)
    cp = p.c()
    _check(_lib.audiokv_evict_accumulated_workspace_bytes(C.byref(cp), int(n_seqs), int(max_own), int(budget), C.byref(out)))
    return out.value


def evict_accumulated(p: Params, slots: Slots, n_seqs: int, budget: int, recent: int, max_own: int, *,
                      budgets: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> None:
    """Cuts the rows of every head of `slots` to its budget (`budget`, or the larger of it and budgets[head]) in place, by
    recency and accumulated weight. (More recent rows than the budget: those of the lowest slots stay, not the newest.)"""
    at = _device()
    if budgets is not None and _need_at(budgets, _I32, at, "budgets").numel() < n_seqs * p.n_kv_heads:
        raise ValueError(f"budgets has {budgets.numel()} values, {n_seqs * p.n_kv_heads} needed")
    cs = slots._c(p, n_seqs, at)
    if workspace is not None:
        ws = _workspace_at(workspace, at)
    else:
        ws = torch.empty(max(evict_accumulated_workspace_bytes(p, n_seqs, max_own, budget), 256), dtype=torch.uint8,
                         device=slots.lengths.device)
    _check(_lib.audiokv_evict_accumulated(C.byref(p.c()), C.byref(cs), int(n_seqs), int(budget), _ptr(budgets), int(recent),
                                          int(max_own), _ptr(ws), ws.numel(), _stream()))


PROFILE_STAGES = ("allocate", "score_sweep1", "score_sweep2", "pool_smooth", "select", "compact")


def profile_enable(on: bool) -> None:
    _check(_lib.audiokv_profile_enable(1 if on else 0))


def profile_read() -> dict:
    """Milliseconds of each kernel of the most recent evict() issued while profiling was enabled."""
    buf = (C.c_float * len(PROFILE_STAGES))()
    _check(_lib.audiokv_profile_read(buf))
    return {n: float(buf[i]) for i, n in enumerate(PROFILE_STAGES)}
