"""Python binding of libcertkv.so with the C entry points' names.

Argument marshalling only: shapes and dtypes are read off torch tensors,
outputs and the workspace are allocated with torch on the tensors' device,
and every step of the pass runs in the library's HIP kernels on the current
torch stream.  Layouts follow include/certkv.h.
"""
import ctypes
import math
from dataclasses import dataclass, field
from typing import List, Optional

import torch

from . import _lib
from ._lib import CertKVError


@dataclass
class ProblemSpec:
    layers: int
    kv_heads: int
    group: int
    head_dim: int
    window: int
    seqlens: List[int]
    dtype: torch.dtype = torch.bfloat16
    softmax_scale: float = 0.0
    causal: bool = True
    dry_run: bool = False
    keep_window: bool = False   # window keys ranked first, never evicted
    # one-factor ablations: "centered" | "uncentered" | "tail_mass";
    # "lagrangian" | "uniform" | "greedy"; slot=False gives the slot's row to
    # one more real token per head
    statistic: str = "centered"
    allocator: str = "lagrangian"
    slot: bool = True
    status: Optional[torch.Tensor] = None  # device int32 [1]: CERTKV_ENONFINITE on non-finite input
    _cu: object = field(default=None, repr=False)

    @property
    def batch(self):
        return len(self.seqlens)

    @property
    def total_tokens(self):
        return int(sum(self.seqlens))

    @property
    def units(self):
        return self.layers * self.batch * self.kv_heads

    def cu_seqlens(self):
        cu = [0]
        for n in self.seqlens:
            cu.append(cu[-1] + int(n))
        return cu

    def c_problem(self):
        """The problem as the C entry points take it, the caller's own to change."""
        cu = self.cu_seqlens()
        self._cu = (ctypes.c_int64 * len(cu))(*cu)  # kept alive with the spec
        dt = _dtype_code(self.dtype)
        flags = (_lib.CERTKV_CAUSAL if self.causal else 0) | (
            _lib.CERTKV_DRY_RUN if self.dry_run else 0) | (
            _lib.CERTKV_KEEP_WINDOW if self.keep_window else 0) | {
            "centered": 0, "uncentered": _lib.CERTKV_STAT_UNCENTERED,
            "tail_mass": _lib.CERTKV_STAT_TAIL_MASS}[self.statistic] | {
            "lagrangian": 0, "uniform": _lib.CERTKV_ALLOC_UNIFORM,
            "greedy": _lib.CERTKV_ALLOC_GREEDY}[self.allocator] | (
            0 if self.slot else _lib.CERTKV_NO_SLOT)
        return _lib.Problem(self.layers, self.batch, self.kv_heads, self.group, self.head_dim,
                            self.window, ctypes.cast(self._cu, ctypes.POINTER(ctypes.c_int64)),
                            dt, dt, float(self.softmax_scale), flags,
                            self.status.data_ptr() if self.status is not None else None)

    def _problem(self):
        # c_problem for this module's calls, which do not change it: made anew when a field
        # has changed (a call of a small problem would take longer to describe than to run)
        key = (self.layers, self.kv_heads, self.group, self.head_dim, self.window,
               tuple(self.seqlens), self.dtype, self.softmax_scale, self.causal, self.dry_run,
               self.keep_window, self.statistic, self.allocator, self.slot,
               self.status.data_ptr() if self.status is not None else None)
        kept = self.__dict__.get("_c")
        if kept is not None and kept[0] == key:
            return kept[1]
        p = self.c_problem()
        self.__dict__["_c"] = (key, p)
        return p

    def __getstate__(self):  # (a copy describes itself anew)
        return {k: v for k, v in self.__dict__.items() if k not in ("_c", "_paged")}


def _dtype_code(dt):
    if dt == torch.bfloat16:
        return _lib.CERTKV_BF16
    if dt == torch.float32:
        return _lib.CERTKV_F32
    raise ValueError(f"unsupported dtype {dt}")


def _tensor(t: torch.Tensor) -> _lib.Tensor:
    s = t.stride()
    if len(s) != 4 or s[3] != 1:
        raise ValueError("expected a [layers][tokens][heads][head_dim] tensor with contiguous last dim")
    return _lib.Tensor(t.data_ptr(), s[0], s[1], s[2])


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(device):
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _run(dev, what, *args):
    """The entry point `what` with args and the current stream of dev, dev being current."""
    fn = getattr(_lib.lib(), what)
    index = dev.index
    if index is None:
        raise ValueError(f"{what}: expected tensors on a GPU")
    if index == torch._C._cuda_getDevice():
        _check(fn(*args, torch._C._cuda_getCurrentRawStream(index)), what)
    else:
        with torch.cuda.device(dev):
            _check(fn(*args, torch._C._cuda_getCurrentRawStream(index)), what)


def _check(st, what):
    if st != _lib.CERTKV_OK:
        raise CertKVError(st, what)


def workspace_size(spec: ProblemSpec, stage: int) -> int:
    p = spec._problem()
    return int(_lib.lib().certkv_workspace_size(ctypes.byref(p), stage))


def _workspace(spec, stage, device):
    n = workspace_size(spec, stage)
    if n == 0:
        return None, 0
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    assert ws.data_ptr() % 256 == 0
    return ws, n


def _lse_shape(spec):
    return (spec.layers, spec.batch * spec.window, spec.kv_heads * spec.group)


def score(spec: ProblemSpec, q_win, k, with_ksum=False, lse_in=None, with_lse=False):
    """Window-mass scores [L][H][T] fp32; with_ksum adds sum_j (s_j)_+ k_j [U][d] fp64 and
    with_lse the row log-sum-exp [L][B*w][Hq] fp32 (in that order).  lse_in: the caller's
    row log-sum-exp in the same layout (the row-sum pass is then skipped)."""
    L = _lib.lib()
    dev = k.device
    scores = torch.empty((spec.layers, spec.kv_heads, spec.total_tokens), dtype=torch.float32,
                         device=dev)
    ksum = torch.empty((spec.units, spec.head_dim), dtype=torch.float64, device=dev) \
        if with_ksum else None
    lse = torch.empty(_lse_shape(spec), dtype=torch.float32, device=dev) if with_lse else None
    if lse_in is not None:
        assert lse_in.dtype == torch.float32 and lse_in.is_contiguous()
        assert tuple(lse_in.shape) == _lse_shape(spec)
    ws, n = _workspace(spec, _lib.STAGE_SCORE, dev)
    p = spec._problem()
    _check(L.certkv_score(ctypes.byref(p), _tensor(q_win), _tensor(k), _ptr(lse_in), _ptr(scores),
                          _ptr(ksum), _ptr(lse), _ptr(ws), n, _stream(dev)), "certkv_score")
    out = [scores] + ([ksum] if with_ksum else []) + ([lse] if with_lse else [])
    return out[0] if len(out) == 1 else tuple(out)


def score_noalloc(spec: ProblemSpec, q_win, k, scores, ksum=None, lse_out=None, lse_in=None):
    """certkv_score with the library's fixed device workspace: the caller
    passes every output (scores [L][H][T] fp32; optional ksum [U][d] fp64 and
    lse_out [L][B*w][Hq] fp32) and nothing is allocated."""
    L = _lib.lib()
    dev = k.device
    assert scores.dtype == torch.float32 and scores.is_contiguous()
    assert tuple(scores.shape) == (spec.layers, spec.kv_heads, spec.total_tokens)
    if ksum is not None:
        assert ksum.dtype == torch.float64 and tuple(ksum.shape) == (spec.units, spec.head_dim)
    for t in (lse_in, lse_out):
        if t is not None:
            assert t.dtype == torch.float32 and t.is_contiguous()
            assert tuple(t.shape) == _lse_shape(spec)
    p = spec._problem()
    _check(L.certkv_score_noalloc(ctypes.byref(p), _tensor(q_win), _tensor(k), _ptr(lse_in),
                                  _ptr(scores), _ptr(ksum), _ptr(lse_out), _stream(dev)),
           "certkv_score_noalloc")
    return scores


def allocate(spec: ProblemSpec, scores, v, n_keep, alpha=0.2, steps=40, with_perm=False,
             with_curves=False, with_vsum=False):
    """Budgets [U] int32 (+ perm, curves [L][H][T], vsum [U][d])."""
    L = _lib.lib()
    dev = v.device
    budgets = torch.empty(spec.units, dtype=torch.int32, device=dev)
    shape = (spec.layers, spec.kv_heads, spec.total_tokens)
    perm = torch.empty(shape, dtype=torch.int32, device=dev) if with_perm else None
    curves = torch.empty(shape, dtype=torch.float32, device=dev) if with_curves else None
    vsum = torch.empty((spec.units, spec.head_dim), dtype=torch.float64, device=dev) \
        if with_vsum else None
    nk = (ctypes.c_int32 * spec.batch)(*[int(x) for x in n_keep])
    ws, n = _workspace(spec, _lib.STAGE_ALLOCATE, dev)
    p = spec._problem()
    _check(L.certkv_allocate(ctypes.byref(p), _ptr(scores), _tensor(v), nk, float(alpha),
                             int(steps), _ptr(budgets), _ptr(perm), _ptr(curves), _ptr(vsum),
                             _ptr(ws), n, _stream(dev)), "certkv_allocate")
    out = {"budgets": budgets}
    if with_perm:
        out["perm"] = perm
    if with_curves:
        out["curves"] = curves
    if with_vsum:
        out["vsum"] = vsum
    return out


def allocate_curves(spec: ProblemSpec, curves, n_keep, alpha=0.2, steps=40):
    """Budgets [U] int32 from caller-supplied fp32 curves [L][H][T]."""
    L = _lib.lib()
    dev = curves.device
    budgets = torch.empty(spec.units, dtype=torch.int32, device=dev)
    nk = (ctypes.c_int32 * spec.batch)(*[int(x) for x in n_keep])
    # min/max scratch: same layout as the allocation stage's
    ws, n = _workspace(spec, _lib.STAGE_ALLOCATE, dev)
    p = spec._problem()
    _check(L.certkv_allocate_curves(ctypes.byref(p), _ptr(curves), nk, float(alpha), int(steps),
                                    _ptr(budgets), _ptr(ws), n, _stream(dev)),
           "certkv_allocate_curves")
    return budgets


def select(spec: ProblemSpec, scores, budgets=None, mode="budget", retain_mass=0.9,
           with_mask=False):
    """(budgets, kept_offsets [U+1] int64, kept_idx int32[, kept_mask [L][H][T] uint8])."""
    L = _lib.lib()
    dev = scores.device
    if mode == "budget":
        assert budgets is not None
        b = budgets.clone()
        cap = int(b.clamp(min=0).sum().item()) if b.numel() else 0
        m = _lib.CERTKV_SELECT_BUDGET
    else:
        b = torch.empty(spec.units, dtype=torch.int32, device=dev)
        cap = spec.layers * spec.kv_heads * spec.total_tokens
        m = _lib.CERTKV_SELECT_COVERAGE
    kept_offsets = torch.empty(spec.units + 1, dtype=torch.int64, device=dev)
    kept_idx = torch.empty(max(cap, 1), dtype=torch.int32, device=dev)
    mask = torch.empty((spec.layers, spec.kv_heads, spec.total_tokens), dtype=torch.uint8,
                       device=dev) if with_mask else None
    ws, n = _workspace(spec, _lib.STAGE_SELECT, dev)
    p = spec._problem()
    _check(L.certkv_select(ctypes.byref(p), _ptr(scores), _ptr(b), m, float(retain_mass),
                           _ptr(kept_offsets), _ptr(kept_idx), cap, _ptr(mask), _ptr(ws), n,
                           _stream(dev)), "certkv_select")
    return (b, kept_offsets, kept_idx, mask) if with_mask else (b, kept_offsets, kept_idx)


def tail_summary(spec: ProblemSpec, scores, k, v, kept_offsets, kept_idx, ksum=None, vsum=None):
    """(k_star [U][d] fp32, v_star [U][d] fp32, tail_mass [U] fp64)."""
    L = _lib.lib()
    dev = k.device
    k_star = torch.empty((spec.units, spec.head_dim), dtype=torch.float32, device=dev)
    v_star = torch.empty_like(k_star)
    tail_mass = torch.empty(spec.units, dtype=torch.float64, device=dev)
    ws, n = _workspace(spec, _lib.STAGE_TAIL, dev)
    p = spec._problem()
    _check(L.certkv_tail_summary(ctypes.byref(p), _ptr(scores), _tensor(k), _tensor(v),
                                 _ptr(kept_offsets), _ptr(kept_idx), _ptr(ksum), _ptr(vsum),
                                 _ptr(k_star), _ptr(v_star), _ptr(tail_mass), _ptr(ws), n,
                                 _stream(dev)), "certkv_tail_summary")
    return k_star, v_star, tail_mass


def compact(spec: ProblemSpec, k, v, kept_offsets, kept_idx, k_star, v_star):
    """(k_packed, v_packed [rows][d], pos_packed [rows], packed_offsets [U+1])."""
    L = _lib.lib()
    dev = k.device
    rows = int(kept_offsets[-1].item()) + (spec.units if spec.slot else 0)
    k_packed = torch.empty((rows, spec.head_dim), dtype=k.dtype, device=dev)
    v_packed = torch.empty_like(k_packed)
    pos_packed = torch.empty(rows, dtype=torch.int32, device=dev)
    packed_offsets = torch.empty(spec.units + 1, dtype=torch.int64, device=dev)
    p = spec._problem()
    _check(L.certkv_compact(ctypes.byref(p), _tensor(k), _tensor(v), _ptr(kept_offsets),
                            _ptr(kept_idx), _ptr(k_star), _ptr(v_star), _ptr(k_packed),
                            _ptr(v_packed), _ptr(pos_packed), _ptr(packed_offsets), _stream(dev)),
           "certkv_compact")
    return k_packed, v_packed, pos_packed, packed_offsets


def decode_workspace_size(spec: ProblemSpec, tq: int, max_rows: int = 0) -> int:
    p = spec._problem()
    return int(_lib.lib().certkv_decode_workspace_size(ctypes.byref(p), int(tq), int(max_rows)))


class DecodeBuffers:
    """Preallocated outputs and workspace of certkv_decode (reusable); with fmt
    ("bf16", "mxfp8" or "mxfp4") those of certkv_decode_mx and certkv_decode_tree
    over a cache of that format and tn new rows per sequence, with pages (a PagedCache)
    those of certkv_decode_paged over it."""

    def __init__(self, spec: ProblemSpec, tq: int, device, with_lse=False, max_rows=0, tn=0,
                 fmt=None, pages=None):
        self.tq = int(tq)
        self.max_rows = int(max_rows)
        rows = spec.layers * spec.batch * self.tq
        hq = spec.kv_heads * spec.group
        self.out = torch.empty((spec.layers, spec.batch * self.tq, hq, spec.head_dim),
                               dtype=torch.float32, device=device)
        self.lse = torch.empty((spec.layers, spec.batch * self.tq, hq), dtype=torch.float32,
                               device=device) if with_lse else None
        self.tn = int(tn)
        self.fmt = fmt
        self.paged = pages is not None
        if pages is not None:
            self.ws_bytes = decode_paged_workspace_size(spec, pages, self.tq, self.max_rows)
        elif fmt is None:
            self.ws_bytes = decode_workspace_size(spec, self.tq, self.max_rows)
        else:
            self.ws_bytes = decode_cache_workspace_size(spec, fmt, self.tq, self.tn, self.max_rows)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        assert self.ws.data_ptr() % 256 == 0 and rows > 0


def decode(spec: ProblemSpec, q_new, k_packed, v_packed, packed_offsets, tq, with_lse=False,
           bufs=None, max_rows=0):
    """Attention of tq new queries per sequence (q_new [L][B*tq][Hq][d]) over the packed
    cache: out [L][B*tq][Hq][d] fp32 (and the natural-log lse [L][B*tq][Hq] with_lse).
    max_rows bounds the rows of any head's segment (0: what the longest sequence can have)."""
    L = _lib.lib()
    dev = q_new.device
    if bufs is None:
        bufs = DecodeBuffers(spec, tq, dev, with_lse=with_lse, max_rows=max_rows)
    assert bufs.tq >= int(tq)  # (the outputs' room)
    assert k_packed.is_contiguous() and v_packed.is_contiguous()
    p = spec._problem()
    _check(L.certkv_decode(ctypes.byref(p), _tensor(q_new), int(tq), bufs.max_rows, _ptr(k_packed),
                           _ptr(v_packed), _ptr(packed_offsets), _ptr(bufs.out), _ptr(bufs.lse),
                           _ptr(bufs.ws), bufs.ws_bytes, _stream(dev)), "certkv_decode")
    return (bufs.out, bufs.lse) if with_lse else bufs.out


def cluster_tail(spec: ProblemSpec, k, v, perm, budgets, m):
    """Clustered tail summaries: m contiguous groups of each head's evicted
    ranks.  Returns dict(kbar, vbar [U][m][d] in the cache dtype, count [U][m]
    int32, rk, rv [U][m] fp32 radii, vmax_kept [U] fp32)."""
    L = _lib.lib()
    dev = k.device
    U, D = spec.units, spec.head_dim
    out = dict(kbar=torch.empty((U, m, D), dtype=k.dtype, device=dev),
               vbar=torch.empty((U, m, D), dtype=k.dtype, device=dev),
               count=torch.empty((U, m), dtype=torch.int32, device=dev),
               rk=torch.empty((U, m), dtype=torch.float32, device=dev),
               rv=torch.empty((U, m), dtype=torch.float32, device=dev),
               vmax_kept=torch.empty(U, dtype=torch.float32, device=dev))
    p = spec._problem()
    _check(L.certkv_cluster_tail(ctypes.byref(p), _tensor(k), _tensor(v), _ptr(perm),
                                 _ptr(budgets), int(m), _ptr(out["kbar"]), _ptr(out["vbar"]),
                                 _ptr(out["count"]), _ptr(out["rk"]), _ptr(out["rv"]),
                                 _ptr(out["vmax_kept"]), _stream(dev)), "certkv_cluster_tail")
    return out


def decode_clustered(spec: ProblemSpec, q_new, k_packed, v_packed, packed_offsets, tq, clusters,
                     max_rows=0):
    """Decode over kept-row segments plus the clustered tail summaries of
    cluster_tail: (out [L][B*tq][Hq][d], lse, bound [L][B*tq][Hq]) fp32, the
    bound being the runtime certificate (inf where it does not hold)."""
    L = _lib.lib()
    dev = q_new.device
    bufs = DecodeBuffers(spec, tq, dev, with_lse=True, max_rows=max_rows)
    bound = torch.empty_like(bufs.lse)
    m = clusters["count"].shape[1]
    p = spec._problem()
    _check(L.certkv_decode_clustered(
        ctypes.byref(p), _tensor(q_new), int(tq), bufs.max_rows, _ptr(k_packed), _ptr(v_packed),
        _ptr(packed_offsets), int(m), _ptr(clusters["kbar"]), _ptr(clusters["vbar"]),
        _ptr(clusters["count"]), _ptr(clusters["rk"]), _ptr(clusters["rv"]),
        _ptr(clusters["vmax_kept"]), _ptr(bufs.out), _ptr(bufs.lse), _ptr(bound), _ptr(bufs.ws),
        bufs.ws_bytes, _stream(dev)), "certkv_decode_clustered")
    return bufs.out, bufs.lse, bound


_FORMATS = {"bf16": _lib.CERTKV_CACHE_BF16, "mxfp8": _lib.CERTKV_CACHE_MXFP8,
            "mxfp4": _lib.CERTKV_CACHE_MXFP4}


def _format_code(fmt):
    if fmt not in _FORMATS:
        raise ValueError(f"unsupported cache format {fmt!r}")
    return _FORMATS[fmt]


@dataclass
class MxCache:
    """A packed cache in microscaled codes ("mxfp8": k, v [rows][d] uint8; "mxfp4":
    [rows][d/2], the even dim in the low half of a byte), a scale byte for every 32 dims
    (k_scales, v_scales [rows][d/32]), the units' offsets [U+1] int64 and, where
    compact_mx wrote it, the rows' positions [rows] int32."""
    format: str
    k: torch.Tensor
    k_scales: torch.Tensor
    v: torch.Tensor
    v_scales: torch.Tensor
    offsets: torch.Tensor
    pos: Optional[torch.Tensor] = None

    @staticmethod
    def empty(spec: ProblemSpec, rows: int, fmt: str, device):
        """Buffers for a cache of `rows` packed rows."""
        if _format_code(fmt) == _lib.CERTKV_CACHE_BF16:
            raise ValueError("a microscaled cache is mxfp8 or mxfp4")
        d = spec.head_dim
        codes = (rows, d if fmt == "mxfp8" else d // 2)
        u8 = dict(dtype=torch.uint8, device=device)
        return MxCache(fmt, torch.empty(codes, **u8), torch.empty((rows, d // 32), **u8),
                       torch.empty(codes, **u8), torch.empty((rows, d // 32), **u8),
                       torch.empty(spec.units + 1, dtype=torch.int64, device=device),
                       torch.empty(rows, dtype=torch.int32, device=device))

    @property
    def rows(self):
        return self.k.shape[0]

    @property
    def head_dim(self):
        return self.k.shape[1] * (1 if self.format == "mxfp8" else 2)

    def __setattr__(self, name, value):
        object.__setattr__(self, "_seen", None)
        object.__setattr__(self, name, value)

    def _check_tensors(self):
        if self.format not in ("mxfp8", "mxfp4"):
            raise ValueError(f"a microscaled cache is mxfp8 or mxfp4, not {self.format!r}")
        k, ks, v, vs = self.k, self.k_scales, self.v, self.v_scales
        rows, wide = k.shape
        scales = (rows, wide // (32 if self.format == "mxfp8" else 16))
        assert v.shape == k.shape and ks.shape == scales and vs.shape == scales
        assert k.dtype == v.dtype == ks.dtype == vs.dtype == torch.uint8
        assert k.is_contiguous() and v.is_contiguous() and ks.is_contiguous() and vs.is_contiguous()
        assert self.offsets.dtype == torch.int64 and self.offsets.is_contiguous()
        assert v.device == ks.device == vs.device == self.offsets.device == k.device
        if self.pos is not None:
            assert self.pos.dtype == torch.int32 and self.pos.is_contiguous()
            assert self.pos.numel() >= rows and self.pos.device == k.device

    def _addresses(self):
        """Of k, k_scales, v, v_scales, offsets, pos, whose shapes and types are checked when a
        field has changed, or one of them in place: its address, or the rows that k says there
        are (others keep the memory that they had under the same address)."""
        k, pos = self.k, self.pos
        seen = (k.data_ptr(), self.k_scales.data_ptr(), self.v.data_ptr(),
                self.v_scales.data_ptr(), self.offsets.data_ptr(),
                None if pos is None else pos.data_ptr(), k.numel())
        if seen != self._seen:
            self._check_tensors()
            object.__setattr__(self, "_seen", seen)
        return seen

    def c_cache(self):
        k, ks, v, vs, off, _, _ = self._addresses()
        return _lib.Cache(_FORMATS[self.format], k, v, ks, vs, off)


_READ_SPECS = {}


def compact_mx(spec: ProblemSpec, k, v, kept_offsets, kept_idx, k_star, v_star, fmt, cache=None):
    """compact with the packed rows quantised as they are written: an MxCache of format fmt
    ("mxfp8" or "mxfp4"), `cache` if one is given (its rows past the last packed one are left
    as they are; rows that it has no room for are left out, and reported in spec.status)."""
    dev = k.device
    if cache is None:
        rows = int(kept_offsets[-1].item()) + (spec.units if spec.slot else 0)
        cache = MxCache.empty(spec, rows, fmt, dev)
    units, d = spec.units, spec.head_dim
    assert k.dtype == v.dtype == spec.dtype
    assert k.shape == v.shape == (spec.layers, sum(spec.seqlens), spec.kv_heads, d)
    assert v.device == kept_offsets.device == kept_idx.device == cache.k.device == dev
    assert kept_offsets.dtype == torch.int64 and kept_idx.dtype == torch.int32
    assert kept_offsets.is_contiguous() and kept_idx.is_contiguous()
    assert cache.offsets.numel() == kept_offsets.numel() == units + 1
    assert cache.format == fmt and cache.pos is not None
    assert cache.k.shape[1] == (d if fmt == "mxfp8" else d // 2)
    if k_star is not None and v_star is not None:
        assert k_star.dtype == v_star.dtype == torch.float32 and k_star.device == v_star.device == dev
        assert k_star.numel() == v_star.numel() == units * d
        assert k_star.is_contiguous() and v_star.is_contiguous()
    c_k, c_ks, c_v, c_vs, c_off, c_pos, _ = cache._addresses()
    _run(dev, "certkv_compact_mx_bounded", ctypes.byref(spec._problem()), _format_code(fmt),
         _tensor(k), _tensor(v), kept_offsets.data_ptr(), kept_idx.data_ptr(), kept_idx.numel(),
         _ptr(k_star), _ptr(v_star), c_k, c_ks, c_v, c_vs, c_pos, cache.k.shape[0], c_off)
    return cache


def read_mx(cache: MxCache, dtype=torch.bfloat16, first_row=0, rows=None, out=None):
    """The values (k, v) [rows][d] of a cache's rows first_row .. first_row + rows - 1 (all
    from first_row on by default), exact in bf16 and fp32; out: the two tensors to write."""
    c = cache.c_cache()
    rows_all, d = cache.k.shape
    d = d if cache.format == "mxfp8" else 2 * d
    n = rows_all - first_row if rows is None else int(rows)
    assert 0 <= first_row and 0 <= n and first_row + n <= rows_all
    if out is None:
        out = [torch.empty((n, d), dtype=dtype, device=cache.k.device) for _ in range(2)]
    ko, vo = out
    assert ko.shape == vo.shape == (n, d) and ko.dtype == vo.dtype
    assert ko.is_contiguous() and vo.is_contiguous() and ko.device == vo.device == cache.k.device
    if d not in _READ_SPECS:  # (of the problem only the row length is read)
        _READ_SPECS[d] = ProblemSpec(1, 1, 1, d, 1, [1])
    _run(cache.k.device, "certkv_read_mx", ctypes.byref(_READ_SPECS[d]._problem()), c,
         int(first_row), n, _dtype_code(ko.dtype), ko.data_ptr(), vo.data_ptr())
    return ko, vo


def decode_cache_workspace_size(spec: ProblemSpec, fmt: str, tq: int, tn: int = 0,
                                max_rows: int = 0) -> int:
    p = spec._problem()
    return int(_lib.lib().certkv_decode_cache_workspace_size(
        ctypes.byref(p), _format_code(fmt), int(tq), int(tn), int(max_rows)))


def _check_queries(spec, q_new, tq):
    assert q_new.dtype == torch.bfloat16
    assert q_new.shape == (spec.layers, spec.batch * int(tq), spec.kv_heads * spec.group,
                           spec.head_dim)


def _cache_buffers(spec, q_new, fmt, tq, tn, dev, with_lse, bufs, max_rows):
    if bufs is None:
        bufs = DecodeBuffers(spec, tq, dev, with_lse=with_lse, max_rows=max_rows, tn=tn, fmt=fmt)
    assert bufs.fmt == fmt and bufs.tq == int(tq) and bufs.tn == int(tn)
    assert bufs.out.shape == q_new.shape and bufs.out.device == dev  # (as the queries, checked)
    assert bufs.lse is not None or not with_lse
    return bufs


def decode_mx(spec: ProblemSpec, q_new, cache: MxCache, tq, with_lse=False, bufs=None, max_rows=0):
    """decode over a microscaled packed cache: out [L][B*tq][Hq][d] fp32 (and the natural-log
    lse [L][B*tq][Hq] with_lse).  bufs: DecodeBuffers(..., fmt=cache.format).  spec.dtype is
    bfloat16, the queries': a cache written from fp32 rows is attended under
    dataclasses.replace(spec, dtype=torch.bfloat16)."""
    dev = q_new.device
    _check_queries(spec, q_new, tq)
    assert cache.head_dim == spec.head_dim and cache.offsets.numel() == spec.units + 1
    assert cache.k.device == dev
    bufs = _cache_buffers(spec, q_new, cache.format, tq, 0, dev, with_lse, bufs, max_rows)
    _run(dev, "certkv_decode_mx", ctypes.byref(spec._problem()), _tensor(q_new), bufs.tq,
         bufs.max_rows, cache.c_cache(), bufs.out.data_ptr(), _ptr(bufs.lse), bufs.ws.data_ptr(),
         bufs.ws_bytes)
    return (bufs.out, bufs.lse) if with_lse else bufs.out


def decode_tree(spec: ProblemSpec, q_new, cache, tq, k_new, v_new, mask=None, with_lse=False,
                bufs=None, max_rows=0):
    """Attention of tq drafted tokens per sequence (q_new [L][B*tq][Hq][d]) over the packed
    cache and tn new rows per sequence (k_new, v_new [L][B*tn][H][d]): the tokens since the
    compression, a tree of drafted ones.  cache: an MxCache, or (k_packed, v_packed,
    packed_offsets) of a bf16 one.  mask [B][tq][tn] bool or uint8: the new rows that each
    query sees; None: j <= tn - tq + t, the last tq rows being the queries' own.  Returns out
    [L][B*tq][Hq][d] fp32 (and lse [L][B*tq][Hq] with_lse); a query that sees nothing is out 0,
    lse -inf.  bufs: DecodeBuffers(..., tn=tn, fmt=format of the cache)."""
    dev = q_new.device
    _check_queries(spec, q_new, tq)
    tn = k_new.shape[1] // spec.batch
    new = (spec.layers, spec.batch * tn, spec.kv_heads, spec.head_dim)
    assert k_new.shape == new and v_new.shape == new
    assert k_new.dtype == v_new.dtype == torch.bfloat16
    assert k_new.device == v_new.device == dev
    if mask is not None:
        assert mask.device == dev
        assert mask.dtype in (torch.bool, torch.uint8) and mask.is_contiguous()
        assert mask.shape == (spec.batch, int(tq), tn)
    if isinstance(cache, MxCache):
        fmt, offsets, c = cache.format, cache.offsets, cache.c_cache()
        assert cache.head_dim == spec.head_dim
    else:
        kp, vp, offsets = cache
        assert kp.is_contiguous() and vp.is_contiguous() and kp.shape == vp.shape
        assert kp.dtype == vp.dtype == torch.bfloat16 and kp.shape[1] == spec.head_dim
        assert kp.device == vp.device == dev and offsets.is_contiguous()
        fmt = "bf16"
        c = _lib.Cache(_format_code(fmt), kp.data_ptr(), vp.data_ptr(), None, None,
                       offsets.data_ptr())
    assert offsets.dtype == torch.int64 and offsets.numel() == spec.units + 1
    assert offsets.device == dev
    bufs = _cache_buffers(spec, q_new, fmt, tq, tn, dev, with_lse, bufs, max_rows)
    _run(dev, "certkv_decode_tree", ctypes.byref(spec._problem()), _tensor(q_new), bufs.tq,
         bufs.max_rows, c, _tensor(k_new), _tensor(v_new), tn, _ptr(mask), bufs.out.data_ptr(),
         _ptr(bufs.lse), bufs.ws.data_ptr(), bufs.ws_bytes)
    return (bufs.out, bufs.lse) if with_lse else bufs.out


@dataclass
class PagedCache:
    """Rows of K and V in pages of a pool, `page` rows of one list to a page.  Lists are
    sequences (k, v [L][pages][page][H][d], any order of the axes in memory but for d, whose rows
    are consecutive), or, per_head, the (layer, sequence, head) units ([pages][page][d]).  format
    "bf16", or "mxfp8" and "mxfp4": k, v uint8 codes (of d or d/2 bytes), k_scales and v_scales
    as them with d/32 bytes.  table [lists][max_pages] int32, offsets [lists+1] int64, ring
    [pages] int32 and free [2] int64 (first place and number of the ring's free pages).  k and v
    may be None where only tables are planned."""
    format: str
    page: int
    k: Optional[torch.Tensor]
    v: Optional[torch.Tensor]
    table: torch.Tensor
    offsets: torch.Tensor
    k_scales: Optional[torch.Tensor] = None
    v_scales: Optional[torch.Tensor] = None
    ring: Optional[torch.Tensor] = None
    free: Optional[torch.Tensor] = None
    per_head: bool = False

    @staticmethod
    def empty(spec: ProblemSpec, num_pages: int, page: int, max_pages: int, device, fmt="bf16",
              per_head=False, head_major=False):
        """A pool of num_pages free pages and empty lists of max_pages pages at most.  head_major:
        the rows of one head of a page are consecutive, not the heads of one row."""
        code = _format_code(fmt)
        d = spec.head_dim
        wide, dt = {_lib.CERTKV_CACHE_BF16: (d, torch.bfloat16), _lib.CERTKV_CACHE_MXFP8:
                    (d, torch.uint8), _lib.CERTKV_CACHE_MXFP4: (d // 2, torch.uint8)}[code]
        L, H = spec.layers, spec.kv_heads

        def pool(width, dtype):
            if per_head:
                return torch.empty((num_pages, page, width), dtype=dtype, device=device)
            if head_major:
                return torch.empty((L, num_pages, H, page, width), dtype=dtype,
                                   device=device).transpose(2, 3)
            return torch.empty((L, num_pages, page, H, width), dtype=dtype, device=device)

        lists = spec.units if per_head else spec.batch
        scales = [pool(d // 32, torch.uint8) if fmt != "bf16" else None for _ in range(2)]
        return PagedCache(fmt, page, pool(wide, dt), pool(wide, dt),
                          torch.full((lists, max_pages), -1, dtype=torch.int32, device=device),
                          torch.zeros(lists + 1, dtype=torch.int64, device=device), *scales,
                          ring=torch.arange(num_pages, dtype=torch.int32, device=device),
                          free=torch.tensor([0, num_pages], device=device), per_head=per_head)

    @property
    def lists(self):
        return self.offsets.numel() - 1

    @property
    def num_pages(self):
        if self.k is None:
            return self.ring.numel()
        return self.k.shape[0 if self.per_head else 1]

    def layer(self, layer: int, layers: int):
        """Layer `layer` of `layers` as a cache of its own, of the same tensors, for calls whose
        spec has one layer (not to be resized: its lists are the whole cache's)."""
        assert 0 <= layer < layers
        if self.per_head:
            assert self.lists % layers == 0
            n = self.lists // layers
            rows, at = (self.k, self.v, self.k_scales, self.v_scales), slice(layer * n, layer * n + n)
            table, offsets = self.table[at], self.offsets[layer * n:layer * n + n + 1]
        else:
            assert self.k.shape[0] == layers
            rows = [t if t is None else t[layer:layer + 1]
                    for t in (self.k, self.v, self.k_scales, self.v_scales)]
            table, offsets = self.table, self.offsets
        return PagedCache(self.format, self.page, rows[0], rows[1], table, offsets, rows[2], rows[3],
                          per_head=self.per_head)

    def __setattr__(self, name, value):
        object.__setattr__(self, "_seen", None)
        object.__setattr__(self, name, value)

    def __getstate__(self):  # (a copy describes itself anew)
        return {k: v for k, v in self.__dict__.items() if k != "_seen"}

    def __setstate__(self, state):
        self.__dict__.update(state, _seen=None)

    def _strides(self, t, width):
        # in rows: of layer, page, row and head
        s = t.stride()
        assert s[-1] == 1 and t.shape[-1] == width
        n = len(s) - 1
        # (an axis of one element may have any stride)
        rows = [0 if t.shape[i] == 1 and i != n - (1 if self.per_head else 2) else s[i]
                for i in range(n)]
        assert all(x % width == 0 for x in rows), "rows of a page's pool are consecutive"
        rows = [x // width for x in rows]
        return [0, rows[0], rows[1], 0] if self.per_head else rows

    def _c_pages(self, spec):
        """(what it was made from, the cache as the C entry points take it, a reference to that, the
        tensors' GPU, their device).  Shapes and types are checked when a field has changed, or a
        tensor's address, or the lists and heads that the spec says there are."""
        k, ks, ring = self.k, self.k_scales, self.ring
        seen = (self.table.data_ptr(), self.table.numel(), self.offsets.data_ptr(), spec.layers,
                spec.kv_heads, spec.head_dim, len(spec.seqlens))
        if k is not None:
            v = self.v
            seen += (k.data_ptr(), k.numel(), k.stride(), v.data_ptr(), v.stride())
        if ks is not None:
            vs = self.v_scales
            seen += (ks.data_ptr(), ks.stride(), vs.data_ptr(), vs.stride())
        if ring is not None:
            seen += (ring.data_ptr(), self.free.data_ptr())
        kept = self._seen
        if kept is not None and kept[0] == seen:
            return kept
        dev = self.table.device
        strides = [0, 0, 1, 0]
        if k is not None:
            d = spec.head_dim
            width = {"bf16": d, "mxfp8": d, "mxfp4": d // 2}.get(self.format)
            if width is None:
                raise ValueError(f"unsupported cache format {self.format!r}")
            shape = (k.shape[0], self.page) if self.per_head else \
                (spec.layers, k.shape[1], self.page, spec.kv_heads)
            dt = torch.bfloat16 if self.format == "bf16" else torch.uint8
            strides = self._strides(k, width)
            for t in (k, self.v):
                assert t.shape == shape + (width,) and t.dtype == dt and t.device == dev
                assert self._strides(t, width) == strides
            if self.format != "bf16":
                for t in (self.k_scales, self.v_scales):
                    assert t.shape == shape + (d // 32,) and t.dtype == torch.uint8
                    assert t.device == dev and self._strides(t, d // 32) == strides
        lists = spec.units if self.per_head else spec.batch
        assert self.table.dtype == torch.int32 and self.table.is_contiguous()
        assert self.table.dim() == 2 and self.table.shape[0] == lists
        assert self.offsets.dtype == torch.int64 and self.offsets.is_contiguous()
        assert self.offsets.numel() == lists + 1 and self.offsets.device == dev
        if ring is not None:
            assert ring.dtype == torch.int32 and ring.is_contiguous()
            assert ring.numel() == self.num_pages and ring.device == dev
            assert self.free.dtype == torch.int64 and self.free.is_contiguous()
            assert self.free.numel() == 2 and self.free.device == dev
        mx = k is not None and self.format != "bf16"
        c = _lib.Pages(_format_code(self.format), int(self.page), self.num_pages,
                       self.table.shape[1], int(self.per_head), *strides, _ptr(k), _ptr(self.v),
                       self.k_scales.data_ptr() if mx else None,
                       self.v_scales.data_ptr() if mx else None, self.table.data_ptr(),
                       self.offsets.data_ptr(), _ptr(ring), _ptr(self.free))
        kept = (seen, c, ctypes.byref(c), self.table.get_device(), dev)
        object.__setattr__(self, "_seen", kept)
        return kept


def _page_problem(spec):
    # The problem as the paged calls read it, without the sequences' lengths: kept with the spec
    # until a field changes.
    key = (spec.layers, len(spec.seqlens), spec.kv_heads, spec.group, spec.head_dim, spec.dtype,
           spec.softmax_scale, spec.dry_run, None if spec.status is None else spec.status.data_ptr())
    kept = spec.__dict__.get("_paged")
    if kept is not None and kept[0] == key:
        return kept[1]
    dt = _dtype_code(spec.dtype)
    p = _lib.Problem(key[0], key[1], key[2], key[3], key[4], 1, None, dt, dt, float(key[6]),
                     _lib.CERTKV_DRY_RUN if key[7] else 0, key[8])
    spec.__dict__["_paged"] = (key, ctypes.byref(p))
    return spec.__dict__["_paged"][1]


_PAGED = {}  # the paged entry points, by name


def _run_paged(index, what, *args):
    """_run with the GPU's index (a call of few rows takes longer to make than to run)."""
    fn = _PAGED.get(what)
    if fn is None:
        fn = _PAGED[what] = getattr(_lib.lib(), what)
    if index < 0:
        raise ValueError(f"{what}: expected tensors on a GPU")
    if index == torch._C._cuda_getDevice():
        st = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(index):
            st = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    if st:
        _check(st, what)


def _there(kept, *tensors):
    # whether tensors are where a cache's are (kept: its _c_pages)
    index = kept[3]
    if index >= 0:
        for t in tensors:
            if t.get_device() != index:
                return False
        return True
    return all(t.device == kept[4] for t in tensors)


class ResizeBuffers:
    """Preallocated outputs and workspace of page_resize (reusable): slots for `capacity` appended
    rows, and each list's first of them."""

    def __init__(self, cache: PagedCache, capacity: int, device):
        lists = cache.lists
        self.slots = torch.empty(int(capacity), dtype=torch.int32, device=device)
        self.slot_offsets = torch.empty(lists + 1, dtype=torch.int64, device=device)
        one = _lib.Problem(1, lists, 1, 1, 64, 1, None, _lib.CERTKV_BF16, _lib.CERTKV_BF16, 0.0, 0,
                           None)
        c = _lib.Pages(0, int(cache.page), cache.num_pages, cache.table.shape[1], 0, 0, 0, 1, 0,
                       None, None, None, None, cache.table.data_ptr(), cache.offsets.data_ptr(),
                       None, None)
        self.ws_bytes = int(_lib.lib().certkv_page_workspace_size(ctypes.byref(one),
                                                                  ctypes.byref(c)))
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)


def page_resize(spec: ProblemSpec, cache: PagedCache, change, bufs=None, into=None):
    """Block table and slots of a step: change [lists] int32, the rows that each list gains (> 0:
    pages come from the ring) or loses (< 0: its last ones; their pages go back).  Returns (slots
    int32, one for each appended row, lists one after another, slot_offsets [lists+1] int64).  The
    cache's offsets and free are updated in place, or, where `into` is two tensors like them, left
    as they are and the new ones written there.  A list that does not fit is refused: its slots are
    -1, it stays as it was, and spec.status says CERTKV_ERANGE.  bufs: ResizeBuffers (without, the
    rows to append are counted on the device first)."""
    kept = cache._c_pages(spec)
    lists = cache.lists
    assert change.dtype == torch.int32 and change.is_contiguous() and change.numel() == lists
    assert _there(kept, change) and cache.ring is not None and cache.free is not None
    if bufs is None:
        bufs = ResizeBuffers(cache, int(change.clamp(min=0).sum().item()), change.device)
    if into is None:
        offsets, free = cache.offsets, cache.free
    else:
        offsets, free = into
        assert offsets.dtype == torch.int64 and offsets.numel() == lists + 1
        assert free.dtype == torch.int64 and free.numel() == 2
        assert offsets.is_contiguous() and free.is_contiguous() and _there(kept, offsets, free)
    slots, slot_offsets = bufs.slots, bufs.slot_offsets
    assert slot_offsets.numel() == lists + 1 and _there(kept, slots)
    _run_paged(kept[3], "certkv_page_resize", _page_problem(spec), kept[2], change.data_ptr(),
               offsets.data_ptr(), free.data_ptr(), slots.data_ptr(), slots.numel(),
               slot_offsets.data_ptr(), bufs.ws.data_ptr(), bufs.ws_bytes)
    return slots, slot_offsets


def _check_slots(cache, kept, slots, slot_offsets):
    assert slots.dtype == torch.int32 and slots.is_contiguous()
    assert slot_offsets.dtype == torch.int64 and slot_offsets.is_contiguous()
    assert slot_offsets.numel() == cache.lists + 1 and _there(kept, slots, slot_offsets)


def page_write(spec: ProblemSpec, cache: PagedCache, k, v, slots, slot_offsets, tn=0):
    """Rows of new tokens to their slots (of page_resize): k, v [L][tokens][H][d] in spec.dtype,
    sequence after sequence, or, with tn, tn tokens of each sequence, of which a list takes as many
    as it has slots.  Slots that no token fills are reported (CERTKV_ERANGE)."""
    kept = cache._c_pages(spec)
    shape = k.shape
    assert shape == v.shape and len(shape) == 4 and cache.k is not None
    layers, tokens, heads, d = shape
    assert layers == spec.layers and heads == spec.kv_heads and d == spec.head_dim
    assert k.dtype == v.dtype == spec.dtype and _there(kept, k, v)
    _check_slots(cache, kept, slots, slot_offsets)
    _run_paged(kept[3], "certkv_page_write", _page_problem(spec), kept[2], _tensor(k), _tensor(v),
               tokens, int(tn), slots.data_ptr(), slots.numel(), slot_offsets.data_ptr())


def page_adopt(spec: ProblemSpec, cache: PagedCache, packed, slots, slot_offsets):
    """A packed cache's rows to the slots of lists (units') that take them whole: an MxCache, or
    (k_packed, v_packed, packed_offsets) of a bf16 one, of the pages' format."""
    kept = cache._c_pages(spec)
    assert cache.k is not None
    if isinstance(packed, MxCache):
        src, rows, d, k = packed.c_cache(), packed.rows, packed.head_dim, packed.k
        assert packed.format == cache.format
    else:
        k, v = packed[0], packed[1]
        assert k.is_contiguous() and v.is_contiguous() and k.shape == v.shape
        assert k.dtype == v.dtype == torch.bfloat16 and v.device == k.device
        assert cache.format == "bf16"
        rows, d = k.shape
        src = _lib.Cache(_lib.CERTKV_CACHE_BF16, k.data_ptr(), v.data_ptr(), None, None, None)
    assert d == spec.head_dim and _there(kept, k)
    _check_slots(cache, kept, slots, slot_offsets)
    _run_paged(kept[3], "certkv_page_adopt", _page_problem(spec), kept[2], src, rows,
               slots.data_ptr(), slots.numel(), slot_offsets.data_ptr())


def page_read(spec: ProblemSpec, cache: PagedCache, dtype=torch.bfloat16, rows=None, out=None):
    """The rows of all lists, out of their pages: (k, v) [L][rows][H][d], as compress takes them, or
    of units' lists [rows][d], a packed cache.  rows: their number (None: asked of the device);
    out: the two tensors to write, whose rows past the lists' last are left as they are."""
    kept = cache._c_pages(spec)
    assert cache.k is not None
    if out is None:
        n = int((cache.offsets[-1] - cache.offsets[0]).item()) if rows is None else int(rows)
        shape = (n, spec.head_dim) if cache.per_head else \
            (spec.layers, n, spec.kv_heads, spec.head_dim)
        out = [torch.empty(shape, dtype=dtype, device=kept[4]) for _ in range(2)]
    ko, vo = out
    n = ko.shape[0 if cache.per_head else 1]
    shape = (n, spec.head_dim) if cache.per_head else (spec.layers, n, spec.kv_heads, spec.head_dim)
    assert ko.shape == vo.shape == shape and ko.dtype == vo.dtype
    assert ko.is_contiguous() and vo.is_contiguous() and _there(kept, ko, vo)
    _run_paged(kept[3], "certkv_page_read", _page_problem(spec), kept[2], n, _dtype_code(ko.dtype),
               ko.data_ptr(), vo.data_ptr())
    return ko, vo


def decode_paged_workspace_size(spec: ProblemSpec, cache: PagedCache, tq: int,
                                max_rows: int = 0) -> int:
    return int(_lib.lib().certkv_decode_paged_workspace_size(
        _page_problem(spec), cache._c_pages(spec)[2], int(tq), int(max_rows)))


def decode_paged(spec: ProblemSpec, q_new, cache: PagedCache, tq, q_lens=None, with_lse=False,
                 bufs=None, max_rows=0):
    """decode over a paged cache, whose lists' last rows are the new tokens' own: query t of
    sequence b's n = q_lens[b] (int32 [B]; None: tq) sees the rows up to len - n + t (a chain: no
    mask over the new tokens, as decode_tree's).  Returns out
    [L][B*tq][Hq][d] fp32 (and the natural-log lse [L][B*tq][Hq] with_lse); a query that sees
    nothing (t >= n, an empty list) is out 0, lse -inf.  bufs: DecodeBuffers(..., pages=cache)."""
    kept = cache._c_pages(spec)
    _check_queries(spec, q_new, tq)
    assert cache.k is not None and _there(kept, q_new)
    if q_lens is not None:
        assert q_lens.dtype == torch.int32 and q_lens.is_contiguous()
        assert q_lens.shape == (spec.batch,) and _there(kept, q_lens)
    if bufs is None:
        bufs = DecodeBuffers(spec, tq, q_new.device, with_lse=with_lse, max_rows=max_rows,
                             pages=cache)
    out, lse = bufs.out, bufs.lse
    assert bufs.paged and bufs.tq == tq and out.shape == q_new.shape and _there(kept, out)
    assert lse is not None or not with_lse
    _run_paged(kept[3], "certkv_decode_paged", _page_problem(spec), _tensor(q_new), bufs.tq,
               None if q_lens is None else q_lens.data_ptr(), bufs.max_rows, kept[2],
               out.data_ptr(), None if lse is None else lse.data_ptr(), bufs.ws.data_ptr(),
               bufs.ws_bytes)
    return (out, lse) if with_lse else out


class CompressBuffers:
    """Preallocated outputs and workspace of the fused pass (reusable); with fmt
    ("mxfp8" or "mxfp4") the packed cache is an MxCache, `mx`, in place of
    k_packed and v_packed, and shares pos_packed and packed_offsets."""

    def __init__(self, spec: ProblemSpec, n_keep, device, with_curves=False, with_perm=False,
                 with_mask=False, with_lse=False, fmt=None):
        self.spec = spec
        self.n_keep = [int(x) for x in n_keep]
        H, D = spec.kv_heads, spec.head_dim
        U = spec.units
        slot = 1 if spec.slot else 0
        kept = spec.layers * sum(H * nk - slot * H for nk in self.n_keep)
        rows = kept + slot * U
        self.rows = rows
        shape = (spec.layers, H, spec.total_tokens)
        dt = spec.dtype
        self.scores = torch.empty(shape, dtype=torch.float32, device=device)
        self.budgets = torch.empty(U, dtype=torch.int32, device=device)
        self.kept_offsets = torch.empty(U + 1, dtype=torch.int64, device=device)
        self.kept_idx = torch.empty(max(kept, 1), dtype=torch.int32, device=device)
        self.k_star = torch.empty((U, D), dtype=torch.float32, device=device)
        self.v_star = torch.empty((U, D), dtype=torch.float32, device=device)
        self.tail_mass = torch.empty(U, dtype=torch.float64, device=device)
        self.mx = MxCache.empty(spec, rows, fmt, device) if fmt is not None else None
        if self.mx is None:
            self.k_packed = torch.empty((rows, D), dtype=dt, device=device)
            self.v_packed = torch.empty((rows, D), dtype=dt, device=device)
            self.pos_packed = torch.empty(rows, dtype=torch.int32, device=device)
            self.packed_offsets = torch.empty(U + 1, dtype=torch.int64, device=device)
        else:
            self.k_packed = self.v_packed = None
            self.pos_packed, self.packed_offsets = self.mx.pos, self.mx.offsets
        self.curves = torch.empty(shape, dtype=torch.float32, device=device) if with_curves else None
        self.perm = torch.empty(shape, dtype=torch.int32, device=device) if with_perm else None
        self.alloc_stats = torch.zeros((spec.layers * spec.batch, 3), dtype=torch.int64,
                                       device=device)
        self.kept_mask = torch.empty(shape, dtype=torch.uint8, device=device) if with_mask else None
        self.lse = torch.empty(_lse_shape(spec), dtype=torch.float32, device=device) \
            if with_lse else None
        self.ws, self.ws_bytes = _workspace(spec, _lib.STAGE_COMPRESS, device)
        self._nk = (ctypes.c_int32 * spec.batch)(*self.n_keep)
        self._p = spec.c_problem()
        self._out = _lib.Outputs(*[
            (t.data_ptr() if t is not None else None) for t in (
                self.scores, self.budgets, self.kept_offsets, self.kept_idx, self.k_star,
                self.v_star, self.tail_mass, self.k_packed, self.v_packed, self.pos_packed,
                self.packed_offsets, self.curves, self.perm, self.alloc_stats, self.kept_mask,
                self.lse)])

    def as_dict(self):
        return {k: getattr(self, k) for k in (
            "scores", "budgets", "kept_offsets", "kept_idx", "k_star", "v_star", "tail_mass",
            "k_packed", "v_packed", "pos_packed", "packed_offsets", "curves", "perm",
            "alloc_stats", "kept_mask", "lse")}


def compress(spec: ProblemSpec, q_win, k, v, n_keep, alpha=0.2, steps=40, bufs=None,
             with_curves=False, with_perm=False, with_mask=False, with_lse=False, lse_in=None,
             fmt=None):
    """The whole pass; returns the CompressBuffers holding every output.  fmt ("mxfp8" or
    "mxfp4"): the packed cache in microscaled codes (bufs.mx)."""
    L = _lib.lib()
    dev = k.device
    if bufs is None:
        bufs = CompressBuffers(spec, n_keep, dev, with_curves=with_curves, with_perm=with_perm,
                               with_mask=with_mask, with_lse=with_lse, fmt=fmt)
    if lse_in is not None:
        assert lse_in.dtype == torch.float32 and lse_in.is_contiguous()
        assert tuple(lse_in.shape) == _lse_shape(spec)
    if fmt is not None:
        assert bufs.mx is not None and bufs.mx.format == fmt
    if bufs.mx is not None:
        assert bufs.mx.rows >= bufs.rows and bufs.mx.head_dim == spec.head_dim
        c = bufs.mx.c_cache()
        _run(dev, "certkv_compress_mx", ctypes.byref(bufs._p), c.format, _tensor(q_win),
             _tensor(k), _tensor(v), _ptr(lse_in), bufs._nk, float(alpha), int(steps),
             ctypes.byref(bufs._out), c.k, c.k_scales, c.v, c.v_scales, _ptr(bufs.ws),
             bufs.ws_bytes)
        return bufs
    _check(L.certkv_compress(ctypes.byref(bufs._p), _tensor(q_win), _tensor(k), _tensor(v),
                             _ptr(lse_in), bufs._nk, float(alpha), int(steps),
                             ctypes.byref(bufs._out), _ptr(bufs.ws), bufs.ws_bytes, _stream(dev)),
           "certkv_compress")
    return bufs


def profile_enable(on=True):
    _lib.lib().certkv_profile_enable(1 if on else 0)


def profile_reset():
    _lib.lib().certkv_profile_reset()


def profile_read(max_entries=64):
    """{kernel name: (launch count, total ms)} of the launches recorded so far."""
    names = (ctypes.c_char * 64 * max_entries)()
    counts = (ctypes.c_int64 * max_entries)()
    ms = (ctypes.c_double * max_entries)()
    k = _lib.lib().certkv_profile_read(names, counts, ms, max_entries)
    return {names[i].value.decode(): (int(counts[i]), float(ms[i])) for i in range(min(k, max_entries))}
