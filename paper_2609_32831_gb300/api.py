"""Python binding of the UniCache C ABI (same names, minus the ``uc_`` prefix).

Torch supplies device memory and the current stream; every computation runs
in the CUDA library. Each function marshals its arguments and calls one C
entry point; nothing here computes any part of the method.
"""
from __future__ import annotations

import ctypes as C
import struct
from functools import partial
from typing import List, Optional, Sequence, Tuple

import torch

from . import _lib
from ._lib import (GROUP, HEAD_DIM, KIND_EVICT, KIND_EVICT_QUANT, KIND_FULL, KIND_QUANT,
                   MAX_BATCH, MAX_SEGMENTS, POLICY_EVICT, POLICY_PROTECTED, POLICY_QUANT,
                   UcSegment, UcSegmentSizes, UcSegmentTable, UniCacheError, check, lib)

KIND_NAMES = {"full": KIND_FULL, "evict": KIND_EVICT, "quant": KIND_QUANT, "evict_quant": KIND_EVICT_QUANT}


_raw_stream = None   # torch's handle lookup without a Stream object, once CUDA is initialised


def _stream(stream=None) -> int:
    """The cudaStream_t of ``stream``, else of the current device's current stream."""
    global _raw_stream
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        handle = torch.cuda.current_stream().cuda_stream
        _raw_stream = torch._C._cuda_getCurrentRawStream
        return handle
    return _raw_stream(torch._C._cuda_getDevice())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _capturing(stream=None) -> bool:
    """Whether what is launched on ``stream`` (the current one if None) goes into a graph."""
    if stream is None:
        return torch.cuda.is_current_stream_capturing()
    with torch.cuda.stream(stream):
        return torch.cuda.is_current_stream_capturing()


_STATUS_BYTES = 16   # of a workspace's first bytes (see uc_workspace_status)


class Workspace:
    """Zero-filled device scratch, grown on demand and reused across calls.

    ``uc_attend`` and ``uc_attend_batch`` keep self-resetting counters
    in their workspaces, so each gets a buffer of its own ("attend",
    "attend_batch"); every other entry point shares the "scratch" buffer. Calls
    that may run at the same time, on two streams or in two graphs, need a Workspace
    each, or, on streams, one that keeps its buffers ``per_stream``. A buffer that a graph's
    launches work in stays as long as the Workspace does."""

    def __init__(self, device=None, per_stream: bool = False):
        self.device = torch.device(device or "cuda")
        self.per_stream = per_stream   # then the streams other than the default one have buffers (kind, handle)
        self.bufs = {}
        self._at = {}     # (kind, stream handle) -> (address, bytes), for the streams that have worked in the buffer
        self._kept = []   # buffers replaced during a graph's capture, for their status words
        self._graphs = {}  # address -> buffer, of captured launches: replays use them whatever the next calls need

    def get(self, nbytes: int, kind: str = "scratch", stream=None, handle: Optional[int] = None) -> Tuple[int, int]:
        """(address, bytes) of a buffer of at least ``nbytes`` for a launch on
        ``stream`` (the current one if None; its handle, where the caller has it)."""
        if handle is None and self.device.type == "cuda":
            handle = _stream(stream)
        in_graph = bool(handle) and _capturing(stream)   # (the default stream, 0, is in no capture)
        at = self._at.get((kind, handle))
        if at is not None and at[1] >= nbytes and not in_graph:
            return at
        nbytes = max(256, int(nbytes))
        key = self._key(kind, handle, nbytes, in_graph) if self.per_stream and handle else kind
        buf = self.bufs.get(key)
        if buf is None or buf.numel() < nbytes:
            buf = self._grow(buf, nbytes, key, stream)
        elif self.device.type == "cuda":
            self._record(buf, stream)
        at = buf.data_ptr(), buf.numel()
        if in_graph:
            self._graphs[at[0]] = buf
        else:
            self._at[kind, handle] = at
        return at

    def _key(self, kind: str, handle: int, nbytes: int, in_graph: bool):
        """Under capture a buffer that is large enough already, whichever stream it is of, the default
        one's first: a new one would lie in the graph's memory, and be cleared by every replay."""
        if not in_graph:
            return kind, handle
        keys = [kind, *(k for k in self.bufs if k[0] == kind)]
        return next((k for k in keys if k in self.bufs and self.bufs[k].numel() >= nbytes), kind)

    @staticmethod
    def _record(buf: torch.Tensor, stream) -> None:
        """The allocator gives ``buf`` to nobody else before ``stream`` is done with it."""
        buf.record_stream(stream or torch.cuda.current_stream())

    def _grow(self, old: Optional[torch.Tensor], nbytes: int, key, stream) -> torch.Tensor:
        """A larger buffer, cleared on the launch's own stream (a fill on another
        one could run beside the launch); it takes the status word over."""
        if self.device.type != "cuda":
            buf = torch.zeros(nbytes, dtype=torch.uint8, device=self.device)
            if old is not None:
                buf[:_STATUS_BYTES] = old[:_STATUS_BYTES]
        else:
            if old is not None:
                self._record(old, stream)
            with torch.cuda.stream(stream):
                buf = torch.zeros(nbytes, dtype=torch.uint8, device=self.device)
                if old is not None:
                    if _capturing():
                        self._kept.append(old)   # (a captured copy would read it at every replay)
                    else:
                        buf[:_STATUS_BYTES].copy_(old[:_STATUS_BYTES])
        kind = key if isinstance(key, str) else key[0]
        self._at = {k: at for k, at in self._at.items() if k[0] != kind}
        self.bufs[key] = buf
        return buf

    def status(self, stream=None) -> int:
        """Synchronise and read (then clear) the device status words."""
        code = 0
        if self.per_stream and self.device.type == "cuda":
            torch.cuda.synchronize(self.device)   # (buffers of any stream)
        for buf in {b.data_ptr(): b for b in [*self.bufs.values(), *self._kept, *self._graphs.values()]}.values():
            c = lib().uc_workspace_status(C.c_void_p(buf.data_ptr()), _stream(stream))
            code = code or c
        self._kept.clear()
        return code


_default_ws = {}


def default_workspace(device) -> Workspace:
    """What calls that are given no workspace use: buffers for each stream, so that calls on several
    streams may run at the same time. (Graphs captured with it share buffers, with one another
    and with calls that are not captured.)"""
    key = torch.device(device).index or 0
    if key not in _default_ws:
        _default_ws[key] = Workspace(device, per_stream=True)
    return _default_ws[key]


class Segment:
    """One cache type of one layer for B sequences and Hkv KV heads, with its
    storage in torch device tensors (see ``uc_segment`` in unicache.h)."""

    def __init__(self, kind, bits: int, batch: int, n_kv_heads: int, n_src: int, cap: int,
                 device="cuda", label: int = 0):
        kind = KIND_NAMES.get(kind, kind)
        if kind == KIND_FULL:
            raise ValueError("use Segment.view() for full-precision segments")
        if kind in (KIND_QUANT, KIND_EVICT_QUANT):
            cap = (cap + 63) // 64 * 64
        else:
            bits = 16
        self.device = torch.device(device)
        c = UcSegment()
        c.kind, c.bits, c.batch, c.n_kv_heads = kind, bits, batch, n_kv_heads
        c.head_dim, c.n_src, c.cap, c.label = HEAD_DIM, n_src, cap, label
        sz = UcSegmentSizes()
        check("uc_segment_sizes_of", lib().uc_segment_sizes_of(C.byref(c), C.byref(sz)))
        self._t = {}

        def alloc(name, nbytes, dtype=torch.uint8):
            if nbytes == 0:
                return None
            el = torch.tensor([], dtype=dtype).element_size()
            t = torch.zeros(int(nbytes) // el, dtype=dtype, device=self.device)
            self._t[name] = t
            return t.data_ptr()

        c.n_kept = alloc("n_kept", sz.n_kept, torch.int32)
        c.kept_idx = alloc("kept_idx", sz.kept_idx, torch.int32)
        c.k = alloc("k", sz.k, torch.bfloat16)
        c.v = alloc("v", sz.v, torch.bfloat16)
        c.k_codes = alloc("k_codes", sz.k_codes)
        c.k_params = alloc("k_params", sz.k_params)
        c.v_codes = alloc("v_codes", sz.v_codes)
        c.v_params = alloc("v_params", sz.v_params)
        nbh = batch * n_kv_heads
        if kind in (KIND_QUANT, KIND_EVICT_QUANT):
            c.row_stride, c.row_offset, c.rows_total = GROUP, 0, nbh * GROUP
        else:
            c.row_stride, c.row_offset, c.rows_total = cap, 0, nbh * cap
        self.c = c

    @classmethod
    def view(cls, k: torch.Tensor, v: torch.Tensor, begin: int, n: int, label: int = 0) -> "Segment":
        """A full-precision segment over tokens [begin, begin + n) of caller
        tensors k, v [B, Hkv, N, 128] (bf16, contiguous). Borrowed, not copied."""
        assert k.dtype == torch.bfloat16 and k.is_contiguous() and v.is_contiguous()
        B, hkv, N, d = k.shape
        self = cls.__new__(cls)
        self.device = k.device
        c = UcSegment()
        c.kind, c.bits, c.batch, c.n_kv_heads = KIND_FULL, 16, B, hkv
        c.head_dim, c.n_src, c.cap, c.label = d, n, n, label
        for b in range(B):
            c.n_kept_host[b] = n
        nk = torch.full((B,), n, dtype=torch.int32, device=k.device)
        self._t = {"n_kept": nk, "k": k, "v": v}
        c.n_kept = nk.data_ptr()
        c.kept_idx = None
        c.k, c.v = k.data_ptr(), v.data_ptr()
        c.row_stride, c.row_offset, c.rows_total = N, begin, B * hkv * N
        self.c = c
        return self

    # -------------------------------------------------------------- views
    @property
    def kind(self) -> int:
        return self.c.kind

    @property
    def bits(self) -> int:
        return self.c.bits

    @property
    def batch(self) -> int:
        return self.c.batch

    @property
    def n_kv_heads(self) -> int:
        return self.c.n_kv_heads

    @property
    def cap(self) -> int:
        return self.c.cap

    def n_kept(self) -> List[int]:
        return [int(self.c.n_kept_host[b]) for b in range(self.c.batch)]

    def sync_host(self) -> None:
        """Copy the device kept counts into the host mirror (after appends
        that only advance the device counts, e.g. replayed graphs)."""
        counts = self._t["n_kept"].cpu().tolist()
        for b, n in enumerate(counts):
            self.c.n_kept_host[b] = int(n)

    def set_keep(self, keep: Sequence[int]) -> None:
        """Number of tokens to keep per sequence (before compress_segment)."""
        for b in range(self.c.batch):
            self.c.n_kept_host[b] = int(keep[b] if hasattr(keep, "__len__") else keep)

    def tensor(self, name: str) -> Optional[torch.Tensor]:
        return self._t.get(name)

    def stored_bytes(self, with_index: bool = False) -> int:
        """Bytes the stored tokens occupy in the packed layout (K + V)."""
        tot = 0
        for n in self.n_kept():
            per_head = 0
            if self.c.bits == 16:
                per_head = n * 4 * HEAD_DIM
            else:
                ng = n // GROUP
                per_head = (2 * GROUP * ng * HEAD_DIM * self.c.bits // 8 + ng * HEAD_DIM * 4 +
                            GROUP * ng * 16 + (n - GROUP * ng) * 4 * HEAD_DIM)
            if with_index and self.c.kind != KIND_FULL:
                per_head += 4 * n
            tot += per_head * self.c.n_kv_heads
        return tot


# ---------------------------------------------------------------- host policy

def concentration(mass, top_frac: float = 0.1) -> float:
    import numpy as np
    m = np.ascontiguousarray(mass, dtype=np.float32)
    out = C.c_double()
    check("uc_concentration", lib().uc_concentration(
        m.ctypes.data_as(C.c_void_p), m.size, top_frac, C.byref(out)))
    return out.value


class SegmentTable:
    """uc_segment_table: per-type candidates, sizes, policies and budgets."""

    def __init__(self, n_tokens: Sequence[int], candidate: Sequence[bool]):
        t = UcSegmentTable()
        t.n_types = len(n_tokens)
        for a, (n, c) in enumerate(zip(n_tokens, candidate)):
            t.n_tokens[a] = int(n)
            t.candidate[a] = 1 if c else 0
            t.policy[a] = POLICY_PROTECTED if not c else POLICY_EVICT
        self.c = t

    def field(self, name):
        arr = getattr(self.c, name)
        return [arr[a] for a in range(self.c.n_types)]


def calibrate_policy(table: SegmentTable, mass_vectors, top_frac: float = 0.1,
                     threshold: float = 0.5) -> None:
    """mass_vectors[e][a]: per-token mass (host array) of type a in example e."""
    import numpy as np
    n_ex = len(mass_vectors)
    nt = table.c.n_types
    keep_alive = []
    ptrs = (C.c_void_p * (n_ex * nt))()
    for e in range(n_ex):
        for a in range(nt):
            m = np.ascontiguousarray(mass_vectors[e][a], dtype=np.float32)
            if m.size != table.c.n_tokens[a]:
                raise ValueError(f"example {e} type {a}: {m.size} != {table.c.n_tokens[a]}")
            keep_alive.append(m)
            ptrs[e * nt + a] = m.ctypes.data_as(C.c_void_p)
    check("uc_calibrate_policy", lib().uc_calibrate_policy(
        C.byref(table.c), C.cast(ptrs, C.c_void_p), n_ex, top_frac, threshold))


def allocate_budget(table: SegmentTable, rho: float, first_chunk: bool = True) -> None:
    """Eq. 2 with B = rho * sum_a S_a; previous budgets are table.budget (or S
    on the first chunk). Fills table budget / keep / bits / kind."""
    check("uc_allocate_budget", lib().uc_allocate_budget(C.byref(table.c), float(rho), int(first_chunk)))


def retention_schedule(rho_prev, rho_init, rho_min, m_c, m_0) -> float:
    out = C.c_double()
    check("uc_retention_schedule", lib().uc_retention_schedule(
        float(rho_prev), float(rho_init), float(rho_min), float(m_c), float(m_0), C.byref(out)))
    return out.value


def retention_step(table: "SegmentTable", first_chunk: bool, rho_prev: float, rho_init: float, rho_min: float,
                   m_0: float = 0.0):
    """Eq. 3 for one (sequence, layer chunk) with M^(c) formed from the
    table's candidate masses; returns (rho, m_0) (see unicache.h)."""
    m0 = C.c_double(m_0)
    rho = C.c_double()
    check("uc_retention_step", lib().uc_retention_step(C.byref(table.c), int(first_chunk), float(rho_prev),
                                                       float(rho_init), float(rho_min), C.byref(m0),
                                                       C.byref(rho)))
    return rho.value, m0.value


def plan_batch(tables, type_index: int):
    """One segment configuration of type ``type_index`` for a batch of
    per-sequence tables (after allocate_budget): returns (kind, bits,
    full_view, keep list)."""
    from ._lib import UcTypeConfig
    n = len(tables)
    arr = (UcSegmentTable * n)(*[t.c for t in tables])
    keep = (C.c_int32 * n)()
    cfg = UcTypeConfig()
    check("uc_plan_batch", lib().uc_plan_batch(arr, n, int(type_index), keep, C.byref(cfg)))
    return int(cfg.kind), int(cfg.bits), bool(cfg.full_view), [int(x) for x in keep]


def keep_count(n: int, keep_frac: float) -> int:
    """Tokens a fixed keep fraction retains (see unicache.h)."""
    out = C.c_int32()
    check("uc_keep_count", lib().uc_keep_count(int(n), float(keep_frac), C.byref(out)))
    return int(out.value)


# ---------------------------------------------------------------- device calls

def score_accumulate(qwin: torch.Tensor, k: torch.Tensor, n_ctx: Optional[int] = None,
                     out: Optional[torch.Tensor] = None, ws: Optional[Workspace] = None,
                     stream=None) -> torch.Tensor:
    """qwin [B, Hq, W, 128], k [B, Hkv, N, 128] (bf16) -> scores [B, Hkv, n_ctx] fp32."""
    B, hq, W, d = qwin.shape
    _, hkv, N, _ = k.shape
    n_ctx = N if n_ctx is None else n_ctx
    if out is None:
        out = torch.empty((B, hkv, n_ctx), dtype=torch.float32, device=k.device)
    ws = ws or default_workspace(k.device)
    need = lib().uc_score_workspace_size(B, hq, hkv, W, n_ctx)
    wp, wn = ws.get(need, stream=stream)
    check("uc_score_accumulate", lib().uc_score_accumulate(
        _ptr(qwin), _ptr(k), B, hq, hkv, W, n_ctx, N, _ptr(out), wp, wn, _stream(stream)))
    return out


def segment_mass(scores: torch.Tensor, ranges: Sequence[Tuple[int, int]], n_q_heads: int,
                 window: int, out: Optional[torch.Tensor] = None, weight: float = 1.0,
                 accumulate: bool = False, stream=None) -> torch.Tensor:
    """Eq. 1 term per (sequence, type) from observation scores -> [B, n_seg]
    fp32; with accumulate=True adds weight * term into ``out``."""
    B, hkv, n_ctx = scores.shape
    ns = len(ranges)
    if out is None:
        out = torch.zeros((B, ns), dtype=torch.float32, device=scores.device)
    beg = (C.c_int32 * ns)(*[r[0] for r in ranges])
    end = (C.c_int32 * ns)(*[r[1] for r in ranges])
    check("uc_segment_mass", lib().uc_segment_mass(
        _ptr(scores), B, hkv, n_ctx, C.cast(beg, C.c_void_p), C.cast(end, C.c_void_p), ns,
        n_q_heads, window, float(weight), int(accumulate), _ptr(out), _stream(stream)))
    return out


def compress_segment(k_src: torch.Tensor, v_src: torch.Tensor, seg: Segment, begin: int = 0,
                     scores: Optional[torch.Tensor] = None, scores_begin: Optional[int] = None,
                     n_recent: int = 0, ws: Optional[Workspace] = None, stream=None) -> Segment:
    """Compress tokens [begin, begin + n_src) of k_src, v_src [B, Hkv, N, 128]
    into ``seg`` (keep counts set with ``seg.set_keep``). scores [B, Hkv, Ns]."""
    B, hkv, N, d = k_src.shape
    ws = ws or default_workspace(k_src.device)
    wp, wn = ws.get(lib().uc_compress_workspace_size(C.byref(seg.c)), stream=stream)
    s_stride = scores.shape[-1] if scores is not None else 0
    s_off = (begin if scores_begin is None else scores_begin) if scores is not None else 0
    check("uc_compress_segment", lib().uc_compress_segment(
        _ptr(k_src), _ptr(v_src), N, begin, _ptr(scores), s_stride, s_off, n_recent,
        C.byref(seg.c), wp, wn, _stream(stream)))
    return seg


class _CudaArray:
    """Device memory described by __cuda_array_interface__ (a view for torch)."""

    def __init__(self, iface):
        self.__cuda_array_interface__ = iface


class OwnedSegment(Segment):
    """A segment whose storage the library allocated (uc_compress_budget);
    its storage goes back to the allocator with uc_segment_free when this
    object is released (or on free())."""

    def __init__(self, ptr, device, keepalive=()):
        self._ptr = ptr
        self.c = ptr.contents
        self.device = torch.device(device)
        self._t = {}
        self._keep = keepalive   # the source rows a full view reads, the allocator's callbacks

    def sync_host(self) -> None:
        counts = self.tensor("n_kept").cpu().tolist()
        for b, n in enumerate(counts):
            self.c.n_kept_host[b] = int(n)

    def tensor(self, name: str) -> Optional[torch.Tensor]:
        """A view (no copy) of one of the segment's device arrays; valid while
        the segment lives."""
        if not self._ptr:
            return None
        sz = UcSegmentSizes()
        check("uc_segment_sizes_of", lib().uc_segment_sizes_of(C.byref(self.c), C.byref(sz)))
        dtypes = {"n_kept": ("<i4", 4), "kept_idx": ("<i4", 4), "k": ("<u2", 2), "v": ("<u2", 2),
                  "k_codes": ("|u1", 1), "k_params": ("|u1", 1), "v_codes": ("|u1", 1), "v_params": ("|u1", 1)}
        ptr = getattr(self.c, name)
        if name not in dtypes or not ptr:
            return None
        typestr, el = dtypes[name]
        nbytes = int(getattr(sz, name))
        if self.c.kind == KIND_FULL and name in ("k", "v"):
            nbytes = int(self.c.rows_total) * HEAD_DIM * 2
        iface = {"shape": (nbytes // el,), "typestr": typestr, "data": (int(ptr), False), "version": 3,
                 "strides": None}
        t = torch.as_tensor(_CudaArray(iface), device=self.device)
        return t.view(torch.bfloat16) if name in ("k", "v") else t

    def free(self) -> None:
        """Return the storage (uc_segment_free). The structure the library
        handed out goes with it, so this object keeps an empty one: a call
        that is given a freed segment fails its argument checks."""
        if self._ptr:
            self.c = UcSegment()
            lib().uc_segment_free(C.cast(self._ptr, C.c_void_p))
            self._ptr = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def compress_budget(k_src: torch.Tensor, v_src: torch.Tensor, tables, type_index: int, begin: int = 0,
                    scores: Optional[torch.Tensor] = None, scores_begin: Optional[int] = None,
                    n_recent: int = 0, allocator: Optional["_lib.UcAllocator"] = None,
                    stream=None) -> OwnedSegment:
    """The budget form of compression: type ``type_index`` of k_src, v_src
    [B, Hkv, N, 128] (tokens [begin, begin + n)) compressed as the
    per-sequence tables (after allocate_budget) configure it, into storage
    the library allocates (through ``allocator``, else cudaMallocAsync)."""
    B, hkv, N, d = k_src.shape
    n = int(tables[0].c.n_tokens[type_index])
    arr = (UcSegmentTable * len(tables))(*[t.c for t in tables])
    s_stride = scores.shape[-1] if scores is not None else 0
    s_off = (begin if scores_begin is None else scores_begin) if scores is not None else 0
    out = C.POINTER(UcSegment)()
    check("uc_compress_budget", lib().uc_compress_budget(
        _ptr(k_src), _ptr(v_src), B, hkv, n, N, begin, _ptr(scores), s_stride, s_off, n_recent,
        arr, int(type_index), None if allocator is None else C.byref(allocator), _stream(stream),
        C.byref(out)))
    keep = (k_src, v_src, allocator) if out.contents.kind == KIND_FULL else (allocator,)
    return OwnedSegment(out, k_src.device, keep)


def recompress_segment(src: Segment, dst: Segment, scores: Optional[torch.Tensor] = None,
                       scores_begin: int = 0, n_recent: int = 0, ws: Optional[Workspace] = None,
                       stream=None) -> Segment:
    """Compress the tokens ``src`` still holds further into ``dst`` (keep counts
    set with ``dst.set_keep``). scores [B, Hkv, Ns] fp32 indexed by logical
    token (position scores_begin + token index), needed when dst evicts."""
    ws = ws or default_workspace(src.device)
    wp, wn = ws.get(lib().uc_recompress_workspace_size(C.byref(src.c), C.byref(dst.c)), stream=stream)
    s_stride = scores.shape[-1] if scores is not None else 0
    check("uc_recompress_segment", lib().uc_recompress_segment(
        C.byref(src.c), _ptr(scores), s_stride, scores_begin, n_recent, C.byref(dst.c), wp, wn,
        _stream(stream)))
    return dst


def accumulate_scores(q: torch.Tensor, seg: Segment, lse: torch.Tensor, acc: torch.Tensor, acc_begin: int = 0,
                      ws: Optional[Workspace] = None, stream=None) -> torch.Tensor:
    """Add one decode call's probabilities on the stored tokens of the bf16
    segment ``seg`` into ``acc`` [B, Hkv, N] fp32 at logical index
    acc_begin + token (lse: that call's [B, Hq, T] output)."""
    B, hq, T, d = q.shape
    ws = ws or default_workspace(q.device)
    st = _stream(stream)
    wp, wn = ws.get(256, "scratch", stream, st)
    check("uc_accumulate_scores", lib().uc_accumulate_scores(
        _ptr(q), hq, T, C.byref(seg.c), _ptr(lse), _ptr(acc), acc.shape[-1], acc_begin, wp, wn,
        st))
    return acc


def attention_mass(mass: torch.Tensor, out: Optional[torch.Tensor] = None, weight: float = 1.0,
                   accumulate: bool = False, stream=None) -> torch.Tensor:
    """Eq. 1 term per (sequence, segment) from attend's mass [B, Hq, T, n_seg]
    -> [B, n_seg] fp32; with accumulate=True adds weight * term into ``out``."""
    B, hq, T, ns = mass.shape
    if out is None:
        out = torch.zeros((B, ns), dtype=torch.float32, device=mass.device)
    check("uc_attention_mass", lib().uc_attention_mass(
        _ptr(mass), B, hq, T, ns, float(weight), int(accumulate), _ptr(out), _stream(stream)))
    return out


def _seg_array(segs: Sequence[Segment]):
    """A C array of the segments' addresses (valid while ``segs`` are)."""
    return (C.c_void_p * len(segs))(*[C.addressof(s.c) for s in segs])


def attend(q: torch.Tensor, segs: Sequence[Segment], out: Optional[torch.Tensor] = None,
           lse: Optional[torch.Tensor] = None, mass: Optional[torch.Tensor] = None,
           want_lse: bool = True, want_mass: bool = True, ws: Optional[Workspace] = None,
           stream=None):
    """q [B, Hq, T, 128] bf16 -> (O bf16 [B, Hq, T, 128], lse fp32 [B, Hq, T],
    mass fp32 [B, Hq, T, n_seg])."""
    B, hq, T, d = q.shape
    ns = len(segs)
    arr = _seg_array(segs)
    if out is None:
        out = torch.empty_like(q)
    if want_lse and lse is None:
        lse = torch.empty((B, hq, T), dtype=torch.float32, device=q.device)
    if want_mass and mass is None:
        mass = torch.empty((B, hq, T, ns), dtype=torch.float32, device=q.device)
    ws = ws or default_workspace(q.device)
    L = lib()
    # the call plans once and says if the workspace at hand is too small for
    # it (nothing is launched then): only then is the size asked for
    st = _stream(stream)
    wp, wn = ws.get(0 if "attend" in ws.bufs else L.uc_attend_workspace_size(arr, ns, hq, T), "attend", stream, st)
    args = (q.data_ptr(), hq, T, arr, ns, out.data_ptr(), _ptr(lse), _ptr(mass))
    code = L.uc_attend(*args, wp, wn, st)
    if code == _lib.UC_ERR_OOM:
        wp, wn = ws.get(L.uc_attend_workspace_size(arr, ns, hq, T), "attend", stream, st)
        code = L.uc_attend(*args, wp, wn, st)
    check("uc_attend", code)
    return out, lse, mass


def attend_plan(segs, n_q_heads: int, n_qtok: int, slots: int = 0) -> dict:
    """How ``attend`` splits a decode-shaped call into work items and what it
    launches (cluster, ctas, stages, merge_width), for ``slots`` resident CTAs
    (0: this device's occupancy). Host only when slots > 0. ``segs``: Segment
    objects or raw UcSegment structures."""
    from ._lib import UcAttendLaunchInfo, UcAttendPlanInfo
    raw = [s.c if hasattr(s, "c") else s for s in segs]
    sp = (C.POINTER(UcSegment) * len(raw))(*[C.pointer(r) for r in raw])
    info = UcAttendPlanInfo()
    check("uc_attend_plan", lib().uc_attend_plan(C.cast(sp, C.c_void_p), len(raw), n_q_heads, n_qtok, slots,
                                                 C.byref(info)))
    run = UcAttendLaunchInfo()
    check("uc_attend_launch", lib().uc_attend_launch(C.cast(sp, C.c_void_p), len(raw), n_q_heads, n_qtok, slots,
                                                     C.byref(run)))
    n = len(raw)
    return {"items_per_bh": info.items_per_bh, "n_heavy": info.n_heavy, "n_light": info.n_light,
            "grid": info.grid, "merge_kernel": bool(info.merge_kernel),
            "n_chunks": list(info.n_chunks)[:n], "light": [bool(x) for x in list(info.light)[:n]],
            "cluster": run.cluster, "ctas": run.ctas, "stages": run.stages, "merge_width": run.merge_width}


def attend_batch(calls, ws: Optional[Workspace] = None, stream=None):
    """Several decode-shaped attention calls in one launch. ``calls``: a list
    of (q, segs) or (q, segs, out, lse, mass) with q [B, Hq, T, 128] bf16
    (T <= 8; every call the same number of 8-row query tiles). Returns the
    list of (O, lse, mass) per call."""
    n = len(calls)
    given = [(list(call[2:5]) + [None, None, None])[:3] for call in calls]
    shapes = [(B, hq, T, len(call[1])) for call in calls for B, hq, T, _ in [call[0].shape]]
    dev = calls[0][0].device if n else None   # (an empty batch with a workspace is the library's to refuse)
    if n > 1 and all(g[1] is None and g[2] is None for g in given) and all(x == shapes[0] for x in shapes) \
            and all(call[0].device == dev for call in calls):
        # one allocation each for the calls' lse and masses
        B, hq, T, ns = shapes[0]
        lses = torch.empty((n, B, hq, T), dtype=torch.float32, device=dev).unbind(0)
        masses = torch.empty((n, B, hq, T, ns), dtype=torch.float32, device=dev).unbind(0)
        given = [(g[0], lses[i], masses[i]) for i, g in enumerate(given)]
    keep, results, structs = [], [], []
    for call, (out, lse, mass), (B, hq, T, ns) in zip(calls, given, shapes):
        q, segs = call[0], call[1]
        if out is None:
            out = torch.empty_like(q)
        if lse is None:
            lse = torch.empty((B, hq, T), dtype=torch.float32, device=q.device)
        if mass is None:
            mass = torch.empty((B, hq, T, ns), dtype=torch.float32, device=q.device)
        sp = _seg_array(segs)
        keep.append(sp)
        structs.append(_lib.UcAttendCall(q.data_ptr(), hq, T, C.addressof(sp), ns, out.data_ptr(), lse.data_ptr(),
                                         mass.data_ptr()))
        results.append((out, lse, mass))
    arr = (_lib.UcAttendCall * n)(*structs)
    ws = ws or default_workspace(calls[0][0].device)
    L = lib()
    # as in attend(): the size is asked for only when the call needs more
    st = _stream(stream)
    wp, wn = ws.get(0 if "attend_batch" in ws.bufs else L.uc_attend_batch_workspace_size(arr, n), "attend_batch", stream,
                    st)
    code = L.uc_attend_batch(arr, n, wp, wn, st)
    if code == _lib.UC_ERR_OOM:
        wp, wn = ws.get(L.uc_attend_batch_workspace_size(arr, n), "attend_batch", stream, st)
        code = L.uc_attend_batch(arr, n, wp, wn, st)
    check("uc_attend_batch", code)
    return results


def attend_workspace_size(segs: Sequence[Segment], n_q_heads: int, n_qtok: int) -> int:
    return int(lib().uc_attend_workspace_size(_seg_array(segs), len(segs), n_q_heads, n_qtok))


def append(seg: Segment, k_new: torch.Tensor, v_new: torch.Tensor, position: int,
           ws: Optional[Workspace] = None, stream=None) -> None:
    """Append one token per sequence: k_new, v_new [B, Hkv, 128] (or [B, Hkv, 1, 128])."""
    ws = ws or default_workspace(k_new.device)
    st = _stream(stream)
    wp, wn = ws.get(256, "scratch", stream, st)
    check("uc_append", lib().uc_append(
        C.byref(seg.c), _ptr(k_new), _ptr(v_new), int(position), wp, wn, st))



def append_next(seg: Segment, k_new: torch.Tensor, v_new: torch.Tensor, base_position: int,
                ws: Optional[Workspace] = None, stream=None) -> None:
    """Like ``append`` with the logical index base_position + n_kept[b] taken on
    the device and no host-side state: capturable in a CUDA graph."""
    ws = ws or default_workspace(k_new.device)
    st = _stream(stream)
    wp, wn = ws.get(256, "scratch", stream, st)
    check("uc_append_next", lib().uc_append_next(
        C.byref(seg.c), _ptr(k_new), _ptr(v_new), int(base_position), wp, wn, st))


# -------------------------------------- layers with a state of constant size

def _new(stream, *makers):
    """New outputs of a launch on ``stream``: from that stream's memory (the
    current one's may hold what its queued work still uses), and not given away
    before the current stream, which called, is done with them."""
    if stream is None:
        return [make() for make in makers]
    here = torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        made = [make() for make in makers]
    for t in made:
        t.record_stream(here)
    return made


_pack_rows = struct.Struct("=Qqqq").pack   # uc_rows (bytes are built faster than a Structure)
_pack_item = struct.Struct("=QQQQQ").pack  # uc_reorder_item


def linear_attend(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: Sequence[float],
                  state: Optional[torch.Tensor] = None, out_state: Optional[torch.Tensor] = None,
                  lengths: Optional[Sequence[int]] = None, out: Optional[torch.Tensor] = None,
                  ws: Optional[Workspace] = None, stream=None):
    """Linear attention with a decay for each KV head (uc_linear_attend):
    S_t = exp(log_decay) S_{t-1} + k_t v_t^T, o_t = S_t^T q_t / sqrt(128).

    q [B, Hq, T, 128], k, v [B, Hkv, T, 128] bf16 with contiguous rows and any
    strides that are multiples of 8 (so [B, T, H, 128] memory transposed to
    [B, H, T, 128] works). log_decay: Hkv host floats <= 0. state [B, Hkv,
    128, 128] fp32: what earlier tokens left (None: zeros). out_state: where
    the new state goes (may be ``state``: in place). lengths: host tokens per
    sequence (None: T); outputs behind them are zero. Returns (out, out_state),
    out with q's shape (and its strides where q has no gaps)."""
    B, hq, T, d = q.shape
    kv = k.shape
    hkv = kv[1]
    sq, sk, sv = q.stride(), k.stride(), v.stride()
    if not q.dtype is k.dtype is v.dtype is torch.bfloat16 or d != HEAD_DIM:
        raise ValueError("linear_attend: q, k and v are bf16 with 128 channels")
    if kv != (B, hkv, T, d) or v.shape != kv or not sq[3] == sk[3] == sv[3] == 1:
        raise ValueError("linear_attend: k and v are [B, Hkv, T, 128], every row contiguous")
    if len(log_decay) != hkv or (lengths is not None and len(lengths) != B):
        raise ValueError("linear_attend: one log_decay per KV head, one length per sequence")
    if out is None:
        out = torch.empty_like(q) if stream is None else _new(stream, lambda: torch.empty_like(q))[0]
    elif out.shape != q.shape or out.dtype != q.dtype or out.stride(3) != 1:
        raise ValueError("linear_attend: out has q's shape and type, every row contiguous")
    for s in (state,) if out_state is None or out_state is state else (state, out_state):
        if s is not None and (s.shape != (B, hkv, d, d) or s.dtype is not torch.float32 or not s.is_contiguous()):
            raise ValueError("linear_attend: states are contiguous fp32 [B, Hkv, 128, 128]")
    if out_state is None:
        out_state = _new(stream, lambda: torch.empty((B, hkv, d, d), dtype=torch.float32, device=q.device))[0] \
            if state is None or stream is not None else torch.empty_like(state)
    ws = ws or default_workspace(q.device)
    L = lib()
    so = out.stride()
    args = (_pack_rows(q.data_ptr(), sq[0], sq[1], sq[2]), _pack_rows(k.data_ptr(), sk[0], sk[1], sk[2]),
            _pack_rows(v.data_ptr(), sv[0], sv[1], sv[2]), B, hq, hkv, T,
            None if lengths is None else (C.c_int32 * B)(*lengths), (C.c_float * hkv)(*log_decay), _ptr(state),
            out_state.data_ptr(), _pack_rows(out.data_ptr(), so[0], so[1], so[2]))
    st = _stream(stream)
    code = L.uc_linear_attend(*args, *ws.get(256, "scratch", stream, st), st)
    if code == _lib.UC_ERR_OOM:   # nothing is launched then: only now is the size asked for
        code = L.uc_linear_attend(*args, *ws.get(L.uc_linear_workspace_size(B, hq, hkv, T), "scratch", stream, st), st)
    check("uc_linear_attend", code)
    return out, out_state


# ----------------------------------- several continuations (beams) per request

_LOGIT_TYPES = {torch.float32: _lib.FP32, torch.bfloat16: _lib.BF16, torch.float16: _lib.FP16}


def beam_select(logits: torch.Tensor, scores: torch.Tensor, n: int, finished: Optional[torch.Tensor] = None,
                eos: int = -1, ws: Optional[Workspace] = None, stream=None):
    """The best n continuations of every request (uc_beam_select): logits [B,
    K, V] fp32, bf16 or fp16 (rows contiguous), scores [B, K] fp32, finished
    [B, K] bool or None -> (scores fp32, parent int32, token int32, finished
    bool), each [B, n], best first."""
    B, K, V = logits.shape
    sb, sk, sv = logits.stride()
    kind = _LOGIT_TYPES.get(logits.dtype)
    if kind is None or sv != 1:
        raise ValueError("beam_select: logits are fp32, bf16 or fp16 with contiguous rows")
    if scores.shape != (B, K) or scores.dtype != torch.float32 or not scores.is_contiguous():
        raise ValueError("beam_select: scores are contiguous fp32 [B, K]")
    if finished is not None and (finished.shape != (B, K) or finished.dtype not in (torch.bool, torch.uint8)
                                 or not finished.is_contiguous()):
        raise ValueError("beam_select: finished is contiguous bool [B, K]")
    dev = logits.device
    best, parent, token, done = _new(stream, *(partial(torch.empty, (B, n), dtype=t, device=dev)
                                               for t in (torch.float32, torch.int32, torch.int32, torch.bool)))
    ws = ws or default_workspace(dev)
    L = lib()
    args = (logits.data_ptr(), kind, sb, sk, B, K, V, scores.data_ptr(), _ptr(finished), eos, n,
            best.data_ptr(), parent.data_ptr(), token.data_ptr(), done.data_ptr())
    st = _stream(stream)
    code = L.uc_beam_select(*args, *ws.get(256, "scratch", stream, st), st)
    if code == _lib.UC_ERR_OOM:   # nothing is launched then: only now is the size asked for
        code = L.uc_beam_select(*args, *ws.get(L.uc_beam_workspace_size(B, K, V, n), "scratch", stream, st), st)
    check("uc_beam_select", code)
    return best, parent, token, done


def reorder(pairs, parent: torch.Tensor, ws: Optional[Workspace] = None, stream=None) -> None:
    """Caches follow their beams (uc_reorder). ``pairs``: (source, target)
    pairs of Segments, or of contiguous tensors [sequences, ...] such as the
    states of ``linear_attend``. parent [groups, n_to] int32: sequence g * n_to
    + i of a target becomes sequence g * n_from + parent[g, i] of its source,
    n_from = the sources' sequences / groups. Sources and targets share no
    storage: callers keep two of each and use them in turn."""
    if parent.dtype != torch.int32 or parent.dim() != 2 or not parent.is_contiguous():
        raise ValueError("reorder: parent is a contiguous int32 [groups, n_to]")
    groups, n_to = parent.shape
    items, n_seq = [], None
    for src, dst in pairs:
        if isinstance(src, Segment):
            have = src.batch
            items.append(_pack_item(C.addressof(src.c), C.addressof(dst.c), 0, 0, 0))
        else:
            have, *rest = src.shape
            to, *same = dst.shape
            if rest != same or to != groups * n_to or src.dtype != dst.dtype \
                    or not (src.is_contiguous() and dst.is_contiguous()):
                raise ValueError("reorder: tensors are contiguous [sequences, ...] of one type and shape per sequence")
            items.append(_pack_item(0, 0, src.data_ptr(), dst.data_ptr(),
                                    src.element_size() * (src.numel() // have if have else 0)))
        if n_seq not in (None, have):
            raise ValueError("reorder: the sources hold different numbers of sequences")
        n_seq = have
    if n_seq is None or groups == 0 or n_seq % groups:
        raise ValueError("reorder: the sources' sequences are a multiple of the groups")
    ws = ws or default_workspace(parent.device)
    st = _stream(stream)
    wp, wn = ws.get(256, "scratch", stream, st)
    check("uc_reorder", lib().uc_reorder(b"".join(items), len(items), parent.data_ptr(),
                                         groups, n_seq // groups, n_to, wp, wn, st))


# ------------------------------------------------- positions of tokens (rotary)

_BF16 = torch.bfloat16


def _device_of(fn: str, first: torch.Tensor, *others: Optional[torch.Tensor]) -> None:
    """The library takes plain addresses: what it cannot see of tensors."""
    at = first.get_device()
    if at < 0 or at != torch._C._cuda_getDevice():
        raise ValueError(f"{fn}: every tensor is on the current CUDA device")
    for t in others:
        if t is not None and t.get_device() != at:
            raise ValueError(f"{fn}: every tensor is on the current CUDA device")


def _head_rows(fn: str, name: str, x: torch.Tensor, like, dtype) -> bytes:
    """uc_rows of x [batch, heads, tokens, 128] of the shape ``like``."""
    s = x.stride()
    if x.shape != like or x.dtype is not dtype or s[-1] != 1:
        raise ValueError(f"{fn}: {name} is {dtype} {list(like)}, every row contiguous")
    return _pack_rows(x.data_ptr(), s[0], s[1], s[2])


def _counts(fn: str, name: str, x: torch.Tensor, batch: int) -> int:
    if x.dtype is not torch.int32 or x.dim() != 1 or x.shape[0] != batch or not x.is_contiguous():
        raise ValueError(f"{fn}: {name} is contiguous int32 [{batch}]")
    return x.data_ptr()


def _like(x: torch.Tensor, stream) -> torch.Tensor:
    return torch.empty_like(x) if stream is None else _new(stream, lambda: torch.empty_like(x))[0]


class Rotary:
    """A rotation by position (uc_rotary_table): ``freqs`` are the pairs'
    radians per token, 1 to 64 host floats; pair i is channels (i, i + pairs),
    or (2 i, 2 i + 1) where ``interleaved``; turned channels are multiplied by
    ``scale``, the others stay as they are. Long-context rescalings are a matter
    of the frequencies and the scale."""

    def __init__(self, freqs: Sequence[float], interleaved: bool = False, scale: float = 1.0):
        freqs = [float(f) for f in freqs]
        if not 1 <= len(freqs) <= _lib.MAX_ROTARY_PAIRS:
            raise ValueError(f"Rotary: 1 to {_lib.MAX_ROTARY_PAIRS} frequencies")
        self.c = _lib.UcRotaryTable(len(freqs), int(bool(interleaved)), float(scale))
        self.c.freq[:len(freqs)] = freqs
        self._at = C.addressof(self.c)


def rotary(table: Rotary, positions: torch.Tensor, q: torch.Tensor, k: Optional[torch.Tensor] = None,
           out_q: Optional[torch.Tensor] = None, out_k: Optional[torch.Tensor] = None, stream=None):
    """Rotary positions (uc_rotary) of q [B, Hq, T, 128] and k [B, Hkv, T, 128],
    fp32, bf16 or fp16 with contiguous rows and strides as ``linear_attend``
    takes them. positions int32: [B, T], or [B, 1] for the first token's.
    out_q, out_k: where they go (may be q and k themselves: in place). Returns (out_q, out_k),
    with the strides of q and k where these have no gaps."""
    dtype, shape = q.dtype, q.shape
    kind = _LOGIT_TYPES.get(dtype)
    if kind is None or len(shape) != 4 or shape[3] != HEAD_DIM:
        raise ValueError("rotary: q is fp32, bf16 or fp16 [B, Hq, T, 128]")
    B, hq, T, d = shape
    at = positions.shape
    if positions.dtype is not torch.int32 or len(at) != 2 or at[0] != B or at[1] not in (1, T) \
            or not positions.is_contiguous():
        raise ValueError("rotary: positions are contiguous int32 [B, T] or [B, 1]")
    rq, rk, ok, hkv = _head_rows("rotary", "q", q, shape, dtype), None, None, 0
    if k is not None:
        if k.dim() != 4:
            raise ValueError("rotary: k is [B, Hkv, T, 128]")
        hkv = k.shape[1]
        rk = _head_rows("rotary", "k", k, (B, hkv, T, d), dtype)
    elif out_k is not None:
        raise ValueError("rotary: out_k is the result for k")
    _device_of("rotary", q, k, positions, out_q, out_k)
    if out_q is None:
        out_q = _like(q, stream)
    oq = _head_rows("rotary", "out_q", out_q, shape, dtype)
    if k is not None:
        if out_k is None:
            out_k = _like(k, stream)
        ok = _head_rows("rotary", "out_k", out_k, k.shape, dtype)
    check("uc_rotary", lib().uc_rotary(table._at, positions.data_ptr(), at[1] == T, kind, B, T, rq, oq, hq, rk, ok, hkv,
                                       _stream(stream)))
    return out_q, out_k


# ----------------------------- layers with a sliding window and first tokens

class WindowCache:
    """The cache of a layer whose queries see the last ``window`` tokens and the
    first ``n_sink`` ones (uc_window_cache), over caller tensors k, v [B, Hkv,
    rows, 128] bf16 with contiguous rows. Token p lies in row p, or, where p >=
    n_sink, in row n_sink + (p - n_sink) mod (rows - n_sink): a ring, unless the rows
    hold every token. T tokens that are appended and then attend at once need window +
    T - 1 rows behind the first ones: with fewer their first queries miss tokens that
    the last of them replaced, which nothing reports. (A longer prompt attends over a
    WindowCache of its own k and v, turned by ``rotary``, and is appended afterwards.)
    An n_sink of all rows or more counts as one less. How many tokens a sequence holds
    is the caller's, on the device."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, window: int, n_sink: int = 0):
        if k.dim() != 4 or k.shape[3] != HEAD_DIM:
            raise ValueError("WindowCache: k and v are bf16 [B, Hkv, rows, 128]")
        for x, name in ((k, "k"), (v, "v")):
            _head_rows("WindowCache", name, x, k.shape, torch.bfloat16)
        if window < 1 or n_sink < 0:
            raise ValueError("WindowCache: window is at least 1, n_sink at least 0")
        if k.device != v.device:
            raise ValueError("WindowCache: k and v are on one device")
        self.k, self.v, self.window, self.n_sink = k, v, int(window), int(n_sink)
        self.batch, self.n_kv_heads, self.n_rows, _ = k.shape
        rows = [_lib.UcRows(x.data_ptr(), *x.stride()[:3]) for x in (k, v)]
        self.c = _lib.UcWindowCache(*rows, self.batch, self.n_kv_heads, self.n_rows, min(self.window, 1 << 30),
                                    min(self.n_sink, 1 << 30))
        self._at = C.addressof(self.c)


def window_append(cache: WindowCache, k: torch.Tensor, v: torch.Tensor, held: torch.Tensor,
                  n_new: Optional[torch.Tensor] = None, rotary: Optional[Rotary] = None,
                  q: Optional[torch.Tensor] = None, out_q: Optional[torch.Tensor] = None,
                  total: Optional[torch.Tensor] = None, ws: Optional[Workspace] = None, stream=None):
    """New tokens into ``cache`` (uc_window_append): k, v bf16 [B, Hkv, T, 128],
    token t < n_new[b] of sequence b at position held[b] + t, k turned by ``rotary``
    where that is given. q [B, Hq, T, 128]: turned beside them, into out_q (may
    be q). held, n_new: device int32 [B] (None: T each). Returns (total, out_q),
    total = held + n_new (another array than held)."""
    fn, shape = "window_append", k.shape
    if len(shape) != 4 or shape[0] != cache.batch or shape[1] != cache.n_kv_heads or shape[3] != HEAD_DIM:
        raise ValueError("window_append: k and v are bf16 [B, Hkv, T, 128]")
    B, T = shape[0], shape[2]
    rk, rv = _head_rows(fn, "k", k, shape, _BF16), _head_rows(fn, "v", v, shape, _BF16)
    if held is None or (out_q is not None if q is None else rotary is None or q.dim() != 4):
        raise ValueError("window_append: held is needed, and a rotary where there is a q [B, Hq, T, 128]")
    n_held = _counts(fn, "held", held, B)
    n_add = None if n_new is None else _counts(fn, "n_new", n_new, B)
    rq = oq = None
    hq = 0
    if q is not None:
        hq = q.shape[1]
        rq = _head_rows(fn, "q", q, (B, hq, T, HEAD_DIM), _BF16)
    _device_of(fn, k, v, cache.k, held, n_new, q, out_q, total)
    if total is None:
        total = _like(held, stream)
    if q is not None:
        if out_q is None:
            out_q = _like(q, stream)
        oq = _head_rows(fn, "out_q", out_q, q.shape, _BF16)
    ws = ws or default_workspace(k.device)
    st = _stream(stream)
    wp, wn = ws.get(256, "scratch", stream, st)
    check("uc_window_append", lib().uc_window_append(
        cache._at, rk, rv, T, n_held, n_add, None if rotary is None else rotary._at, rq, oq, hq,
        _counts(fn, "total", total, B), wp, wn, st))
    return total, out_q


def window_attend(q: torch.Tensor, cache: WindowCache, lengths: torch.Tensor, n_query: Optional[torch.Tensor] = None,
                  out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, want_lse: bool = True,
                  ws: Optional[Workspace] = None, stream=None):
    """Attention with a sliding window and first tokens (uc_window_attend): the
    queries q bf16 [B, Hq, T, 128] are the last n_query[b] (None: T) of the
    lengths[b] tokens that sequence b holds in ``cache``, their own among them (as
    far as a ring still has what they see: see WindowCache); device int32 [B]. Returns (out, lse): out with q's shape (and its strides
    where q has no gaps), 0 behind a sequence's last query; lse fp32 [B, Hq, T] or None."""
    fn, shape = "window_attend", q.shape
    if len(shape) != 4 or shape[0] != cache.batch or shape[3] != HEAD_DIM or lengths is None:
        raise ValueError("window_attend: lengths are needed, and q is bf16 [B, Hq, T, 128]")
    B, hq, T, _ = shape
    rq = _head_rows(fn, "q", q, shape, _BF16)
    n = _counts(fn, "lengths", lengths, B)
    n_last = None if n_query is None else _counts(fn, "n_query", n_query, B)
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != (B, hq, T) or not lse.is_contiguous()):
        raise ValueError("window_attend: lse is contiguous fp32 [B, Hq, T]")
    _device_of(fn, q, cache.k, lengths, n_query, out, lse)
    if out is None:
        out = _like(q, stream)
    ro = _head_rows(fn, "out", out, shape, _BF16)
    if want_lse and lse is None:
        lse = _new(stream, lambda: torch.empty((B, hq, T), dtype=torch.float32, device=q.device))[0]
    ws = ws or default_workspace(q.device)
    L = lib()
    st = _stream(stream)
    args = (cache._at, rq, hq, T, n, n_last, ro, None if lse is None else lse.data_ptr())
    code = L.uc_window_attend(*args, *ws.get(256, "scratch", stream, st), st)
    if code == _lib.UC_ERR_OOM:   # nothing is launched then: only now is the size asked for
        code = L.uc_window_attend(*args, *ws.get(L.uc_window_workspace_size(cache._at, hq, T), "scratch", stream, st), st)
    check("uc_window_attend", code)
    return out, lse


# ------------------------------------------------------------- drafted tokens

def verify_draft(logits: torch.Tensor, tokens: torch.Tensor, u: Optional[torch.Tensor] = None,
                 noise: Optional[torch.Tensor] = None, draft_logits: Optional[torch.Tensor] = None,
                 n_draft: Optional[torch.Tensor] = None, temperature: float = 1.0, ws: Optional[Workspace] = None,
                 stream=None):
    """Drafted tokens against the target's probabilities (uc_verify_draft):
    logits [B, T + 1, V] of the target, draft_logits [B, T, V] of the drafter (None:
    the drafts are taken as certain), fp32, bf16 or fp16 with contiguous rows; tokens
    int32 [B, T] the drafts, n_draft int32 [B] how many (None: T each). u fp32
    [B, T] uniform in [0, 1), noise fp32 [B, V] exponential variates; neither is
    needed at temperature 0. Returns (accepted int32 [B], tokens int32 [B, T + 1]:
    the accepted drafts, the next token, then -1; log probabilities fp32 [B, T + 1])."""
    fn, shape, strides = "verify_draft", logits.shape, logits.stride()
    kind = _LOGIT_TYPES.get(logits.dtype)
    if kind is None or len(shape) != 3 or strides[2] != 1:
        raise ValueError("verify_draft: logits are fp32, bf16 or fp16 [B, T + 1, V] with contiguous rows")
    B, T1, V = shape
    T = T1 - 1
    if tokens.dtype is not torch.int32 or tokens.shape != (B, T) or not tokens.is_contiguous():
        raise ValueError("verify_draft: tokens are contiguous int32 [B, T]")
    pd, db, dt = None, 0, 0
    if draft_logits is not None:
        db, dt, dv = draft_logits.stride() if draft_logits.dim() == 3 else (0, 0, 0)
        if draft_logits.dtype is not logits.dtype or draft_logits.shape != (B, T, V) or dv != 1:
            raise ValueError("verify_draft: draft_logits are [B, T, V] of the logits' type with contiguous rows")
        pd = draft_logits.data_ptr()
    pu = pe = None
    if u is not None:
        if u.dtype is not torch.float32 or u.shape != (B, T) or not u.is_contiguous():
            raise ValueError("verify_draft: u is contiguous fp32 [B, T]")
        pu = u.data_ptr()
    if noise is not None:
        if noise.dtype is not torch.float32 or noise.shape != (B, V) or not noise.is_contiguous():
            raise ValueError("verify_draft: noise is contiguous fp32 [B, V]")
        pe = noise.data_ptr()
    if temperature != 0 and (pu is None or pe is None):
        raise ValueError("verify_draft: u and noise are needed unless temperature is 0")
    n = None if n_draft is None else _counts(fn, "n_draft", n_draft, B)
    _device_of(fn, logits, tokens, draft_logits, u, noise, n_draft)
    dev = logits.device
    if stream is None:
        accepted = torch.empty((B,), dtype=torch.int32, device=dev)
        out = torch.empty((B, T1), dtype=torch.int32, device=dev)
        logprob = torch.empty((B, T1), dtype=torch.float32, device=dev)
    else:
        accepted, out, logprob = _new(stream, partial(torch.empty, (B,), dtype=torch.int32, device=dev),
                                      partial(torch.empty, (B, T1), dtype=torch.int32, device=dev),
                                      partial(torch.empty, (B, T1), dtype=torch.float32, device=dev))
    ws = ws or default_workspace(dev)
    L = lib()
    args = (logits.data_ptr(), strides[0], strides[1], pd, db, dt, kind, B, T, V, tokens.data_ptr(), n, pu, pe,
            temperature, accepted.data_ptr(), out.data_ptr(), logprob.data_ptr())
    st = _stream(stream)
    code = L.uc_verify_draft(*args, *ws.get(256, "scratch", stream, st), st)
    if code == _lib.UC_ERR_OOM:   # nothing is launched then: only now is the size asked for
        code = L.uc_verify_draft(*args, *ws.get(L.uc_verify_workspace_size(B, T, V), "scratch", stream, st), st)
    check("uc_verify_draft", code)
    return accepted, out, logprob


def set_dense_serial_pv(serial: bool) -> bool:
    """A setting of the dense attention kernel kept for its callers, without
    effect any more (see unicache.h); returns the previous one."""
    return bool(lib().uc_set_dense_serial_pv(1 if serial else 0))


def set_wait_limit(ns: int) -> int:
    """Limit of the decode kernels' bounded waits in ns (0: the default,
    2 s); returns the previous value."""
    return int(lib().uc_set_wait_limit(int(ns)))


def set_programmatic_launch(on: bool) -> bool:
    """Programmatic dependent launch of the decode kernels (see
    unicache.h for the ordering it asks of the caller); returns the previous
    setting."""
    return bool(lib().uc_set_programmatic_launch(1 if on else 0))


def debug_withhold_tile(pos: int) -> None:
    """Test hook: the next decode attention call never copies the first tile
    of its work item at processing position ``pos``, or the next quantization
    or chunked linear attention one of its copies (see unicache.h)."""
    lib().uc_debug_withhold_tile(int(pos))


def launch_count() -> int:
    return int(lib().uc_launch_count())


def version() -> int:
    return int(lib().uc_version())
