"""Decode-step runtime over the C ABI (device memory and streams via torch).

Per layer and decode step t (Fig. 1; Section 4):

    stream S (critical):    score_topk(q_t) -> IS^t, A^t   | repair(A^t, P^t, spec) -> o_t
    stream P (speculation): spec_attn(q_t, P^t)            | predict(IS^t) -> P^{t+1}

spec_attn needs only q_t and P^t (predicted at the end of step t-1), so it runs while
the selection is in flight; repair waits for both; the EMA update and the next
prediction wait for the selection only and are off the critical path.  The serial
baseline is score_topk followed by repair with no prediction, on one stream.

Around the step, PagedCache (and a LayerState's prefill and append) writes new tokens with their rotary
positions into the paged cache, attends prompts and whole caches, and keeps a cache in e4m3.

All arithmetic happens in libprr.so; this module only allocates, uploads and orders.
"""
from __future__ import annotations

import ctypes
import dataclasses
from typing import List, Optional, Sequence

import numpy as np
import torch

from . import _lib as L


@dataclasses.dataclass
class PathConfig:
    num_q_heads: int
    num_kv_heads: int
    page_size: int
    num_tokens: int
    k_select: int
    forced: Sequence[int] = ()
    forced_in_budget: bool = True
    dtype: str = "bf16"  # "bf16" | "f16"
    meta_kind: str = "minmax"  # "minmax" | "mean"
    alpha: float = 0.5
    beta: float = 0.5
    gamma: float = 0.0
    p_select: Optional[int] = None  # |P| budget; default = k_select (delta = 1)
    chunk_pages: int = 8
    mode: int = L.PRR_EXACT_SELECTED
    max_pages: Optional[int] = None

    @property
    def group(self):
        return self.num_q_heads // self.num_kv_heads

    @property
    def num_pages(self):
        return (self.num_tokens + self.page_size - 1) // self.page_size

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == "bf16" else torch.float16

    def dims(self):
        return L.make_dims(self.num_q_heads, self.num_kv_heads, self.page_size, self.max_pages or self.num_pages,
                           L.PRR_BF16 if self.dtype == "bf16" else L.PRR_F16,
                           L.PRR_META_MEAN if self.meta_kind == "mean" else L.PRR_META_MINMAX)

    def list_cap(self):
        """Entries of the longest list, for as many tokens as the pages can hold."""
        nf = len(self.forced)
        pages = self.max_pages or self.num_pages
        def size(k):
            return min(pages, max(k, nf) if self.forced_in_budget else k + nf)
        return max(1, size(self.k_select), size(self.p_select if self.p_select is not None else self.k_select))


def bits_tensor(bits: np.ndarray, dtype: torch.dtype, device) -> torch.Tensor:
    """Upload 16-bit storage patterns as a tensor of the given 16-bit dtype."""
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16))
    return t.to(device).view(dtype)


class Rope:
    """Rotary positions of a model: frequencies (prr_rope_freqs, or given: one per pair) on the device, layout and scale
    (None: that of the frequencies' rule, 1 for given ones)."""

    KINDS = {"plain": L.PRR_ROPE_PLAIN, "linear": L.PRR_ROPE_LINEAR, "ntk": L.PRR_ROPE_NTK,
             "by_parts": L.PRR_ROPE_BY_PARTS, "yarn": L.PRR_ROPE_YARN}

    def __init__(self, device, rot_dim=128, base=10000.0, kind="plain", factor=1.0, trained_len=1, lo=1.0, hi=32.0,
                 interleaved=False, freqs=None, scale=None):
        rule = 1.0
        if freqs is None:
            freqs, rule = L.prr_rope_freqs(self.KINDS[kind], rot_dim, base, factor, trained_len, lo, hi)
        self.freqs = torch.as_tensor(freqs, dtype=torch.float64).to(device).contiguous()
        if self.freqs.dim() != 1 or not len(self.freqs):
            raise ValueError(f"freqs: shape {tuple(self.freqs.shape)}, expected one number per pair")
        self.rot_dim, self.scale = 2 * self.freqs.numel(), float(rule if scale is None else scale)
        self.layout = L.PRR_ROPE_INTERLEAVED if interleaved else L.PRR_ROPE_HALF


class Batch:
    """The sequences of a call: their new tokens, their tokens in the cache (the new ones included) and
    their rows of the page table.  The lengths live on the device (cu_q, kv_len), where a captured graph
    reads them; max_q, max_kv and total_q (rows of the packed tensors) bound them for as long as the batch is
    used: the device cuts what is beyond."""

    def __init__(self, device, new: Sequence[int], kv: Sequence[int], page_table=None, max_q=None, max_kv=None, total_q=None):
        if len(new) != len(kv) or not len(new) or min(new) < 0 or min(kv) < 0:
            raise ValueError("new and kv: lengths of the same sequences, at least one, none negative")
        cu = np.concatenate([[0], np.cumsum(np.asarray(new, dtype=np.int64))]).astype(np.int32)
        for name, bound, least in (("max_q", max_q, max(new)), ("max_kv", max_kv, max(kv)), ("total_q", total_q, int(cu[-1]))):
            if bound is not None and bound < least:
                raise ValueError(f"{name} {bound}: the lengths need {least}")
        self._longest, self._max_kv = max(kv), max(kv) if max_kv is None else max_kv
        self.kv_len = torch.tensor(list(kv), dtype=torch.int32, device=device)
        if page_table is not None:
            _check(page_table, "page_table", (len(new), page_table.shape[-1]), torch.int32, self.kv_len.device)
        self.page_table = page_table
        # one new token each: rows are sequences
        self.cu_q = None if all(n == 1 for n in new) else torch.from_numpy(cu).to(device)
        self.total_q = int(cu[-1]) if total_q is None else total_q
        self.native = L.make_batch(len(self.kv_len), self.total_q, max(new) if max_q is None else max_q,
                                   self._max_kv, self.cu_q, self.kv_len, page_table,
                                   0 if page_table is None else page_table.shape[-1])

    def set_lengths(self, kv: Sequence[int]):
        """Tokens of each sequence in the cache from now on (on the current stream)."""
        if len(kv) != len(self.kv_len) or min(kv) < 0 or max(kv) > self._max_kv:
            raise ValueError(f"{len(self.kv_len)} lengths within [0, {self._max_kv}] are needed")
        self.kv_len.copy_(torch.tensor(list(kv), dtype=torch.int32))
        self._longest = max(kv)

    def advance(self):
        """Every sequence is one token longer (on the current stream).  Replays of a captured graph that holds
        this are not counted here: max_kv has to leave room for them."""
        if self._longest >= self._max_kv:
            raise ValueError(f"a sequence of {self._longest} tokens cannot grow beyond max_kv {self._max_kv}")
        self._longest += 1
        self.kv_len.add_(1)


class _OnStream:
    """torch.cuda.stream() for a stream of the current device, without its look-ups (under 2 us, not 6)."""
    __slots__ = ("stream", "before")

    def __init__(self, stream):
        self.stream = stream

    def __enter__(self):
        s = self.stream
        self.before = torch._C._cuda_getCurrentStream(s.device_index)
        torch._C._cuda_setStream(stream_id=s.stream_id, device_index=s.device_index, device_type=s.device_type)

    def __exit__(self, *_):
        i, device, kind = self.before
        torch._C._cuda_setStream(stream_id=i, device_index=device, device_type=kind)


def _stream_context(stream, device):
    """What is allocated inside belongs to `stream` (None: the device's current one), as the kernels that write it."""
    if stream is None:
        return torch.cuda.device(device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device)
    return _OnStream(stream) if stream.device_index == torch._C._cuda_getDevice() else torch.cuda.stream(stream)


def _check(x, name, shape, dtype, device, dense=True):
    """x has the shape, type and device that the kernels take for granted."""
    if x is None:
        raise ValueError(f"{name} is missing")
    if x.dtype != dtype or x.shape != shape or x.device != device or (dense and not x.is_contiguous()):
        raise ValueError(f"{name}: {x.dtype} {tuple(x.shape)}, strides {x.stride()}, on {x.device}; expected "
                         f"{'dense ' if dense else ''}{dtype} {tuple(shape)} on {device}")


class PagedCache:
    """One layer's paged cache, in 16 bits or e4m3, for any number of sequences: new tokens are appended with
    their rotary positions, prompts and single tokens attend it, e4m3 pages are read back.

    A call's workspace, and outputs that are not given, are allocated on the call's stream; the workspace goes back
    there when the call returns.  So calls on other streams never share one, and a captured graph has its own, in its pool."""

    def __init__(self, cfg: PathConfig, device, kind="16", k=None, v=None, k_scale=None, v_scale=None):
        """k, v: given caches (e4m3 codes with k_scale, v_scale, the exponent bytes of their rows' powers of two), or None
        for empty ones."""
        self.cfg, self.dims = cfg, cfg.dims()
        self.kind = {"16": L.PRR_KV_16, "e4m3": L.PRR_KV_E4M3}[kind]
        shape = (cfg.num_kv_heads, self.dims.max_pages, cfg.page_size, 128)
        dtype = cfg.torch_dtype if kind == "16" else torch.float8_e4m3fn
        self.k = torch.zeros(shape, dtype=torch.uint8, device=device).view(dtype) if k is None and kind == "e4m3" else \
            torch.zeros(shape, dtype=dtype, device=device) if k is None else k
        self.v = torch.zeros_like(self.k) if v is None else v
        for x, name in ((self.k, "k"), (self.v, "v")):
            _check(x, name, shape, dtype, self.k.device)
        if self.k.device.type != torch.device(device).type:
            raise ValueError(f"k: on {self.k.device}, expected on {device}")
        for x, scale, name in ((k, k_scale, "k_scale"), (v, v_scale, "v_scale")):
            if kind == "e4m3" and (x is None) != (scale is None):
                raise ValueError(f"{name}: codes come with their scales, or neither is given")
            if scale is not None:
                if kind != "e4m3":
                    raise ValueError(f"{name}: a 16-bit cache has no scales")
                _check(scale, name, shape[:3], torch.uint8, self.k.device)
        self.k_scale, self.v_scale = k_scale, v_scale
        if kind == "e4m3":  # (127 is 1)
            empty = lambda: torch.full(shape[:3], 127, dtype=torch.uint8, device=self.k.device)  # noqa: E731
            self.k_scale = empty() if k_scale is None else k_scale
            self.v_scale = empty() if v_scale is None else v_scale

    def _check_batch(self, batch, q):
        """The device of the batch's lengths; the queries of a call that attends."""
        if batch.kv_len.device != self.k.device:
            raise ValueError(f"batch: on {batch.kv_len.device}, expected on {self.k.device}")
        if q is not None:
            _check(q, "q", (batch.total_q, self.cfg.num_q_heads, 128), self.cfg.torch_dtype, self.k.device)

    def _workspace(self, nbytes, stream):
        if not nbytes:
            return None
        if stream is None:
            return torch.empty(nbytes, dtype=torch.uint8, device=self.k.device)
        with _stream_context(stream, self.k.device):
            return torch.empty(nbytes, dtype=torch.uint8, device=self.k.device)

    def append(self, batch: Batch, q, k, v, rope: Optional[Rope] = None, positions=None, q_out=None, stream=None):
        """New tokens' keys and values into the cache, rotated; returns the rotated queries."""
        cfg, rows = self.cfg, batch.total_q
        for x, name, heads, dense in ((q, "q", cfg.num_q_heads, False), (k, "k", cfg.num_kv_heads, False),
                                      (v, "v", cfg.num_kv_heads, False), (q_out, "q_out", cfg.num_q_heads, True)):
            if x is not None:
                _check(x, name, (rows, heads, 128), cfg.torch_dtype, self.k.device, dense)
        self._check_batch(batch, None)
        if positions is not None:
            _check(positions, "positions", (rows,), torch.int32, self.k.device)
        if rope is not None and rope.freqs.device != self.k.device:
            raise ValueError(f"rope: on {rope.freqs.device}, expected on {self.k.device}")
        if q is not None and q_out is None:
            with _stream_context(stream, self.k.device):
                q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        L.prr_rope_append(self.dims, batch.native, q, k, v, positions, None if rope is None else rope.freqs,
                          0 if rope is None else rope.rot_dim, L.PRR_ROPE_HALF if rope is None else rope.layout,
                          1.0 if rope is None else rope.scale, q_out, self.kind, self.k, self.v, self.k_scale, self.v_scale,
                          stream)
        return q_out

    def prompt(self, batch: Batch, q, out=None, stream=None):
        """Causal attention of the new tokens: (o in the 16-bit type, m, l); in `out`, m and l may both be None."""
        if self.kind != L.PRR_KV_16:
            raise ValueError("prompts attend a 16-bit cache: read() the pages back first")
        self._check_batch(batch, q)
        nbytes = L.prr_prompt_workspace_size(self.dims, batch.native)
        if out is None:
            with _stream_context(stream, self.k.device):
                n, hq = q.shape[:2]
                out = (torch.zeros_like(q), *(torch.zeros(n, hq, dtype=torch.float32, device=q.device) for _ in range(2)))
        else:
            for x, name, ref in zip(out, ("o", "m", "l"), (q.shape, q.shape[:2], q.shape[:2]), strict=True):
                if x is None and name != "o":
                    continue  # (the call itself refuses one of m and l alone)
                _check(x, name, ref, q.dtype if name == "o" else torch.float32, self.k.device)
        L.prr_prompt_attn(self.dims, batch.native, q, self.k, self.v, *out, self._workspace(nbytes, stream), nbytes, stream)
        return out

    def attend(self, batch: Batch, q, pages=None, counts=None, out=None, stream=None):
        """Attention of one token per sequence over its whole cache, or over listed pages
        ([sequence][KV head][cap] and [sequence][KV head]): (o float32, o in the 16-bit type, m, l);
        in `out`, the 16-bit o may be None."""
        self._check_batch(batch, q)
        cap = 0 if pages is None else pages.shape[-1]
        if pages is not None:
            per_head = (batch.native.n_seqs, self.cfg.num_kv_heads)
            _check(pages, "pages", (*per_head, cap), torch.int32, self.k.device)
            _check(counts, "counts", per_head, torch.int32, self.k.device)
        nbytes = L.prr_decode_workspace_size(self.dims, batch.native, self.kind, cap)
        if out is None:
            with _stream_context(stream, self.k.device):
                n, hq = q.shape[:2]
                f32 = dict(dtype=torch.float32, device=q.device)
                out = (torch.zeros(n, hq, 128, **f32), torch.zeros_like(q), torch.zeros(n, hq, **f32), torch.zeros(n, hq, **f32))
        else:
            for x, name, ref in zip(out, ("o32", "o", "m", "l"), (q.shape, q.shape, q.shape[:2], q.shape[:2]), strict=True):
                if x is not None or name != "o":
                    _check(x, name, ref, q.dtype if name == "o" else torch.float32, self.k.device)
        L.prr_decode_attn(self.dims, batch.native, q, self.kind, self.k, self.v, self.k_scale, self.v_scale, pages, counts, cap,
                          *out, self._workspace(nbytes, stream), nbytes, stream)
        return out

    def read(self, num_tokens, page_table=None, page_begin=0, page_end=None, out=None, stream=None):
        """Pages of a sequence of an e4m3 cache in 16 bits: (k, v) [Hkv][pages][page_size][128]."""
        if page_end is None:
            page_end = -(-num_tokens // self.cfg.page_size)
        if page_table is not None:
            _check(page_table, "page_table", (max(page_end, page_table.numel()),), torch.int32, self.k.device)
        shape = (self.cfg.num_kv_heads, page_end - page_begin, self.cfg.page_size, 128)
        if out is None:
            if page_begin < 0 or page_end < page_begin:
                raise ValueError(f"pages {page_begin} to {page_end}")
            with _stream_context(stream, self.k.device):
                out = tuple(torch.zeros(shape, dtype=self.cfg.torch_dtype, device=self.k.device) for _ in range(2))
        else:
            for x, name in zip(out, ("k", "v"), strict=True):
                _check(x, name, shape, self.cfg.torch_dtype, self.k.device)
        L.prr_cache_read(self.dims, self.k, self.v, self.k_scale, self.v_scale, page_table, num_tokens, page_begin, page_end,
                         *out, stream)
        return out


class LayerState:
    """Device memory of one layer: KV cache, metadata, EMA state, lists, partials, outputs."""

    def __init__(self, cfg: PathConfig, device, k=None, v=None, page_table=None):
        self.cfg = cfg
        self.dims = cfg.dims()
        hkv, g, d = cfg.num_kv_heads, cfg.group, 128
        mp = self.dims.max_pages
        dev = device
        self.cap = cfg.list_cap()
        f32 = dict(dtype=torch.float32, device=dev)
        i32 = dict(dtype=torch.int32, device=dev)
        self.k = k if k is not None else torch.zeros(hkv, mp, cfg.page_size, d, dtype=cfg.torch_dtype, device=dev)
        self.v = v if v is not None else torch.zeros_like(self.k)
        self.page_table = page_table
        if cfg.meta_kind == "mean":
            self.meta = torch.zeros(hkv, mp, d, **f32)
        else:
            self.meta = torch.zeros(hkv, mp, 2, d, dtype=cfg.torch_dtype, device=dev)
        self.scores = torch.zeros(hkv, mp, **f32)
        self.level = torch.zeros(hkv, mp, **f32)
        self.trend = torch.zeros(hkv, mp, **f32)
        self.init_bits = torch.zeros(hkv, (mp + 31) // 32, **i32)
        self.sel = torch.zeros(hkv, self.cap, **i32)
        self.sel_count = torch.zeros(hkv, **i32)
        self.pred = [torch.zeros(hkv, self.cap, **i32) for _ in range(2)]
        self.pred_count = [torch.zeros(hkv, **i32) for _ in range(2)]
        _, po, pml, pm = L.prr_spec_state_floats(self.dims, self.cap, cfg.chunk_pages)
        self.part_o = torch.zeros(po, **f32)
        self.part_m = torch.zeros(pml, **f32)
        self.part_l = torch.zeros(pml, **f32)
        self.page_m = torch.zeros(pm, **f32)
        self.out_o32 = torch.zeros(cfg.num_q_heads, d, **f32)
        self.out_o = torch.zeros(cfg.num_q_heads, d, dtype=cfg.torch_dtype, device=dev)
        self.out_m = torch.zeros(cfg.num_q_heads, **f32)
        self.out_l = torch.zeros(cfg.num_q_heads, **f32)
        self.missed = torch.zeros(hkv, **i32)
        self.wasted = torch.zeros(hkv, **i32)
        self.covered = torch.zeros(hkv, **i32)
        self.ws_bytes = L.prr_workspace_size(self.dims, self.cap, cfg.chunk_pages)
        self.workspace = torch.empty(self.ws_bytes // 4 + 64, dtype=torch.int32, device=dev)
        L.prr_workspace_init(self.workspace, self.ws_bytes)
        self.cur = 0  # which predicted-list buffer holds P^t
        self.theta = None  # this layer's (alpha, beta, gamma), host float32 [3], or None (the step's)

    # --------------------------------------------------------------- prompts and new tokens
    def cache(self) -> PagedCache:
        """This layer's keys and values as a PagedCache (the same memory)."""
        if getattr(self, "_cache", None) is None:
            # (as many pages as the layer has, whatever its tokens are by now)
            self._cache = PagedCache(dataclasses.replace(self.cfg, max_pages=self.dims.max_pages), self.k.device, k=self.k, v=self.v)
        return self._cache

    def batch(self, new_tokens, stream=None) -> Batch:
        """The layer's sequence with `new_tokens` new ones at the end of its cfg.num_tokens, for calls on `stream`: its
        lengths are uploaded there, and their memory goes back there (so not in a capture)."""
        table = None if self.page_table is None else self.page_table.view(1, -1)
        with _stream_context(stream, self.k.device):
            if torch.cuda.is_current_stream_capturing():
                raise ValueError("a captured call needs a batch made before: its lengths are uploaded")
            return Batch(self.k.device, [new_tokens], [self.cfg.num_tokens], table)

    def _one(self, batch, new_tokens, stream):
        if batch is not None and batch.native.n_seqs != 1:
            raise ValueError(f"a batch of {batch.native.n_seqs} sequences: a layer holds one")
        return self.batch(new_tokens, stream) if batch is None else batch

    def prefill(self, q, k, v, rope: Optional[Rope] = None, batch: Optional[Batch] = None, stream=None):
        """The last len(q) of the cfg.num_tokens tokens: into the cache, their causal attention, and the metadata
        of the pages that they touch.  q [n][Hq][128], k, v [n][Hkv][128]; returns (o, m, l).  A given batch holds
        this one sequence, of cfg.num_tokens tokens; its rows may be more than its new tokens."""
        cfg = self.cfg
        batch = self._one(batch, q.shape[0], stream)
        q = self.cache().append(batch, q, k, v, rope, stream=stream)
        out = self.cache().prompt(batch, q, stream=stream)
        # (rows behind the tokens, and tokens without a place, count for none)
        self.build_meta(stream, page_begin=max(0, cfg.num_tokens - q.shape[0]) // cfg.page_size)
        return out

    def append(self, q, k, v, rope: Optional[Rope] = None, batch: Optional[Batch] = None, q_out=None, stream=None):
        """One new token, the last of the cfg.num_tokens: into the cache, and its page's metadata; returns the
        rotated query, ready for select() or a decode step.  The metadata's page is that of this moment: a captured graph
        keeps it."""
        cfg = self.cfg
        q = self.cache().append(self._one(batch, 1, stream), q, k, v, rope, q_out=q_out, stream=stream)
        self.build_meta(stream, page_begin=(cfg.num_tokens - 1) // cfg.page_size)
        return q

    # --------------------------------------------------------------- steps
    def build_meta(self, stream=None, page_begin=0, page_end=None):
        cfg = self.cfg
        L.prr_build_page_meta(self.dims, self.k, self.page_table, cfg.num_tokens, page_begin,
                              cfg.num_pages if page_end is None else page_end, self.meta, stream)

    def select(self, q, stream=None):
        cfg = self.cfg
        L.prr_score_topk(self.dims, q, self.meta, cfg.num_pages, cfg.k_select, cfg.forced, cfg.forced_in_budget,
                         self.scores, self.sel, self.sel_count, self.cap, self.workspace, self.ws_bytes, stream)

    def predict(self, with_scores=True, stream=None):
        """EMA update with this step's scores, then P for the next step (into the other buffer)."""
        cfg = self.cfg
        nxt = 1 - self.cur
        L.prr_predict(self.dims, self.level, self.trend, self.init_bits, self.scores if with_scores else None,
                      cfg.num_pages, cfg.alpha, cfg.beta, cfg.gamma,
                      cfg.k_select if cfg.p_select is None else cfg.p_select, cfg.forced, cfg.forced_in_budget,
                      self.pred[nxt], self.pred_count[nxt], self.cap, stream)

    def advance(self):
        self.cur = 1 - self.cur

    def speculate(self, q, stream=None, pages=None, counts=None):
        cfg = self.cfg
        L.prr_spec_attn(self.dims, q, self.k, self.v, self.page_table, cfg.num_tokens,
                        self.pred[self.cur] if pages is None else pages,
                        self.pred_count[self.cur] if counts is None else counts,
                        self.cap, cfg.chunk_pages, self.part_o, self.part_m, self.part_l, self.page_m, stream)

    def repair(self, q, stream=None, serial=False, mode=None, pages=None, counts=None):
        cfg = self.cfg
        pred = None if serial else (self.pred[self.cur] if pages is None else pages)
        cnt = None if serial else (self.pred_count[self.cur] if counts is None else counts)
        L.prr_repair(self.dims, q, self.k, self.v, self.page_table, cfg.num_tokens, cfg.num_pages, self.sel,
                     self.sel_count, pred, cnt, self.cap, cfg.chunk_pages, self.part_o, self.part_m, self.part_l,
                     self.page_m, cfg.mode if mode is None else mode, self.out_o32, self.out_o, self.out_m,
                     self.out_l, self.missed, self.wasted, self.workspace, self.ws_bytes, stream)


    def io(self, q):
        """This layer's buffers as the C ABI's prr_layer_io (q: the layer's query tensor)."""
        def ptr(t):
            return None if t is None else t.data_ptr()
        y = L.prr_layer_io()
        y.q, y.k_cache, y.v_cache, y.page_table, y.meta = ptr(q), ptr(self.k), ptr(self.v), ptr(self.page_table), ptr(self.meta)
        y.scores, y.ema_level, y.ema_trend, y.ema_init_bits = ptr(self.scores), ptr(self.level), ptr(self.trend), ptr(self.init_bits)
        y.selected, y.selected_count = ptr(self.sel), ptr(self.sel_count)
        y.predicted[0], y.predicted[1] = ptr(self.pred[0]), ptr(self.pred[1])
        y.predicted_count[0], y.predicted_count[1] = ptr(self.pred_count[0]), ptr(self.pred_count[1])
        y.part_o, y.part_m, y.part_l, y.page_m = ptr(self.part_o), ptr(self.part_m), ptr(self.part_l), ptr(self.page_m)
        y.out_o32, y.out_o, y.out_m, y.out_l = ptr(self.out_o32), ptr(self.out_o), ptr(self.out_m), ptr(self.out_l)
        y.missed_count, y.wasted_count = ptr(self.missed), ptr(self.wasted)
        y.covered_count = ptr(self.covered)
        y.workspace, y.ws_bytes = ptr(self.workspace), self.ws_bytes
        y.theta = None if self.theta is None else self.theta.ctypes.data
        return y


# Section 4.2: the calibration grid, alpha in 0.2..0.8 step 0.2, beta in 0.1..0.5 step 0.1,
# gamma in 0..0.75 step 0.25 (80 candidates).
THETA_GRID = [(a, b, c) for a in (0.2, 0.4, 0.6, 0.8) for b in (0.1, 0.2, 0.3, 0.4, 0.5)
              for c in (0.0, 0.25, 0.5, 0.75)]


def pick_delta(lut, context, degree=2):
    """Section 4.4's speculation budget for this context length, decided by the library
    (prr_pick_delta) from the profiled table `lut` (rows with "context", "delta",
    "select_us", "spec_us").  Returns the chosen delta."""
    return L.prr_pick_delta(lut, context, degree)[0]


def pick_delta_step(lut, context, degree=2):
    """The budget among those whose speculation fits the selection window (the test of
    pick_delta, per delta) with the shortest profiled step ("fused_prr_late_us") at this
    context; pick_delta's choice when the context was not profiled or the rows carry no
    step latency.  Returns (delta, step latency or None)."""
    rows = [r for r in lut if r["context"] == context and r.get("fused_prr_late_us") is not None]
    if not rows:
        return pick_delta(lut, context, degree), None
    fits = [r for r in rows if r["delta"] == 1.0 or
            L.prr_pick_delta([x for x in lut if x["delta"] == r["delta"]], context, degree)[0] == r["delta"]]
    best = min(fits, key=lambda r: (r["fused_prr_late_us"], r["delta"]))
    return best["delta"], best["fused_prr_late_us"]


_epoch = [0]


def next_epoch():
    """A process-wide increasing value: the fused schedules need a new one for every call
    on a workspace (the device-side hand-offs of a call are tagged with it)."""
    _epoch[0] += 1
    assert _epoch[0] < GRAPH_EPOCH_BASE
    return _epoch[0]


# Captured fused steps read their epoch from one device word per device, advanced by
# every replay; it counts up from 2^30, above every epoch the host hands out.
GRAPH_EPOCH_BASE = 1 << 30
_device_epoch = {}


def device_epoch(device) -> torch.Tensor:
    dev = torch.device(device)
    key = (dev.type, dev.index if dev.index is not None else torch.cuda.current_device())
    if key not in _device_epoch:
        _device_epoch[key] = torch.full((1,), GRAPH_EPOCH_BASE, dtype=torch.int32, device=dev)
    return _device_epoch[key]


class DecodeStack:
    """A stack of layers whose decode step is launched natively by prr_decode_step:
    the two-stream PRR schedule, the serial select-then-attend schedule, or the step-0
    select + EMA initialisation."""

    def __init__(self, layers: List[LayerState], queries, device):
        self.layers = layers
        self.cfg = layers[0].cfg
        self.dims = layers[0].dims
        cfg = self.cfg
        self.io = (L.prr_layer_io * len(layers))(*[st.io(q) for st, q in zip(layers, queries)])
        self.forced = (ctypes.c_int32 * max(1, len(cfg.forced)))(*cfg.forced)
        p = L.prr_step_params()
        p.num_tokens, p.num_pages, p.k_select = cfg.num_tokens, cfg.num_pages, cfg.k_select
        p.p_select = cfg.k_select if cfg.p_select is None else cfg.p_select
        p.cap, p.chunk_pages, p.mode = layers[0].cap, cfg.chunk_pages, cfg.mode
        p.forced_in_budget, p.n_forced = int(bool(cfg.forced_in_budget)), len(cfg.forced)
        p.forced = ctypes.cast(self.forced, ctypes.POINTER(ctypes.c_int32))
        p.alpha, p.beta, p.gamma = cfg.alpha, cfg.beta, cfg.gamma
        self.params = p
        self.events = L.hip_events(3 * len(layers) + 1)
        # the two-stream schedule's fork/join: the caller's events, or (False) the library's
        # stream-memory words
        self.two_stream_events = True

    def set_layer_theta(self, thetas):
        """Per-layer EMA parameters (Section 4.2 calibrates one per layer): a sequence of
        (alpha, beta, gamma) per layer, or None to use the step's for every layer."""
        for i, st in enumerate(self.layers):
            st.theta = None if thetas is None else np.asarray(thetas[i], dtype=np.float32).copy()
            self.io[i].theta = None if st.theta is None else st.theta.ctypes.data

    def set_tokens(self, num_tokens):
        """The sequence now holds num_tokens tokens (as many as the layers' pages hold): for the next steps of every
        layer.  Graphs that were captured keep the tokens of their capture."""
        if not 1 <= num_tokens <= self.dims.max_pages * self.dims.page_size:
            raise ValueError(f"{num_tokens} tokens: the layers hold 1 to {self.dims.max_pages * self.dims.page_size}")
        for st in self.layers:
            st.cfg.num_tokens = num_tokens
        cfg = self.layers[0].cfg
        self.params.num_tokens, self.params.num_pages = cfg.num_tokens, cfg.num_pages

    def _parity(self):
        parity = self.layers[0].cur
        assert all(st.cur == parity for st in self.layers), "layers disagree on the current prediction buffer"
        return parity

    def _advance(self, schedule, parity):
        if schedule not in (L.PRR_SCHED_SERIAL, L.PRR_SCHED_FUSED_SERIAL):
            for st in self.layers:
                st.cur = 1 - parity

    def step(self, schedule, stream, spec_stream=None):
        """One decode step of every layer; P^t is in each layer's predicted[cur]."""
        parity = self._parity()
        self.params.epoch = next_epoch()
        self.params.epoch_dev = None
        events = self.events if (schedule != L.PRR_SCHED_TWO_STREAM or self.two_stream_events) else None
        L.prr_decode_step(self.dims, self.params, self.io, parity, schedule, stream, spec_stream, events)
        self._advance(schedule, parity)

    def capture(self, schedule, stream, tag=None):
        """Capture one fused decode step of every layer as a HIP graph per parity of the
        prediction buffers: an advance of the device epoch word, then the layers' launches
        (which read it).  The step parameters are those of this moment; `tag` names the
        capture when several are kept for one schedule."""
        assert schedule in (L.PRR_SCHED_FUSED_SERIAL, L.PRR_SCHED_FUSED_PRR), "fused steps only"
        if not hasattr(self, "graphs"):
            self.graphs = {}
        ep = device_epoch(self.layers[0].k.device)
        self.params.epoch = 0
        self.params.epoch_dev = ep.data_ptr()
        for parity in (0, 1):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                L.prr_epoch_advance(ep, stream)
                L.prr_decode_step(self.dims, self.params, self.io, parity, schedule, stream, None, self.events)
            self.graphs[(schedule, tag, parity)] = g
        self.params.epoch_dev = None

    def replay(self, schedule, stream, tag=None):
        """One decode step of every layer by replaying the captured graph (see capture)."""
        parity = self._parity()
        with torch.cuda.stream(stream):
            self.graphs[(schedule, tag, parity)].replay()
        self._advance(schedule, parity)


class TwoStream:
    """Fork/join orchestration of one layer step on two HIP streams (default priority)."""

    def __init__(self, device):
        self.s = torch.cuda.Stream(device=device)
        self.p = torch.cuda.Stream(device=device)
        self._events = []

    def _ev(self):
        return torch.cuda.Event()

    def prr_layer(self, st: LayerState, q, mode=None):
        s, p = self.s, self.p
        fork = self._ev()
        fork.record(s)
        p.wait_event(fork)
        st.select(q, stream=s)
        sel = self._ev()
        sel.record(s)
        st.speculate(q, stream=p)
        spec = self._ev()
        spec.record(p)
        s.wait_event(spec)
        st.repair(q, stream=s, mode=mode)
        p.wait_event(sel)
        st.predict(stream=p)
        done = self._ev()
        done.record(p)
        return done

    def serial_layer(self, st: LayerState, q):
        st.select(q, stream=self.s)
        st.repair(q, stream=self.s, serial=True)

    def join(self, events: List[torch.cuda.Event]):
        for e in events:
            self.s.wait_event(e)
