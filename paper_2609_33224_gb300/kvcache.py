"""The serving operators (include/packserve_kv.h) for torch: the paged key/value cache in the scheduler's
16-token blocks, and attention of a batch over it.

``KVCache`` holds the keys and values of one layer: ``write`` stores new tokens (rounding them to the
cache's format), ``read`` gives back what the cache holds, ``attend`` computes attention of a batch that an
``AttentionPlan`` describes.  All three run on torch's current stream of the cache's device and return
without waiting for it; what a kernel finds wrong raises ``PSError`` from the next call, or from ``check``.  They are
operators of serving: no gradient goes through them, and their results are not part of autograd's graph.
"""
from __future__ import annotations

import ctypes
import struct
import weakref

import numpy as np
import torch

from . import PS_ERR_STATE, PS_OK, PSError, PsKvConfig, PsKvRows, lib

FORMATS = {"bf16": 0, "fp16": 1, "fp8": 2}
_TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 3}
BLOCK_TOKENS = 16
_ROWS = struct.Struct("@Pqqi4x")  # ps_kv_rows
assert _ROWS.size == ctypes.sizeof(PsKvRows)
_stream = torch._C._cuda_getCurrentRawStream  # torch's current stream of a device, as a number


def _capturing(device: int) -> bool:
    """Whether torch's current stream of the device, which need not be the current one, is captured into a graph."""
    if torch._C._cuda_getDevice() == device:
        return torch.cuda.is_current_stream_capturing()
    with torch.cuda.device(device):
        return torch.cuda.is_current_stream_capturing()


# ps_kv_span: a run of cached tokens (their blocks start at first_block of the plan's block array) and the
# queries that see it; causal: the last num_queries tokens are the queries' own
SPAN_DTYPE = np.dtype([("first_query", np.uint32), ("num_queries", np.uint32), ("length", np.uint64),
                       ("causal", np.uint32), ("first_block", np.uint64)], align=True)


class KVCache:
    """``num_blocks`` blocks of 16 tokens x ``kv_heads`` x ``head_dim`` (64 or 128) keys and values.

    ``fmt``: "bf16", "fp16", or "fp8" (e4m3 with a power-of-two scale per token and head).  Token t of block b
    has slot ``16 * b + t``.  Without ``device``, torch's current one.
    """

    def __init__(self, num_blocks: int, kv_heads: int, head_dim: int, fmt: str = "bf16", device: int | None = None):
        if fmt not in FORMATS:
            raise ValueError(f"fmt must be one of {', '.join(FORMATS)}")
        self.device = torch.cuda.current_device() if device is None else int(device)
        self.num_blocks, self.kv_heads, self.head_dim, self.fmt = int(num_blocks), int(kv_heads), int(head_dim), fmt
        self.dtype = torch.float16 if fmt == "fp16" else torch.bfloat16  # of the queries and the output
        if not (0 < self.num_blocks < 1 << 32 and 0 < self.kv_heads <= 1024 and self.head_dim in (64, 128)):
            raise ValueError("num_blocks must be in 1..2^32-1, kv_heads in 1..1024, head_dim 64 or 128")
        cfg = PsKvConfig(self.device, self.kv_heads, self.num_blocks, self.head_dim, FORMATS[fmt])
        h = ctypes.c_void_p()
        s = lib().ps_kv_create(ctypes.byref(cfg), ctypes.byref(h))
        if s != PS_OK:
            raise PSError(s, "ps_kv_create failed (invalid configuration or device allocation)")
        self._h = h
        self._lib = lib()
        self._plans = weakref.WeakSet()
        self._device = torch.device("cuda", self.device)
        self._args = (ctypes.c_char * (2 * _ROWS.size))()
        self._arg0 = ctypes.addressof(self._args)
        self._arg1 = self._arg0 + _ROWS.size

    def _check(self, s: int):
        if s != PS_OK:
            raise PSError(s, self._lib.ps_kv_last_error(self._h).decode())

    def close(self):
        """Release the cache's memory, and the plans made for it.  What a CUDA graph's captured calls read is kept for the
        graph, and freed with the next cache or plan made or closed after it."""
        if getattr(self, "_h", None):
            for p in list(self._plans):
                p.close()
            self._lib.ps_kv_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    def _open(self):
        if not self._h:
            raise ValueError("the cache is closed")
        return self._h

    # The calls below are made once per layer and step, and a small one's kernel takes no longer than its call:
    # descriptors are packed into one buffer of the cache, and tensors are asked for nothing twice.
    def _rows(self, at: int, x, name: str, n: int, heads: int):
        """Packs x's ps_kv_rows at slot ``at`` of the cache's buffer."""
        t = _TYPES.get(x.dtype)
        st = x.stride()
        if x.get_device() != self.device or t is None or x.shape != (n, heads, self.head_dim) or st[2] != 1:
            if x.get_device() != self.device:
                raise ValueError(f"{name} must be a tensor on cuda:{self.device}")
            if t is None:
                raise ValueError(f"{name} must be bfloat16, float16 or float32, not {x.dtype}")
            if tuple(x.shape) != (n, heads, self.head_dim):
                raise ValueError(f"{name} must have shape {(n, heads, self.head_dim)}, not {tuple(x.shape)}")
            raise ValueError(f"{name}'s head_dim elements must lie next to each other")
        _ROWS.pack_into(self._args, at, x.data_ptr(), st[0], st[1], t)

    def _out(self, at: int, x, name: str, n: int, heads: int, dtype):
        """Packs the result tensor x, or a new one of ``dtype``."""
        if x is not None:
            if dtype is not None and x.dtype != dtype:
                raise ValueError(f"{name} is not of the dtype asked for")
            self._rows(at, x, name, n, heads)
            return x
        dtype = dtype or self.dtype
        t = _TYPES.get(dtype)
        if t is None:
            raise ValueError(f"dtype must be bfloat16, float16 or float32, not {dtype}")
        x = torch.empty((n, heads, self.head_dim), dtype=dtype, device=self._device)
        _ROWS.pack_into(self._args, at, x.data_ptr(), heads * self.head_dim, self.head_dim, t)
        return x

    def _slots(self, slots) -> int:
        if slots.dtype != torch.int64 or slots.dim() != 1 or slots.get_device() != self.device or \
                not slots.is_contiguous():
            raise ValueError(f"slots must be a contiguous int64 vector on cuda:{self.device}")
        return slots.shape[0]

    def write(self, k, v, slots):
        """Store row t of k and v ([T, kv_heads, head_dim]) at slot ``slots[t]`` (int64; negative: skipped)."""
        h, n = self._open(), self._slots(slots)
        self._rows(0, k, "k", n, self.kv_heads)
        self._rows(_ROWS.size, v, "v", n, self.kv_heads)
        s = self._lib.ps_kv_write(h, self._arg0, self._arg1, slots.data_ptr(), n, _stream(self.device))
        if s:
            self._check(s)

    def read(self, slots, dtype=None, k=None, v=None):
        """The cached keys and values at ``slots``, as (k, v) of ``dtype`` (default: ``self.dtype``) or in the
        tensors given; a negative slot gives zeros."""
        h, n = self._open(), self._slots(slots)
        k = self._out(0, k, "k", n, self.kv_heads, dtype)
        v = self._out(_ROWS.size, v, "v", n, self.kv_heads, dtype)
        s = self._lib.ps_kv_read(h, slots.data_ptr(), n, self._arg0, self._arg1, _stream(self.device))
        if s:
            self._check(s)
        return k, v

    def attend(self, q, plan: "AttentionPlan", scale: float | None = None, out=None, lse=None):
        """Attention of the plan's batch: q [queries, q_heads, head_dim] of ``self.dtype`` -> out of the same shape.

        ``scale`` defaults to head_dim ** -0.5; ``lse``, a contiguous float32 [queries, q_heads] tensor, receives
        the logarithms of the softmax sums (-inf where a query sees no key; its output is zero).
        """
        h, p = self._open(), plan._open()
        n, heads = plan.num_queries, plan.q_heads
        self._rows(0, q, "q", n, heads)
        out = self._out(_ROWS.size, out, "out", n, heads, None if out is not None else q.dtype)
        if lse is not None and (lse.dtype != torch.float32 or lse.device != q.device or not lse.is_contiguous() or
                                tuple(lse.shape) != (n, heads)):
            raise ValueError(f"lse must be a contiguous float32 tensor of shape {(n, heads)} on q's device")
        stream = _stream(self.device)
        nb = plan.workspace_bytes
        ws = plan._workspace(stream, nb) if nb else None
        s = self._lib.ps_kv_attend(h, p, self._arg0, self._arg1, None if lse is None else lse.data_ptr(),
                                   self.head_dim ** -0.5 if scale is None else scale,
                                   None if ws is None else ws.data_ptr(), nb, stream)
        if s:
            self._check(s)
        return out

    def check(self):
        """Wait for the current stream and raise what kernels have reported since the last report."""
        self._check(self._lib.ps_kv_check(self._open(), _stream(self.device)))


class AttentionPlan:
    """The spans of a batch for ``KVCache.attend``: set once per step, used by every layer's call of it.

    ``set(num_queries, spans, blocks)``: ``spans`` is an array of ``SPAN_DTYPE`` (or rows of its five fields),
    ``blocks`` the uint32 block ids that they index.  A prefix shared by a range of queries is one span over
    all of them, a request's own tokens a (causal) span of its own.  ``set`` works on the host (27 us for one request,
    0.1 ms for 256 on a prefix, 2.5 ms for 8192 new tokens of 64 heads) and waits for its copy to the device.  While a
    CUDA graph holds a captured call on the plan, ``set`` is refused and the plan stays as it is.
    """

    def __init__(self, cache: KVCache, q_heads: int, max_queries: int, max_spans: int, max_blocks: int):
        h = ctypes.c_void_p()
        limits = [int(x) for x in (q_heads, max_queries, max_spans, max_blocks)]
        if min(limits) < 0 or max(limits) >= 1 << 32:
            raise ValueError("q_heads and the limits must be in 0..2^32-1")
        self.cache, self.q_heads, self.num_queries, self.workspace_bytes = cache, limits[0], 0, 0
        cache._check(cache._lib.ps_kv_plan_create(cache._open(), *limits, ctypes.byref(h)))
        self._h = h
        self._spaces = {}  # workspace by stream: a stream's calls run one after the other
        cache._plans.add(self)

    def _open(self):
        if not self._h:
            raise ValueError("the plan is closed")
        return self._h

    def _workspace(self, stream: int, nbytes: int):
        if _capturing(self.cache.device):  # a graph's own: it may run beside other calls
            return torch.empty(nbytes, dtype=torch.uint8, device=self.cache._device)
        ws = self._spaces.get(stream)
        if ws is None or ws.numel() < nbytes:
            # a quarter more than asked for: the next steps' batches grow
            ws = self._spaces[stream] = torch.empty(nbytes + nbytes // 4, dtype=torch.uint8, device=self.cache._device)
        return ws

    def set(self, num_queries: int, spans, blocks):
        L, h = self.cache._lib, self._open()
        if not (isinstance(spans, np.ndarray) and spans.dtype == SPAN_DTYPE):
            rows = [tuple(int(x) for x in r) for r in spans]
            if any(len(r) != 5 or min(r) < 0 or max(r[0], r[1], r[3]) >= 1 << 32 for r in rows):
                raise ValueError("a span is (first_query, num_queries, length, causal, first_block), none negative")
            spans = np.array(rows, SPAN_DTYPE)
        spans = np.ascontiguousarray(spans)
        b = np.asarray(blocks)
        if b.ndim != 1 or spans.ndim != 1:
            raise ValueError("spans and blocks are one-dimensional")
        if b.dtype != np.uint32:
            if b.size and (b.dtype.kind not in "iu" or int(b.min()) < 0 or int(b.max()) >= 1 << 32):
                raise ValueError("block ids must be whole numbers in 0..2^32-1")
            b = b.astype(np.uint32)
        b = np.ascontiguousarray(b)
        if not 0 <= int(num_queries) < 1 << 32:
            raise ValueError("num_queries must be in 0..2^32-1")
        s = L.ps_kv_plan_set(h, int(num_queries), spans.ctypes.data if spans.size else None, spans.size,
                             b.ctypes.data if b.size else None, b.size)
        if s != PS_ERR_STATE:  # a plan that a CUDA graph holds stays as it is
            self.num_queries = self.workspace_bytes = 0
        self.cache._check(s)
        n = ctypes.c_uint64()
        self.cache._check(L.ps_kv_plan_workspace(h, ctypes.byref(n)))
        self.num_queries, self.workspace_bytes = int(num_queries), n.value

    def close(self):
        if getattr(self, "_h", None):
            self.cache._lib.ps_kv_plan_destroy(self._h)
            self._h = None
            self._spaces = {}

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def shared_spans(tables, lengths, new_tokens, min_blocks: int = 4):
    """The spans of a batch whose requests hold block tables with common beginnings.

    ``tables[i]``: the block ids of request i's tokens, in order; ``lengths[i]``: its tokens, the last
    ``new_tokens[i]`` of which (at least one) are its queries.  Blocks that hold no query's token and that several
    requests have in common from the start become one span for all of them, level by level as the tables part;
    runs of fewer than ``min_blocks`` common blocks stay with their requests.  Returns ``(order, spans, blocks)``:
    the batch has request ``order[0]``'s queries first, then ``order[1]``'s, and so on; ``spans`` and ``blocks`` are
    what ``AttentionPlan.set`` takes.
    """
    tabs = [np.ascontiguousarray(t, dtype=np.uint32) for t in tables]
    lengths, new = [int(x) for x in lengths], [int(x) for x in new_tokens]
    if not len(tabs) == len(lengths) == len(new):
        raise ValueError("one table, length and number of new tokens per request")
    for t, n, q in zip(tabs, lengths, new):
        if t.ndim != 1 or not 1 <= q <= n or n > BLOCK_TOKENS * t.size:
            raise ValueError("a request needs 1 <= new tokens <= length <= its blocks' tokens")
    full = [(n - q) // BLOCK_TOKENS for n, q in zip(lengths, new)]  # blocks without a query's token
    order = sorted(range(len(tabs)), key=lambda i: tabs[i][:full[i]].astype(">u4").tobytes())
    first = np.concatenate([[0], np.cumsum([new[i] for i in order])]).astype(np.int64) if order else np.zeros(1, np.int64)
    spans, blocks, at = [], [], 0

    def add(lo, hi, ids, length, causal):
        nonlocal at
        spans.append((first[lo], first[hi] - first[lo], length, causal, at))
        blocks.append(ids)
        at += ids.size

    def common(lo, hi):  # of a sorted run: what its ends have in common
        a, b = (tabs[order[x]][:full[order[x]]] for x in (lo, hi - 1))
        n = min(a.size, b.size)
        diff = np.flatnonzero(a[:n] != b[:n])
        return int(diff[0]) if diff.size else n

    todo = [(0, len(order), 0)] if order else []
    while todo:
        lo, hi, depth = todo.pop()
        if hi - lo == 1:
            i = order[lo]
            add(lo, hi, tabs[i][depth:-(-lengths[i] // BLOCK_TOKENS)], lengths[i] - depth * BLOCK_TOKENS, 1)
            continue
        n = common(lo, hi)
        if n - depth >= min_blocks:
            add(lo, hi, tabs[order[lo]][depth:n], (n - depth) * BLOCK_TOKENS, 0)
            depth = n
        # runs that go on together; a request whose table ends here goes on alone
        start = lo
        for x in range(lo + 1, hi + 1):
            i, j = order[start], order[x] if x < hi else -1
            if x < hi and full[i] > n and full[j] > n and tabs[i][n] == tabs[j][n]:
                continue
            todo.append((start, x, depth))
            start = x
    return (np.array(order, np.int64), np.array(spans, SPAN_DTYPE) if spans else np.zeros(0, SPAN_DTYPE),
            np.concatenate(blocks).astype(np.uint32) if blocks else np.zeros(0, np.uint32))
