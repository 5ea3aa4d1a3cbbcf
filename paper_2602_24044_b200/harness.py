"""Device-side harness around the C entry points: allocates the buffers a caller owns
(PyTorch tensors), fills a slot pool from a workload and runs applies.  Used by the GPU
tests, the smoke check and the benchmark.  No arithmetic of the method lives here.
"""
from __future__ import annotations

from typing import Dict, List, Optional, Sequence

import numpy as np
import torch

from . import binding as lb


def bf16_tensor(bits: np.ndarray, device=None, pin: bool = False) -> torch.Tensor:
    """numpy uint16 bf16 bit patterns -> torch.bfloat16 tensor (same bits)."""
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16)
    if pin:
        t = t.pin_memory()
    if device is not None:
        t = t.to(device, non_blocking=False)
    return t


def bf16_bits(t: torch.Tensor) -> np.ndarray:
    """torch.bfloat16 tensor -> numpy uint16 bit patterns (waits for all queued GPU work)."""
    if t.is_cuda:
        torch.cuda.synchronize(t.device)
    return t.detach().contiguous().cpu().view(torch.int16).numpy().view(np.uint16)


class Session:
    """A slot pool on one GPU filled from a workload, plus per-batch scratch buffers."""

    def __init__(self, wl, device: str = "cuda:0", targets: Optional[Sequence[int]] = None,
                 slots: Optional[Sequence[int]] = None, a_layout: int = lb.A_DIN_MAJOR,
                 T_cap: Optional[int] = None, tuning: Optional[Dict[int, int]] = None):
        """targets: the workload's target ids to materialise in the pool (default: all);
        slots: which occupied slots to load (default: every slot the workload marks loaded)."""
        self.wl = wl
        self.device = torch.device(device)
        self.dev_index = self.device.index or 0
        self.target_ids = list(range(len(wl.targets))) if targets is None else list(targets)
        self.pool_targets = [wl.targets[t] for t in self.target_ids]
        self.target_pos = {t: i for i, t in enumerate(self.target_ids)}
        torch.cuda.set_device(self.device)
        self.compute = torch.cuda.Stream(self.device)
        self.load = torch.cuda.Stream(self.device)
        nbytes = lb.pool_bytes(wl.num_slots, wl.r_max, self.pool_targets, self.dev_index)
        self.pool_buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        off = (-self.pool_buf.data_ptr()) % 256
        self.pool_mem = self.pool_buf[off:off + nbytes]
        self.pool = lb.pool_create(wl.num_slots, wl.r_max, self.pool_targets, self.pool_mem,
                                   self.dev_index)
        for key, value in (tuning or {}).items():
            lb.pool_set_tuning(self.pool, key, value)
        self.T_cap = int(T_cap if T_cap is not None else max(wl.T, 1))
        self.ws = torch.empty(lb.workspace_bytes(self.pool, self.T_cap), dtype=torch.uint8,
                              device=self.device)
        self.meta = None
        self.meta_shape = None
        self.slot_idx_dev = torch.from_numpy(np.ascontiguousarray(wl.slot_idx)).to(self.device)
        self.status_host = torch.zeros(4, dtype=torch.int32).pin_memory()
        self._pinned: List[torch.Tensor] = []
        want = [i for i in range(wl.num_slots) if wl.loaded[i]] if slots is None else list(slots)
        for s in want:
            self.load_slot(s, a_layout=a_layout)
        torch.cuda.synchronize(self.device)
        self._pinned.clear()

    # -- pool ----------------------------------------------------------------------------
    def host_adapter(self, slot: int, a_layout: int):
        """Pinned host matrices of one adapter for the pool's targets."""
        A, B = [], []
        for t in self.target_ids:
            a, b = self.wl.adapter_weights(slot, t)
            if a_layout == lb.A_RANK_MAJOR:
                a = np.ascontiguousarray(a.T)
            A.append(bf16_tensor(a, pin=True))
            B.append(bf16_tensor(b, pin=True))
        return A, B

    def host_adapter_packed(self, slot: int):
        """One pinned buffer with every target's A [rank, d_in] and B [rank, d_out] in order."""
        parts = []
        for t in self.target_ids:
            a, b = self.wl.adapter_weights(slot, t)
            parts += [np.ascontiguousarray(a.T).ravel(), np.ascontiguousarray(b).ravel()]
        buf = bf16_tensor(np.concatenate(parts), pin=True)
        return [buf] * len(self.target_ids), [buf] * len(self.target_ids)

    def load_slot(self, slot: int, a_layout: int = lb.A_DIN_MAJOR, src_slot: Optional[int] = None,
                  rank: Optional[int] = None, scale: Optional[float] = None, blobs=None):
        """Queue a swap-in of the workload's adapter `src_slot` (default: `slot`) into `slot`."""
        src = slot if src_slot is None else src_slot
        if blobs is not None:
            A, B = blobs
        elif a_layout == lb.PACKED:
            A, B = self.host_adapter_packed(src)
        else:
            A, B = self.host_adapter(src, a_layout)
        self._pinned += A + B
        lb.pool_load_slot(self.pool, slot, int(self.wl.ranks[src]) if rank is None else rank,
                          float(self.wl.scales[src]) if scale is None else scale, A, B, a_layout,
                          self.load, self.compute)

    def read_slot(self, slot: int, target: int):
        d_in, d_out = self.wl.targets[target]
        A = torch.empty((self.wl.r_max, d_in), dtype=torch.bfloat16).pin_memory()
        B = torch.empty((self.wl.r_max, d_out), dtype=torch.bfloat16).pin_memory()
        lb.pool_read_slot(self.pool, slot, self.target_pos[target], A, B, self.compute)
        self.compute.synchronize()
        return bf16_bits(A), bf16_bits(B)

    def status(self) -> np.ndarray:
        lb.pool_poll_status(self.pool, self.status_host, self.compute)
        self.compute.synchronize()
        return self.status_host.numpy().copy()

    # -- metadata ------------------------------------------------------------------------
    def build_segments(self, tile_m: Optional[int] = None, long_min: Optional[int] = None,
                       slot_idx_dev: Optional[torch.Tensor] = None):
        wl = self.wl
        tile_m = wl.tile_m if tile_m is None else tile_m
        long_min = wl.long_min if long_min is None else long_min
        sidx = self.slot_idx_dev if slot_idx_dev is None else slot_idx_dev
        T = int(sidx.shape[0])
        nbytes = lb.segments_bytes(T, wl.num_slots, tile_m)
        if self.meta is None or self.meta.numel() * 4 < nbytes:
            self.meta = torch.empty((nbytes + 3) // 4, dtype=torch.int32, device=self.device)
        lb.build_segments(self.pool, sidx, T, tile_m, long_min, self.meta, stream=self.compute)
        self.meta_shape = (T, tile_m)
        return self.meta

    def segments_host(self) -> Dict[str, np.ndarray]:
        self.compute.synchronize()
        T, tile_m = self.meta_shape
        return lb.unpack_segments(self.meta.cpu().numpy(), T, self.wl.num_slots, tile_m)

    # -- the forward ---------------------------------------------------------------------
    def apply(self, call: int = 0, x: Optional[torch.Tensor] = None,
              y_base: Optional[torch.Tensor] = None, *, kind: Optional[str] = None,
              grouped: bool = True, in_place: bool = False,
              slot_idx_dev: Optional[torch.Tensor] = None, rebuild: bool = True,
              ws_bytes: Optional[int] = None) -> torch.Tensor:
        """One apply on the compute stream; returns y (device tensor).  x / y_base default to
        the workload's activations for `call`.  ws_bytes: how much of the workspace the call is
        told about (default: all of it)."""
        wl = self.wl
        target = wl.calls[call]
        d_in, d_out = wl.targets[target]
        if x is None:
            x_h, yb_h = wl.activations(call)
            x, y_base = bf16_tensor(x_h, self.device), bf16_tensor(yb_h, self.device)
        T = int(x.shape[0])
        kind = wl.kind if kind is None else kind
        sidx = self.slot_idx_dev if slot_idx_dev is None else slot_idx_dev
        y = y_base if in_place else torch.empty_like(y_base)
        with torch.cuda.stream(self.compute):
            if not in_place:
                # a row the kernels never write must not pass for a result left over in recycled
                # memory: the output starts as a huge finite value in every element
                y.view(torch.int16).fill_(0x7F7F)
            meta = None
            if grouped or kind == "sgmv":
                if rebuild or self.meta_shape is None:
                    self.build_segments(slot_idx_dev=sidx)
                meta = self.meta
            tp = self.target_pos[target]
            if kind == "bgmv":
                lb.bgmv_apply(self.pool, tp, x, x.stride(0), y_base, y_base.stride(0), y,
                              y.stride(0), sidx, T, meta, self.ws, stream=self.compute)
            else:
                lb.sgmv_apply(self.pool, tp, x, x.stride(0), y_base, y_base.stride(0), y,
                              y.stride(0), meta, T, self.ws, ws_bytes, stream=self.compute)
        return y

    def close(self):
        if self.pool:
            torch.cuda.synchronize(self.device)
            lb.pool_destroy(self.pool)
            self.pool = 0

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


def media_spans(requests: Sequence[Sequence]):
    """The images and videos of requests as kv_axis_positions takes them: for each request a list of (first
    token, frames, rows, columns[, step of a frame]), ascending by their first tokens.  Returns int32 arrays
    (spans [n, 8], span_begin [requests + 1])."""
    spans, begin = [], [0]
    for r, mine in enumerate(requests):
        end = at = 0                      # tokens so far, and the position of the next one
        for first, frames, rows, columns, *step in mine:
            step = step[0] if step else 1
            if first < end or min(frames, rows, columns) < 1 or step < 0:
                raise ValueError("media_spans: request %d: a span at token %d overlaps the one before it, or is empty"
                                 % (r, first))
            at += first - end
            spans.append((first, frames, rows, columns, at, step, 0, 0))
            end = first + frames * rows * columns
            at += max((frames - 1) * step + 1, rows, columns)
        begin.append(len(spans))
    return np.array(spans, dtype=np.int32).reshape(-1, 8), np.array(begin, dtype=np.int32)


class KVCache:
    """A paged 4-bit key/value cache on one GPU with the table buffer and workspace of its calls.

    The caller keeps the requests' state (lengths, block table, stack of free pages) as int32 device
    tensors; build_tables() advances it for one batch, then append() and attention() run per layer on
    the tables it left.

    stream: as for the entry points (None is the device's default stream).  Calls on several streams are
    the caller's to order; the cache sees to it that its own buffers are not given back to the allocator
    while work on any stream it was called on is pending.  Tables that grow move: a captured graph keeps
    the old ones, so reserve() for the largest batch before a capture."""

    def __init__(self, num_layers: int, num_pages: int, page_size: int, num_q_heads: int, num_kv_heads: int,
                 head_dim: int, device: int = 0):
        self.device = torch.device("cuda", int(device))
        self._index = int(device)
        self.shape = (num_layers, num_pages, page_size, num_q_heads, num_kv_heads, head_dim)
        self._width = num_q_heads * head_dim
        self._streams = set()            # handles of torch's streams that work on the buffers was queued on
        self._others = False             # and was some on a stream that is not torch's, and may be gone by now?
        nbytes = lb.kv_bytes(*self.shape, device=int(device))
        self.buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        off = (-self.buf.data_ptr()) % 256
        self.mem = self.buf[off:off + nbytes]
        self.kv = lb.kv_create(*self.shape, self.mem, device=int(device))
        self.workspace = torch.empty(lb.kv_workspace_bytes(self.kv), dtype=torch.uint8, device=self.device)
        self._workspace_bytes = self.workspace.numel()
        self.tables, self._tables_bytes = None, 0
        self.slots = self.block_table = None
        self.R = self.T = -1

    def _on(self, stream) -> int:
        """The stream's handle, noted as one that may have work on the buffers."""
        handle = 0 if stream is None else lb.stream_handle(stream)
        if handle not in self._streams:
            if handle and (type(stream) is int or isinstance(stream, torch.cuda.ExternalStream)):
                self._others = True
            else:
                self._streams.add(handle)
        return handle

    def _torch_stream(self, handle: int):
        return torch.cuda.ExternalStream(handle, self.device) if handle else torch.cuda.default_stream(self.device)

    def _let_go(self, *tensors) -> None:
        """Before tensors are dropped: their memory may be handed out once the work queued so far is done."""
        if self._others:
            torch.cuda.synchronize(self.device)
            return
        for handle in self._streams:
            stream = self._torch_stream(handle)
            for t in tensors:
                if t is not None:
                    t.record_stream(stream)

    # -- checks: what the kernels would read or write past a tensor's end, or as another type --------------
    def _ints(self, what: str, t, n: int) -> None:
        if t.dtype is not torch.int32 or t.numel() < n or t.get_device() != self._index or not t.is_contiguous():
            raise ValueError("%s: needs %d int32 in a row on %s" % (what, n, self.device))

    def _rows(self, what: str, t, n: int, width: int) -> int:
        """The leading dimension of n bf16 rows of `width` values (in one or several dimensions)."""
        shape = t.shape
        if t.dtype is torch.bfloat16 and t.get_device() == self._index and len(shape) >= 2 and shape[0] >= n:
            if len(shape) == 2 and shape[1] >= width and t.is_contiguous():
                return shape[1]
            strides, have = t.stride(), 1
            for i in range(len(shape) - 1, 0, -1):
                if strides[i] != have and shape[i] != 1:
                    have = 0
                    break
                have *= shape[i]
            if have >= width:
                return strides[0] if shape[0] > 1 else max(strides[0], have)
        raise ValueError("%s: needs %d bf16 rows of %d values, each in a row, on %s" % (what, n, width, self.device))

    def _table(self, t, R: int) -> int:
        """The leading dimension of a block table, which is also the pages that a request may have."""
        shape = t.shape
        if t.dtype is torch.int32 and t.get_device() == self._index and len(shape) == 2 and shape[0] == R:
            cols = shape[1]
            if t.is_contiguous():
                return cols
            ld, step = t.stride()
            if R == 1 and ld < cols:
                ld = cols
            # rows that are wider than the table: to their ends they have to lie in its memory
            if (cols <= 1 or step == 1) and (ld == cols or (
                    ld > cols and t.storage_offset() + R * ld <= t.untyped_storage().nbytes() // 4)):
                return ld
        raise ValueError("block_table: needs %d rows of int32 pages, each in a row, on %s" % (R, self.device))

    def layer(self, layer: int) -> torch.Tensor:
        """One layer's pages as bytes (a view)."""
        off, n = lb.kv_layer_range(layer, *self.shape, device=self.device.index)
        return self.mem[off:off + n]

    def reserve(self, R: int, T: int) -> None:
        """Makes room for the tables of a batch of R requests and T new tokens, ready for calls on any stream."""
        here = torch.cuda.current_stream(self.device)
        if self._room(R, T, here) and not torch.cuda.is_current_stream_capturing():
            here.synchronize()           # recycled memory is free in the order of the stream it was taken on

    def _room(self, R: int, T: int, stream) -> bool:
        """Room for a batch's tables, taken on `stream` (a torch stream); True when they moved."""
        words = lb.kv_tables_bytes(self.kv, R, T) // 4
        grow = self.tables is None or self.tables.numel() < words
        if grow:
            if self.tables is not None:
                self._let_go(self.tables)
            with torch.cuda.stream(stream):
                self.tables = torch.empty(words, dtype=torch.int32, device=self.device)
            self._tables_bytes = 4 * words
            self.R = -1
        if (R, T) != (self.R, self.T):
            self.R, self.T = R, T
            v = lb.kv_table_views(self.tables, R, T)
            self.header, self.starts, self.lengths = v["header"], v["start"], v["kv_len"]
            self.positions, self.slots = v["position"], v["slot"]
        return grow

    def build_tables(self, kv_len, q_len, T: int, free_pages, free_count, block_table, *, max_q: int = 0,
                     window: int = 0, kv_len_out=None, free_count_out=None, stream=None) -> None:
        """Tables of a batch; kv_len and free_count are advanced in place unless *_out names other
        tensors."""
        R = kv_len.shape[0]
        if q_len.shape[0] != R:
            raise ValueError("q_len needs one entry per request (%d)" % R)
        # (as _ints, written out: the time of this call is the host's.  Lengths have their R by their shape)
        index, int32 = self._index, torch.int32
        if (kv_len.dtype is not int32 or kv_len.get_device() != index or not kv_len.is_contiguous() or
                q_len.dtype is not int32 or q_len.get_device() != index or not q_len.is_contiguous()):
            self._ints("kv_len", kv_len, R), self._ints("q_len", q_len, R)
        if (free_pages.dtype is not int32 or free_pages.get_device() != index or not free_pages.is_contiguous() or
                free_count.dtype is not int32 or free_count.get_device() != index or free_count.numel() < 1):
            self._ints("free_pages", free_pages, 0), self._ints("free_count", free_count, 1)
        if kv_len_out is None:
            kv_len_out = kv_len
        elif (kv_len_out.dtype is not int32 or kv_len_out.get_device() != index or kv_len_out.numel() < R or
              not kv_len_out.is_contiguous()):
            self._ints("kv_len_out", kv_len_out, R)
        if free_count_out is None:
            free_count_out = free_count
        elif free_count_out.dtype is not int32 or free_count_out.get_device() != index or free_count_out.numel() < 1:
            self._ints("free_count_out", free_count_out, 1)
        ld_table = self._table(block_table, R)
        stream = self._on(stream)
        if R != self.R or T != self.T:
            self._room(R, T, self._torch_stream(stream))
        self.block_table, self.ld_table = block_table, ld_table
        lb.kv_build_tables(self.kv, kv_len, q_len, R, T, free_pages, free_count, block_table, self.ld_table,
                           self.tables, max_q=max_q, window=window,
                           kv_len_out=kv_len_out, free_count_out=free_count_out,
                           tables_bytes=self._tables_bytes, stream=stream)

    def release(self, requests, kv_len, block_table, free_pages, free_count, stream=None) -> None:
        """free_pages: room for every page of the cache."""
        n, R = int(requests.shape[0]), int(kv_len.shape[0])
        self._ints("requests", requests, n)
        self._ints("kv_len", kv_len, R)
        self._ints("free_pages", free_pages, self.shape[1])
        self._ints("free_count", free_count, 1)
        lb.kv_release(self.kv, requests, n, R, kv_len, block_table, self._table(block_table, R), free_pages,
                      free_count, stream=self._on(stream))

    def axis_positions(self, spans, span_begin, out, stream=None) -> None:
        """Positions on three axes of the tables' tokens; spans, span_begin: as media_spans returns them, on the
        device; out: int32 [3, tokens]."""
        R, T = self.R, self.T
        if self.block_table is None:
            raise ValueError("axis_positions: no tables have been built")
        # (as _ints, written out: the time of this call is the host's)
        index, int32, have, shape = self._index, torch.int32, spans.shape, out.shape
        if (spans.dtype is not int32 or spans.get_device() != index or not spans.is_contiguous() or len(have) != 2 or
                have[1] != 8):
            raise ValueError("spans: needs rows of 8 int32 in a row on %s" % self.device)
        if (span_begin.dtype is not int32 or span_begin.numel() < R + 1 or span_begin.get_device() != index or
                not span_begin.is_contiguous()):
            self._ints("span_begin", span_begin, R + 1)
        ld = out.stride(0) if len(shape) == 2 else 0
        if (out.dtype is not int32 or out.get_device() != index or ld < T or shape[0] < 3 or shape[1] < T or
                not (out.is_contiguous() or out.stride(1) == 1)):
            raise ValueError("out: needs int32 [3, %d], each axis in a row, on %s" % (T, self.device))
        lb.kv_axis_positions(self.kv, self.tables, R, T, spans, span_begin, have[0], out, ld, stream=self._on(stream))

    def append(self, layer: int, args, slots=None, T: Optional[int] = None, stream=None) -> None:
        """args: binding.qk_args(...); slots: default those of the tables."""
        slots, T = self.slots if slots is None else slots, self.T if T is None else T
        if slots is None:
            raise ValueError("append: no slots, and no tables have been built")
        self._ints("slots", slots, T)
        lb.kv_append(self.kv, layer, args, slots, T, stream=self._on(stream))

    def read(self, layer: int, slots, k_out, v_out, stream=None) -> None:
        n, width = int(slots.shape[0]), self.shape[4] * self.shape[5]
        self._ints("slots", slots, n)
        lb.kv_read(self.kv, layer, slots, n, k_out, 0 if k_out is None else self._rows("k_out", k_out, n, width),
                   v_out, 0 if v_out is None else self._rows("v_out", v_out, n, width), stream=self._on(stream))

    def attention(self, layer: int, q, out, *, scale: float, lse=None, stream=None) -> None:
        """q, out: rows of num_q_heads * head_dim values, one per new token of the tables; lse: fp32 in a row."""
        T, width = self.T, self._width
        if self.block_table is None:
            raise ValueError("attention: no tables have been built")
        shape = q.shape
        if (shape == (T, width) and out.shape == shape and q.dtype is torch.bfloat16 and out.dtype is torch.bfloat16 and
                q.get_device() == out.get_device() == self._index and q.is_contiguous() and out.is_contiguous()):
            ldq = ldo = width        # the usual case without a call each: a small batch's time is the host's
        else:
            ldq, ldo = self._rows("q", q, T, width), self._rows("out", out, T, width)
        if lse is not None and (lse.dtype is not torch.float32 or lse.numel() < T * self.shape[3] or
                                not lse.is_contiguous() or lse.get_device() != self._index):
            raise ValueError("lse: needs %d x %d fp32 in a row on %s" % (T, self.shape[3], self.device))
        lb.kv_attention(self.kv, layer, q, ldq, out, ldo, lse, scale, self.tables, self.R, T, self.block_table,
                        self.ld_table, self.workspace, self._workspace_bytes, stream=self._on(stream))

    def status(self, stream=None):
        return lb.kv_check_status(self.kv, stream)

    def close(self):
        if self.kv:
            torch.cuda.synchronize(self.device)
            lb.kv_destroy(self.kv)
            self.kv = 0

    def __del__(self):   # the handle holds host memory only; the buffers are torch's to free
        try:
            if getattr(self, "kv", 0):
                self._let_go(self.buf, self.workspace, self.tables)
                lb.kv_destroy(self.kv)
        except (TypeError, AttributeError, RuntimeError):   # the interpreter is taking its modules down
            pass
        self.kv = 0

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()
