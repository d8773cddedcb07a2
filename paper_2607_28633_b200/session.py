"""One request batch's pipelined transfer, both ends, on top of the C-ABI calls.

``TransferSender`` is what a prefill worker runs: after every layer's event it ships that
layer's slab to pinned host memory with the checksummed host leg, and at the end it emits one
128-byte header per request (§3.4). ``TransferReceiver`` is the decode side: it places every
layer from the host slab into its own paged pool, checksumming as it goes, and checks the
headers when the last layer is in; a mismatch is reported per request so that the caller can
retry (§3.1). ``DecodeCache`` is what the decode side does next with the pool it has received:
it gives new tokens their pages, writes their K/V, attends to the cache, forks and frees
requests and compacts the pool. All of them only enqueue work on the streams they are given,
library calls and, for the bookkeeping of new tokens, a few small tensor operations: no pack /
unpack arithmetic happens in Python, and nothing here touches the CPU oracle.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

import numpy as np
import torch

from . import binding as tk


@dataclass
class Endpoint:
    """Device-side description of one end: pool, layout, tables (device tensors)."""
    pool: torch.Tensor
    layout: tk.topkv_layout
    block_table: torch.Tensor
    seq_lens: torch.Tensor
    total_tokens: int

    def __post_init__(self):
        dev = self.pool.device
        R = int(self.seq_lens.shape[0])
        self.cu = torch.zeros(R + 1, dtype=torch.int64, device=dev)
        tk.check(tk.topkv_build_plan(tk.make_batch(self.block_table, self.seq_lens), self.cu,
                                     torch.cuda.current_stream(dev)))
        self.batch = tk.make_batch(self.block_table, self.seq_lens, self.total_tokens, self.cu)
        self.n_layer = tk.topkv_wire_layer_bytes(self.layout, self.total_tokens)
        self.ws_bytes = tk.check(tk.topkv_crc_workspace_bytes(
            self.layout, R, int(self.block_table.shape[1])))
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=dev)
        # two staging slabs: consecutive layers alternate between two streams, so that the copy
        # engine moves layer l while the kernel of layer l + 1 runs
        self.stagings = [torch.empty(max(self.n_layer, 16), dtype=torch.uint8, device=dev)
                         for _ in range(2)]
        self.crc = torch.zeros(R * self.layout.kv_factor, dtype=torch.int64, device=dev)
        torch.cuda.current_stream(dev).synchronize()

    @property
    def num_requests(self) -> int:
        return int(self.seq_lens.shape[0])

    def _checksums(self, stream) -> np.ndarray:
        tk.check(tk.topkv_crc_finish(self.layout, self.batch, self.workspace, self.ws_bytes,
                                     self.crc, stream))
        stream.synchronize()
        return self.crc.cpu().numpy().view(np.uint64).reshape(self.num_requests,
                                                              self.layout.kv_factor)


class TransferSender(Endpoint):
    """Ships layers to ``h_wire`` (pinned, ``L`` slabs of ``n_layer`` bytes, layer-major)."""

    def begin(self, stream):
        tk.check(tk.topkv_crc_begin(self.layout, self.batch, self.workspace, self.ws_bytes, stream))

    def send_layer(self, layer: int, h_wire: torch.Tensor, stream, slot: int = 0):
        st = self.stagings[slot]
        tk.check(tk.topkv_pack_layer_to_host_crc(
            layer, self.pool, self.layout, self.batch, h_wire, h_wire.numel(), st, st.numel(),
            self.workspace, self.ws_bytes, stream))

    def finish(self, stream, request_ids, model_id: int, h_seq_lens) -> list[tk.topkv_wire_header]:
        crc = self._checksums(stream)
        headers = []
        for r, rid in enumerate(request_ids):
            h = tk.topkv_wire_header()
            crc_v = int(crc[r, 1]) if self.layout.kv_factor == 2 else 0
            tk.check(tk.topkv_header_fill(h, int(rid), model_id, self.layout, int(h_seq_lens[r]),
                                          int(crc[r, 0]), crc_v))
            headers.append(h)
        return headers


class TransferReceiver(Endpoint):
    """Places layers from ``h_wire`` into its own pool and verifies the headers."""

    def begin(self, stream):
        tk.check(tk.topkv_crc_begin(self.layout, self.batch, self.workspace, self.ws_bytes, stream))

    def recv_layer(self, layer: int, h_wire: torch.Tensor, stream, slot: int = 0):
        st = self.stagings[slot]
        tk.check(tk.topkv_unpack_layer_from_host_crc(
            layer, self.pool, self.layout, self.batch, h_wire, h_wire.numel(), st, st.numel(),
            self.workspace, self.ws_bytes, stream))

    def finish(self, stream, headers, h_seq_lens) -> list[int]:
        """Status per request: TOPKV_OK or TOPKV_ERR_CHECKSUM."""
        crc = self._checksums(stream)
        out = []
        for r, h in enumerate(headers):
            crc_v = int(crc[r, 1]) if self.layout.kv_factor == 2 else 0
            out.append(tk.topkv_header_check(h, self.layout, int(h_seq_lens[r]), int(crc[r, 0]), crc_v))
        return out


class _NewTokens:
    """Which rows of a DecodeCache have tokens whose K/V are still to be written, kept on the device,
    where alone it is known which requests an extension refused. ``append`` writes a row if its last
    wish was met and it is longer than what has been written; every row keeps the wire rows that it
    asked for, so that the caller's slab fits whatever was refused. All methods work on the current
    stream."""

    def __init__(self, seq_lens: torch.Tensor):
        self.seq_lens = seq_lens
        self.row = torch.arange(len(seq_lens), dtype=torch.int32, device=seq_lens.device)
        self.state = torch.zeros((2, len(seq_lens)), dtype=torch.int32, device=seq_lens.device)
        self.written, self.asked = self.state       # tokens whose K/V are there, length asked for
        self.lens = torch.zeros_like(seq_lens)      # append's lengths: 0 leaves a row out
        self.offsets: dict[int, torch.Tensor] = {}  # tokens of a call -> first wire row of each request
        self.known = False                          # an extension says what is new ...
        self.pending = False                        # ... and its appends are not all enqueued yet

    def extending(self, new: torch.Tensor):
        if self.pending:
            torch.minimum(self.written, self.seq_lens, out=self.written)
        else:
            self.written.copy_(self.seq_lens)
        torch.add(self.seq_lens, new.clamp(min=0), out=self.asked)
        self.known = self.pending = True

    def update(self):
        torch.mul(self.seq_lens, (self.seq_lens == self.asked) & (self.seq_lens > self.written), out=self.lens)
        for tokens in self.offsets:
            self.count_rows(tokens)

    def count_rows(self, tokens: int):
        if tokens not in self.offsets:
            self.offsets[tokens] = torch.zeros(len(self.seq_lens) + 1, dtype=torch.int64, device=self.seq_lens.device)
        torch.cumsum(self.asked.clamp(max=tokens), 0, out=self.offsets[tokens][1:])

    def all_written(self):
        torch.maximum(self.written, self.lens, out=self.written)
        self.pending = False

    def freed(self, rows: torch.Tensor):
        if self.pending:
            self.state.masked_fill_((rows[:, None] == self.row).any(0), 0)
            self.update()
        else:
            self.known = False

    def forked(self, parents: torch.Tensor, children: torch.Tensor, before: torch.Tensor | None):
        if self.pending:  # a row that was forked into (its length says so) is where its parent is
            n = len(parents)
            which = torch.where(children[:, None] == self.row, torch.arange(n, device=self.row.device)[:, None], n).amin(0)
            parent = torch.cat([parents, parents.new_zeros(1)])[which].clamp(0, len(self.row) - 1).long()
            self.state.copy_(torch.where(self.seq_lens != before, self.state[:, parent], self.state))
            self.update()
        else:
            self.known = False


class DecodeCache:
    """The paged cache of a decode worker, from the tables of a receiver (or any pool and tables):
    ``rows`` request slots of ``max_pages`` pages each, of which the first ones hold the requests
    that have arrived. All tables live on the device and are changed in place, by the calls below
    alone, which only enqueue work on ``stream``; calls are ordered by the stream they are given, and one
    object's calls must not run at the same time (they share a workspace). ``max_forks`` bounds
    the forks of one call. In a CUDA graph an extension stands together with its appends, or both are
    made outside."""

    def __init__(self, pool: torch.Tensor, layout: tk.topkv_layout, block_table: torch.Tensor, seq_lens: torch.Tensor,
                 rows: int | None = None, max_pages: int | None = None, max_forks: int = 64):
        dev = pool.device
        R, maxp = block_table.shape
        rows, max_pages = R if rows is None else rows, maxp if max_pages is None else max_pages
        if rows < R or max_pages < maxp:
            raise ValueError("rows and max_pages must hold the tables that are taken over")
        self.pool, self.layout, self.max_forks = pool, layout, max_forks
        self.block_table = torch.full((rows, max_pages), -1, dtype=torch.int32, device=dev)
        self.block_table[:R, :maxp] = block_table
        self.seq_lens = torch.zeros(rows, dtype=torch.int32, device=dev)
        self.seq_lens[:R] = seq_lens
        used = torch.arange(max_pages, device=dev)[None, :] * layout.page_tokens < self.seq_lens[:, None]
        self.block_table.masked_fill_(~used, -1)
        self.ref_counts = torch.bincount(self.block_table[used].long(), minlength=layout.num_pool_pages).to(torch.int32)
        self.batch = tk.make_batch(self.block_table, self.seq_lens)
        self.tables = tk.make_page_tables(self.ref_counts, self.block_table, self.seq_lens, self.ref_counts)
        n = tk.check(tk.topkv_page_workspace_bytes(layout, self.batch, max_forks))
        self.workspace = torch.empty(max(n, 16), dtype=torch.uint8, device=dev)
        self.num_used = torch.zeros(1, dtype=torch.int32, device=dev)
        self.page_map = torch.zeros(layout.num_pool_pages, dtype=torch.int32, device=dev)
        self._attend_ws: dict[int, torch.Tensor] = {}
        self._new = _NewTokens(self.seq_lens)
        self._first_rows = None
        torch.cuda.current_stream(dev).synchronize()

    def _on(self, stream):
        """torch's work on the stream that the library's calls are given: a torch stream, a handle or None."""
        if stream is None or stream == 0:
            stream = torch.cuda.default_stream(self.pool.device)
        elif isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, self.pool.device)
        return torch.cuda.stream(stream)

    def _check_ints(self, name: str, t: torch.Tensor, count: int | None = None):
        if t.dtype != torch.int32 or t.ndim != 1 or not t.is_contiguous() or t.device != self.pool.device:
            raise ValueError(f"{name}: a contiguous int32 vector on the pool's device")
        if count is not None and t.numel() != count:
            raise ValueError(f"{name}: {count} entries, one per row")

    def extend(self, new_tokens: torch.Tensor, stream):
        """Room for new_tokens[r] (device int32 [rows]) more tokens of every request. A request for which
        there is no page stays as it is (error bit 8) and is left out by the appends that follow."""
        self._check_ints("new_tokens", new_tokens, len(self.seq_lens))
        with self._on(stream):
            self._new.extending(new_tokens)
            tk.check(tk.topkv_extend_requests(self.layout, self.batch, self.tables, new_tokens, self.workspace,
                                              self.workspace.numel(), stream))
            self._new.update()

    def append(self, layer: int, kv: torch.Tensor, stream, tokens: int = 1):
        """Writes the K/V of the last ``tokens`` tokens of every request that has new ones: ``kv`` is a
        wire slab of min(length, tokens) tokens per request, in request order (empty rows contribute
        none). The tokens of a request that has not grown since the last append, or that the last
        ``extend`` refused, are left as they are; it keeps its place in the slab, a refused one the
        min(length + new_tokens, tokens) tokens that it asked for. Without an ``extend`` since the last
        fork or free every request is written. ``tokens`` beyond what a request grew by write older
        tokens again, which must not lie in shared pages. The last layer's append ends the turn."""
        if tokens < 1 or not kv.is_contiguous() or kv.device != self.pool.device:
            raise ValueError("a contiguous slab of one or more tokens per request, on the pool's device")
        new = self._new
        if new.known:
            if tokens not in new.offsets:
                with self._on(stream):
                    new.count_rows(tokens)
            b = tk.make_batch(self.block_table, new.lens, cu_seq_lens=new.offsets[tokens], window_tokens=tokens)
        else:
            first = None
            if len(self.seq_lens) > tk.TOPKV_MAX_INLINE_R:  # a copy works the wire rows out itself up to there
                if self._first_rows is None:
                    with self._on(stream):
                        self._first_rows = torch.empty(len(self.seq_lens) + 1, dtype=torch.int64, device=self.pool.device)
                first = self._first_rows
                tk.check(tk.topkv_build_plan(tk.make_batch(self.block_table, self.seq_lens, window_tokens=tokens), first, stream))
            b = tk.make_batch(self.block_table, self.seq_lens, cu_seq_lens=first, window_tokens=tokens)
        at = layer * self.layout.wire_layer_stride  # the call adds it: kv is this layer's slab alone
        tk.check(tk.topkv_unpack_layer(layer, self.pool, self.layout, b, kv.data_ptr() - at, kv.numel() * kv.element_size() + at,
                                       stream))
        if new.known and layer == self.layout.num_layers - 1:
            with self._on(stream):
                new.all_written()

    def attend(self, layer: int, q: torch.Tensor, out: torch.Tensor, scale: float, stream, cache_type: int | None = None,
               window_tokens: int = 0, **attention):
        """Attention of the newest token of every request; see topkv_attend_layer. ``q`` and ``out`` have
        one entry per row, the empty ones included. ``attention`` goes to make_attention (value_dim,
        sink_tokens, k_scale, v_scale, lse)."""
        if q.dtype not in (torch.bfloat16, torch.float16) or q.device != self.pool.device:
            raise ValueError("q and out are bfloat16 or float16 on the pool's device")
        if q.ndim != 3 or q.shape[0] != len(self.seq_lens) or q.shape[2] != self.layout.head_dim:
            raise ValueError(f"q is [{len(self.seq_lens)}][heads][{self.layout.head_dim}]")
        io = tk.TOPKV_TYPE_BF16 if q.dtype == torch.bfloat16 else tk.TOPKV_TYPE_FP16
        att = tk.make_attention(q, out, io if cache_type is None else cache_type, io, scale, **attention)
        b = tk.make_batch(self.block_table, self.seq_lens, window_tokens=window_tokens)
        n = tk.check(tk.topkv_attend_workspace_bytes(self.layout, b, att))
        # One per size (a kind of layer has one, whatever the lengths), kept as long as the cache: captured
        # graphs hold the address, and calls on other streams may still be using it.
        if n not in self._attend_ws:
            with self._on(stream):
                self._attend_ws[n] = torch.empty(max(n, 16), dtype=torch.uint8, device=self.pool.device)
        ws = self._attend_ws[n]
        tk.check(tk.topkv_attend_layer(layer, self.pool, self.layout, b, att, q, out, ws, ws.numel(), stream))

    def fork(self, parents: torch.Tensor, children: torch.Tensor, stream):
        """Row children[i] becomes a copy of row parents[i] that shares its full pages."""
        self._check_ints("parents", parents)
        self._check_ints("children", children)
        if parents.numel() != children.numel() or parents.numel() > self.max_forks:
            raise ValueError("as many parents as children, at most max_forks")
        if parents.numel() == 0:
            return
        with self._on(stream):
            before = self.seq_lens.clone() if self._new.pending else None
            tk.check(tk.topkv_fork_requests(self.pool, self.layout, self.batch, self.tables, parents, children, parents.numel(),
                                            self.workspace, self.workspace.numel(), stream))
            self._new.forked(parents, children, before)

    def free(self, rows: torch.Tensor, stream):
        """The rows (device int32) give their pages back and become empty."""
        self._check_ints("rows", rows)
        with self._on(stream):
            tk.check(tk.topkv_free_requests(self.layout, self.batch, self.tables, rows, rows.numel(), stream))
            self._new.freed(rows)

    def compact(self, stream):
        """Afterwards pages 0 .. num_used - 1 are the ones in use; page_map has every page's new id."""
        tk.check(tk.topkv_compact_pages(self.pool, self.layout, self.batch, self.tables, self.num_used, self.page_map,
                                        self.workspace, self.workspace.numel(), stream))


def transfer(sender: TransferSender, receiver: TransferReceiver, h_wire: torch.Tensor,
             request_ids, model_id: int, h_seq_lens, layer_ready=None, corrupt=None):
    """Runs one whole transfer through pinned host memory, pipelined per layer (the receiver
    starts on layer l as soon as it has arrived); each side alternates between two streams. ``layer_ready[l]`` is an
    optional event (e.g. recorded by the prefill) that gates the sending of layer l.
    ``corrupt`` (layer, byte offset) flips one bit of that layer's slab in flight: a test hook
    standing in for a faulty link. Returns (headers, per-request status)."""
    dev = sender.pool.device
    tx = [torch.cuda.Stream(dev), torch.cuda.Stream(dev)]
    rx = [torch.cuda.Stream(dev), torch.cuda.Stream(dev)]
    L = sender.layout.num_layers

    def after(first, second):
        """second starts (continues) only after what first holds so far."""
        ev = torch.cuda.Event()
        ev.record(first)
        second.wait_event(ev)

    sender.begin(tx[0])
    receiver.begin(rx[0])
    after(tx[0], tx[1])
    after(rx[0], rx[1])
    for layer in range(L):
        q = layer & 1
        if layer_ready is not None:
            tx[q].wait_event(layer_ready[layer])
        sender.send_layer(layer, h_wire, tx[q], q)
        arrived = torch.cuda.Event()
        arrived.record(tx[q])
        if corrupt is not None and corrupt[0] == layer:
            arrived.synchronize()
            h_wire[layer * sender.layout.wire_layer_stride + corrupt[1]] ^= 0x04
        rx[q].wait_event(arrived)
        receiver.recv_layer(layer, h_wire, rx[q], q)
    after(tx[1], tx[0])
    after(rx[1], rx[0])
    headers = sender.finish(tx[0], request_ids, model_id, h_seq_lens)
    status = receiver.finish(rx[0], headers, h_seq_lens)
    return headers, status
