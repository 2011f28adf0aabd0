"""PrefillEngine: the per-batch hot path wired over libarckv.

prepare (hash blocks, plan the batch on the host cache, plan the attention work, pack the
metadata: one native call) -> copy metadata to the device -> [project Q/K/V] -> scatter the
computed tokens' K/V -> prefix-cached prefill attention -> release.
kv_format="mx4" holds K and V in 4 bits and runs the same steps over them; gather() reads rows back.
attention_weights() after attention(lse=) adds up what every cached token received, evict() moves
the heaviest tokens into blocks that the caller owns.
Every step is a libarckv call; this class owns the device buffers (PyTorch tensors used
only as device memory) and the host cache handle.  plan() + upload() are the same first
steps as separate calls.
"""

from __future__ import annotations

import contextlib
from dataclasses import dataclass

import numpy as np

from . import (BlockCache, BatchPlan, _current_stream, attention_plan, hash_blocks_batch, lib, unpack_prepared)
from . import _lib


@dataclass
class DeviceBatch:
    """A planned batch on the device.  The arrays lie in the engine's ring of metadata buffers: they hold the batch
    until the fourth prepare() or upload() after it.  Of a batch whose calls were captured into a graph they
    stay, as long as the DeviceBatch (a graph's owner keeps it)."""
    plan: BatchPlan
    block_tables: object
    cu_q: object
    seq_lens: object
    slot_mapping: object
    work: object
    n_work: int
    n_combine: int
    ws_bytes: int
    tile_cols: int
    n_tokens: int = 0          # computed (suffix) tokens of the batch: rows of q / k_new / v_new
    work_ptr: int = 0          # device address of the work array
    true_lens: object = None   # of plan.true_lens: the lengths that project() counts positions by (None: seq_lens)


class PrefillEngine:
    def __init__(self, num_q_heads: int, num_kv_heads: int, head_dim: int, capacity: int,
                 num_phys: int, scratch: int, policy: str = "arc", initial_order=None,
                 ref_order: str = "tail_first", device: str = "cuda", num_cus: int | None = None,
                 pool_fill: int = -1, victim_window: int = 1, intra_batch_reuse: bool = True,
                 frc_p: float = 0.0, kv_format: str = "bf16", private_blocks: int = 0):
        """kv_format: "bf16" (k_pool / v_pool, layout V1) or "mx4" (kv_pool: K and V in 4 bits,
        layout MX4).  private_blocks: blocks num_phys .. num_phys + private_blocks - 1 of the pools
        that the block cache does not manage (a caller's own, e.g. for evicted sessions)."""
        import torch
        if kv_format not in ("bf16", "mx4"):
            raise ValueError(f"kv_format {kv_format!r} is not bf16 or mx4")
        if private_blocks < 0:
            raise ValueError("private_blocks must not be negative")
        self.hq, self.hkv, self.d = num_q_heads, num_kv_heads, head_dim
        self.scale = head_dim ** -0.5
        self.device = self._device_of(device)
        self.num_phys = num_phys
        self.num_blocks = num_phys + private_blocks
        self.kv_format = kv_format
        self.k_pool = self.v_pool = self.kv_pool = None
        # pools hold bf16 bit patterns; the fill (0xFFFF, a NaN pattern) marks untouched slots
        if kv_format == "bf16":
            self.k_pool = torch.full((self.num_blocks, num_kv_heads, 16, head_dim), pool_fill, dtype=torch.int16,
                                     device=self.device)
            self.v_pool = torch.full((self.num_blocks, num_kv_heads, head_dim, 16), pool_fill, dtype=torch.int16,
                                     device=self.device)
        else:                   # every byte the fill's low one: scales of 0xFF read back as NaN too
            self.kv_pool = torch.full((self.num_blocks, num_kv_heads, 17 * head_dim), pool_fill & 0xFF,
                                      dtype=torch.uint8, device=self.device)
        self.cache = BlockCache(policy, capacity, num_phys, scratch, initial_order, ref_order, victim_window,
                                intra_batch_reuse, frc_p)
        if num_cus is None:
            num_cus = torch.cuda.get_device_properties(self.device).multi_processor_count
        self.num_cus = int(num_cus)
        self._ws = torch.empty(0, dtype=torch.uint8, device=self.device)
        self._y = None          # rotary (cos, sin) table of the batch (arckv_qkv_rope workspace)
        # a ring of reusable pinned staging buffers and device metadata buffers, with the events
        # that mark their copies done: the host may prepare up to four batches ahead of the GPU
        # (a slow host step is then absorbed), and no pinned memory is allocated per batch
        self._ring = 4
        self._stage = [None] * self._ring
        self._stage_ev = [None] * self._ring
        self._dev_meta = [None] * self._ring
        self._turn = 0
        # the stream (handle) of the last call: first the one that the pools are being filled on
        self._last = _current_stream(self.device.index) if self.device.type == "cuda" else None
        self._done = None       # an event behind all it has queued, where there is one
        self._home = {}         # of a buffer's address: the stream that it was allocated on

    @staticmethod
    def _device_of(device):
        """With its index: the engine stays on the device that is current now, whichever is later."""
        import torch
        device = torch.device(device)
        if device.type == "cuda" and device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        return device

    # ---- host steps ----------------------------------------------------------------------
    def plan(self, token_lists) -> BatchPlan:
        """Hashes and the cache plan only (prepare() does these and the rest in one call)."""
        hashes = hash_blocks_batch(token_lists)
        return self.cache.plan_batch([(h, len(t)) for h, t in zip(hashes, token_lists)])

    def release(self):
        self.cache.release_batch()

    def prepare(self, token_lists, stream=None, hashes=None, n_tokens=None) -> DeviceBatch:
        """plan() + upload() in one native call (arckv_prepare_batch): hashes, the cache plan
        and the attention work plan are written straight into the next pinned staging buffer of
        the ring, then one asynchronous copy on `stream` moves them to the device.  A caller that
        keeps its requests' block hashes passes `hashes` and `n_tokens` instead of token lists."""
        import torch
        self._not_captured("prepare")
        ts = self._torch_stream(stream)
        t = self._turn
        self._turn = (t + 1) % self._ring
        if self._stage_ev[t] is not None:
            self._stage_ev[t].synchronize()          # the copy that last read this buffer is done
        while True:
            host = None if self._stage[t] is None else self._stage[t].numpy()
            st, d, pl, hb = self.cache.prepare_native(token_lists, self.hq, self.hkv, self.d, self.num_cus, host,
                                                      hashes=hashes, n_tokens=n_tokens)
            if st == _lib.ENOSPC and (host is None or d["n_packed"] > host.size):
                cap = max(d["n_packed"], 1 << 16) * 2
                self._stage[t] = torch.empty(cap, dtype=torch.int32, pin_memory=True)
                self._dev_meta[t] = self._grow(self._dev_meta[t], cap, torch.int32, ts)
                continue
            _lib.check(st, "arckv_prepare_batch")
            break
        n_int = d["n_packed"]
        dev = self._copy_meta(t, n_int, ts)
        plan, ap = unpack_prepared(host, d, pl, hb)
        n, stride = d["n_reqs"], d["bt_stride"]
        bt = dev[d["off_block_tables"]:d["off_block_tables"] + n * stride].view(n, stride)
        cu = dev[d["off_cu_q"]:d["off_cu_q"] + n + 1]
        sl = dev[d["off_seq_lens"]:d["off_seq_lens"] + n]
        sm = dev[d["off_slots"]:d["off_slots"] + d["n_slots"]]
        wk = dev[d["off_work"]:d["off_work"] + (d["n_work"] + d["n_combine"]) * 8].view(-1, 8)
        self._ensure_ws(d["ws_bytes"], ts)
        return DeviceBatch(plan, bt, cu, sl, sm, wk, d["n_work"], d["n_combine"], d["ws_bytes"],
                           d["tile_cols"], int(d["n_slots"]), wk.data_ptr())

    def upload(self, plan: BatchPlan, stream=None) -> DeviceBatch:
        """The metadata of a plan() result to the device, copied on `stream`."""
        import torch
        self._not_captured("upload")
        ts = self._torch_stream(stream)
        ap = attention_plan(plan.cu_q, plan.seq_lens, self.hq, self.hkv, self.d, self.num_cus)
        parts = [plan.block_tables.ravel(), plan.cu_q, plan.seq_lens, plan.slot_mapping, ap.work.ravel()]
        if plan.true_lens is not None:
            if len(plan.true_lens) != plan.n_reqs:
                raise ValueError("true_lens must hold one length per request")
            parts.append(plan.true_lens)
        n_int = sum(p.size for p in parts)
        t = self._turn
        self._turn = (t + 1) % self._ring
        if self._stage_ev[t] is not None:
            self._stage_ev[t].synchronize()          # the copy that last read this buffer is done
        if self._stage[t] is None or self._stage[t].numel() < n_int:
            cap = max(n_int, 1 << 16) * 2
            self._stage[t] = torch.empty(cap, dtype=torch.int32, pin_memory=True)
            self._dev_meta[t] = self._grow(self._dev_meta[t], cap, torch.int32, ts)
        host = self._stage[t].numpy()
        o = 0
        for p in parts:
            host[o:o + p.size] = p
            o += p.size
        dev = self._copy_meta(t, n_int, ts)
        n = plan.n_reqs
        o = 0
        bt = dev[o:o + plan.block_tables.size].view(n, plan.block_tables.shape[1]); o += plan.block_tables.size
        cu = dev[o:o + n + 1]; o += n + 1
        sl = dev[o:o + n]; o += n
        sm = dev[o:o + len(plan.slot_mapping)]; o += len(plan.slot_mapping)
        wk = dev[o:o + ap.work.size].view(-1, 8); o += ap.work.size
        self._ensure_ws(ap.ws_bytes, ts)
        return DeviceBatch(plan, bt, cu, sl, sm, wk, ap.n_work, ap.n_combine, ap.ws_bytes, ap.tile_cols,
                           int(plan.cu_q[-1]), wk.data_ptr(), None if plan.true_lens is None else dev[o:o + n])

    def resume(self, tables, held, new, true_lens, stream=None) -> DeviceBatch:
        """The next batch of sessions that evict() cut: request r holds held[r] tokens in the private blocks
        tables[r] and computes new[r] more behind them, which are the last of the true_lens[r] tokens of
        its prompt: project() rotates them for those positions, as the held ones were for theirs.
        Host integers, tables [n_reqs, >= ceil((held + new) / 16) of the longest]."""
        tables, held, new, true_lens = (np.asarray(x) for x in (tables, held, new, true_lens))
        n = len(held)
        if tables.ndim != 2 or any(x.ndim != 1 for x in (held, new, true_lens)) or \
                not len(tables) == n == len(new) == len(true_lens):
            raise ValueError("tables must be [n_reqs, blocks], held, new and true_lens [n_reqs]")
        if any(x.size and x.dtype.kind not in "iu" for x in (tables, held, new, true_lens)):
            raise ValueError("tables and lengths must hold integers")
        held, new, true_lens = (x.astype(np.int64) for x in (held, new, true_lens))
        seq = held + new
        if n and (min(held.min(), new.min()) < 0 or (true_lens < seq).any() or true_lens.max() > np.iinfo(np.int32).max):
            raise ValueError("a session has no fewer tokens than it holds and computes: 0 <= held, new; held + new <= true_lens")
        blocks = -(-seq // 16)
        if n and blocks.max() > tables.shape[1]:
            raise ValueError(f"tables must have {int(blocks.max())} blocks for the longest session")
        used = np.arange(tables.shape[1]) < blocks[:, None]
        if used.any() and (tables[used].min() < self.num_phys or tables[used].max() >= self.num_blocks):
            raise ValueError(f"tables must name private blocks, {self.num_phys} to {self.num_blocks - 1}")
        bt = np.where(used, tables, -1).astype(np.int32)
        at = [np.arange(h, s) for h, s in zip(held, seq)]
        slots = [bt[r, i // 16].astype(np.int64) * 16 + i % 16 for r, i in enumerate(at)]
        slots = np.concatenate([*slots, np.zeros(0, np.int64)])
        if len(np.unique(slots)) < len(slots):
            raise ValueError("tables let two sessions write one slot")
        i32 = [x.astype(np.int32) for x in (np.concatenate([[0], np.cumsum(new)]), seq, held, held // 16, slots, true_lens)]
        plan = BatchPlan(bt, *i32[:5], int(new.max(initial=0)), int(seq.max(initial=0)), i32[5])
        return self.upload(plan, stream)

    # ---- streams ---------------------------------------------------------------------------
    # `stream` is None (torch's current stream), a torch.cuda.Stream or a raw hipStream_t
    # handle.  The metadata copy, its event and every (re)allocation of a device buffer run on
    # that stream, the stream the kernels then run on: the kernels are ordered after the copy.
    # The pools, the workspaces and the metadata ring are one set for all streams, so an engine's
    # work runs in the order of its calls: a call on another stream than the call before makes
    # its stream wait for what that one has queued.  The event for that is recorded when the stream
    # changes; of a raw handle, which its owner may have destroyed by then, behind every call.  A stream
    # under capture waits for nothing (torch.cuda.graph starts a capture with the device idle).
    def _torch_stream(self, stream):
        import torch
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        elif not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(int(stream), device=self.device)
        self._in_order(stream.cuda_stream)
        return stream

    def _stream(self, stream):
        if stream is None:
            handle = _current_stream(self.device.index)
        else:
            handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
        self._in_order(handle)
        return handle

    def _in_order(self, handle: int):
        if handle != self._last:
            self._change_stream(handle)
        else:
            self._done = None

    def _change_stream(self, handle: int):
        if self._capturing(handle):
            return
        if self._done is None and self._last is not None:
            if self._capturing(self._last):
                return
            self._mark(self._last)
        if self._done is not None:
            self._handle(handle).wait_event(self._done)
        self._last, self._done = handle, None

    def _handle(self, handle: int):
        import torch
        return torch.cuda.ExternalStream(handle, device=self.device) if handle else torch.cuda.default_stream(self.device)

    def _capturing(self, handle: int) -> bool:
        import torch
        with torch.cuda.stream(self._handle(handle)):
            return torch.cuda.is_current_stream_capturing()

    def _mark(self, handle: int):
        import torch
        self._done = torch.cuda.Event()
        self._done.record(self._handle(handle))

    # Calls may be captured by torch.cuda.graph.  A replay reads the metadata and writes the workspaces that were
    # captured, while the engine goes on with other batches and other graphs: so a captured call's
    # workspace is the graph's own memory, and the ring lets go of its batch's buffer (the batch keeps it).
    # A replay is the caller's work, who orders it with the engine's calls on the same blocks.
    @staticmethod
    def _not_captured(name: str):
        import torch
        if torch.cuda.is_current_stream_capturing():
            raise ValueError(f"{name} copies from a staging buffer that it fills again, and cannot be captured")

    def _captured(self, db: DeviceBatch) -> bool:
        import torch
        if not torch.cuda.is_current_stream_capturing():
            return False
        for t, dev in enumerate(self._dev_meta):
            if dev is not None and 0 <= db.cu_q.data_ptr() - dev.data_ptr() < 4 * dev.numel():
                self._dev_meta[t] = self._stage[t] = self._stage_ev[t] = None
        return True

    def _rope_table(self, db: DeviceBatch, stream):
        """The workspace of the producer: a (cos, sin) table of the batch's tokens."""
        import torch
        need = max(4 * db.n_tokens * self.d, 1)
        if self._captured(db):
            return torch.empty(need, dtype=torch.uint8, device=self.device)
        if self._y is None or self._y.numel() < need:
            self._y = self._grow(self._y, need, torch.uint8, self._torch_stream(stream))
        return self._y

    def _grow(self, old, n: int, dtype, ts):
        """A device buffer of n elements, allocated in the order of stream ts, in place of `old`, whose memory goes
        back to the order of the stream that it was allocated on.  That stream may be another, and knows
        nothing of what ts has queued: then the host waits for it."""
        import torch
        if old is not None and self._home.pop(old.data_ptr(), ts.cuda_stream) != ts.cuda_stream:
            ts.synchronize()
        with torch.cuda.stream(ts):
            new = torch.empty(n, dtype=dtype, device=self.device)
        self._home[new.data_ptr()] = ts.cuda_stream
        return new

    def _call(self, name: str, stream, *args, events=()):
        """A library call on the engine's device (made the current one if it is not) and `stream`."""
        import torch
        index = self.device.index
        if index is None or index == torch.cuda.current_device():
            _lib.check(getattr(lib(), name)(*args, self._stream(stream), *events), name)
        else:
            with torch.cuda.device(index):
                _lib.check(getattr(lib(), name)(*args, self._stream(stream), *events), name)
        if isinstance(stream, int) and not self._capturing(stream):
            self._mark(stream)

    @staticmethod
    def _bad(t, shape, size: int = 2) -> bool:
        """Whether t is not a contiguous device tensor of that shape and element size."""
        return tuple(t.shape) != shape or not (t.is_cuda and t.is_contiguous()) or t.element_size() != size

    def _copy_meta(self, t: int, n_int: int, ts):
        """Staging buffer t -> its device buffer on stream ts; the event marks the copy done, so
        that the host refills the staging buffer only after the copy has read it."""
        import torch
        dev = self._dev_meta[t][:n_int]
        with torch.cuda.stream(ts):
            dev.copy_(self._stage[t][:n_int], non_blocking=True)
            ev = torch.cuda.Event()
            ev.record(ts)
        self._stage_ev[t] = self._done = ev
        return dev

    def _ensure_ws(self, nbytes: int, ts):
        if nbytes > self._ws.numel():
            import torch
            self._ws = self._grow(self._ws, nbytes, torch.uint8, ts)

    # ---- device steps --------------------------------------------------------------------
    # The engine built every device buffer itself, so these calls skip the binding's per-call
    # tensor checks and pass raw addresses straight to the C ABI (the library still validates
    # sizes); they only check the shapes of the caller's q / k / v / out.

    def scatter(self, db: DeviceBatch, k_new, v_new, stream=None):
        shape = (db.n_tokens, self.hkv, self.d)
        if self._bad(k_new, shape) or self._bad(v_new, shape):
            raise ValueError(f"k_new / v_new must be contiguous 16-bit {shape}")
        self._captured(db)
        rows = (k_new.data_ptr(), v_new.data_ptr(), db.slot_mapping.data_ptr(), db.n_tokens, self.num_blocks,
                self.hkv, self.d)
        if self.kv_format == "mx4":
            self._call("arckv_kv_scatter_mx4", stream, self.kv_pool.data_ptr(), *rows)
        else:
            self._call("arckv_kv_scatter", stream, self.k_pool.data_ptr(), self.v_pool.data_ptr(), *rows)

    def gather(self, slots, k_out, v_out, stream=None):
        """The K and V rows [n, Hkv, D] that a 4-bit pool holds for `slots` (device int32 [n]), as bf16."""
        if self.kv_format != "mx4":
            raise ValueError("gather reads a 4-bit pool (kv_format mx4)")
        shape = (int(slots.numel()), self.hkv, self.d)
        if self._bad(k_out, shape) or self._bad(v_out, shape):
            raise ValueError(f"k_out / v_out must be contiguous 16-bit {shape}")
        if self._bad(slots, tuple(slots.shape), 4):
            raise ValueError("slots must be contiguous int32 on the device")
        self._call("arckv_kv_gather_mx4", stream, self.kv_pool.data_ptr(), k_out.data_ptr(), v_out.data_ptr(),
                   slots.data_ptr(), shape[0], self.num_blocks, self.hkv, self.d)

    @staticmethod
    def _position_lens(db: DeviceBatch) -> int:
        return (db.seq_lens if db.true_lens is None else db.true_lens).data_ptr()

    def project(self, db: DeviceBatch, x, w_qkv, q, k_new, v_new, rope_theta: float, stream=None):
        """Q/K/V of the batch's computed tokens from their hidden states x [n_tokens, H]
        (projection by w_qkv [(Hq + 2 Hkv) D, H] and rotary embedding, arckv_qkv_rope), rotated for the
        last positions of each request (of its true length, where the batch has them);
        k_new / v_new then go to scatter()."""
        t, h = db.n_tokens, int(x.shape[1])
        n_out = (self.hq + 2 * self.hkv) * self.d
        if self._bad(x, (t, h)) or self._bad(w_qkv, (n_out, h)):
            raise ValueError(f"x must be contiguous 16-bit [{t}, H] and w_qkv [{n_out}, H]")
        for a, c in ((q, self.hq), (k_new, self.hkv), (v_new, self.hkv)):
            if self._bad(a, (t, c, self.d)):
                raise ValueError("q / k_new / v_new must be contiguous 16-bit [n_tokens, heads, D]")
        y = self._rope_table(db, stream)
        self._call("arckv_qkv_rope", stream, x.data_ptr(), w_qkv.data_ptr(), t, h, self.hq, self.hkv, self.d,
                   db.cu_q.data_ptr(), self._position_lens(db), db.plan.n_reqs, float(rope_theta), y.data_ptr(), y.numel(),
                   q.data_ptr(), k_new.data_ptr(), v_new.data_ptr())

    def project_to_pool(self, db: DeviceBatch, x, w_qkv, q, rope_theta: float, stream=None):
        """project() with the KV scatter fused in (arckv_qkv_rope_to_pool): Q into q, the batch's
        K and V straight into the engine's pools at the plan's slots; no scatter() follows."""
        if self.kv_format != "bf16":
            raise ValueError("project_to_pool writes bf16 pools: a 4-bit pool takes project() and scatter()")
        t, h = db.n_tokens, int(x.shape[1])
        n_out = (self.hq + 2 * self.hkv) * self.d
        if self._bad(x, (t, h)) or self._bad(w_qkv, (n_out, h)):
            raise ValueError(f"x must be contiguous 16-bit [{t}, H] and w_qkv [{n_out}, H]")
        if self._bad(q, (t, self.hq, self.d)):
            raise ValueError("q must be contiguous 16-bit [n_tokens, heads, D]")
        y = self._rope_table(db, stream)
        self._call("arckv_qkv_rope_to_pool", stream, x.data_ptr(), w_qkv.data_ptr(), t, h, self.hq, self.hkv, self.d,
                   db.cu_q.data_ptr(), self._position_lens(db), db.plan.n_reqs, float(rope_theta), y.data_ptr(), y.numel(),
                   q.data_ptr(), self.k_pool.data_ptr(), self.v_pool.data_ptr(), self.num_blocks, db.slot_mapping.data_ptr())

    def attention(self, db: DeviceBatch, q, out, stream=None, events=None, lse=None):
        """Attention of the batch over the engine's pools.  `events` (bf16 pools): optional (begin,
        mid, end) torch.cuda.Event triple (already recorded once, so that each has its HIP handle),
        recorded by the library right before the attention kernel, between it and the split-KV
        combine, and after it.  `lse`: optional fp32 [n_tokens, Hq] that receives
        log sum_j exp(scale q . K[j]) of every row and head (for attention_weights)."""
        import torch
        shape = (db.n_tokens, self.hq, self.d)
        if self._bad(q, shape) or self._bad(out, shape):
            raise ValueError(f"q / out must be contiguous 16-bit {shape}")
        if lse is not None:
            self._check_lse(db, lse)
        ws = self._ws
        if self._captured(db) and db.ws_bytes:
            ws = torch.empty(db.ws_bytes, dtype=torch.uint8, device=self.device)
        args = (db.block_tables.data_ptr(), int(db.block_tables.shape[1]), db.cu_q.data_ptr(), db.seq_lens.data_ptr(),
                db.plan.n_reqs, db.n_tokens, self.num_blocks, db.work_ptr, db.n_work, db.n_combine, db.tile_cols,
                self.hq, self.hkv, self.d, self.scale, ws.data_ptr() if db.ws_bytes else None, db.ws_bytes)
        qo = (q.data_ptr(), out.data_ptr())
        if self.kv_format == "mx4":
            if events is not None:
                raise ValueError("events are recorded around the bf16 kernels only")
            self._call("arckv_prefill_attention_mx4", stream, self.kv_pool.data_ptr(), *qo,
                       None if lse is None else lse.data_ptr(), *args)
            return
        pools = (self.k_pool.data_ptr(), self.v_pool.data_ptr())
        if events is not None:
            if lse is not None:
                raise ValueError("the timed call writes no lse")
            self._call("arckv_prefill_attention_timed", stream, *pools, *qo, *args, events=[e.cuda_event for e in events])
        elif lse is not None:
            self._call("arckv_prefill_attention_lse", stream, *pools, *qo, lse.data_ptr(), *args)
        else:
            self._call("arckv_prefill_attention", stream, *pools, *qo, *args)

    def _check_lse(self, db: DeviceBatch, lse):
        if self._bad(lse, (db.n_tokens, self.hq), 4) or not lse.is_floating_point():
            raise ValueError(f"lse must be contiguous fp32 {(db.n_tokens, self.hq)}")

    def attention_weights(self, db: DeviceBatch, q, lse, weights, accumulate: bool = True, stream=None):
        """weights[r, h, j] += (accumulate False: =) the attention weight that token j of request r
        receives from the batch's rows through KV head h; lse from attention(lse=).  weights: fp32
        [n_reqs, Hkv, stride]; tokens past the stride are left out."""
        shape = (db.n_tokens, self.hq, self.d)
        if self._bad(q, shape):
            raise ValueError(f"q must be contiguous 16-bit {shape}")
        self._check_lse(db, lse)
        n = db.plan.n_reqs
        self._check_weights(n, weights)
        self._captured(db)
        mx4 = self.kv_format == "mx4"
        self._call("arckv_attention_weights", stream, (self.kv_pool if mx4 else self.k_pool).data_ptr(),
                   _lib.LAYOUT_MX4 if mx4 else _lib.LAYOUT_V1, q.data_ptr(), lse.data_ptr(), db.block_tables.data_ptr(),
                   int(db.block_tables.shape[1]), db.cu_q.data_ptr(), db.seq_lens.data_ptr(), n, db.n_tokens,
                   self.num_blocks, self.hq, self.hkv, self.d, self.scale, weights.data_ptr(), int(weights.shape[2]),
                   1 if accumulate else 0)

    def _check_weights(self, n: int, weights):
        if weights.dim() != 3 or self._bad(weights, (n, self.hkv, int(weights.shape[2])), 4) or \
                not weights.is_floating_point():
            raise ValueError(f"weights must be contiguous fp32 [{n}, {self.hkv}, stride]")

    def evict(self, db: DeviceBatch, weights, keep: int, dst_tables, n_first: int = 0, n_recent: int = 0, stream=None):
        """Cuts every request of the batch down to at most `keep` tokens for each KV head: the first
        n_first, the last n_recent, and the heaviest others by `weights` (fp32 [n_reqs, Hkv, stride >= the
        longest request]).  Their K and V move into the blocks of dst_tables (host int32 [n_reqs, >=
        ceil(keep / 16)]: private blocks of the caller's, num_phys and up, none twice and none of them a
        block of the batch).  Returns (kept positions int32 [n_reqs, Hkv, keep], -1 behind a shorter request's;
        their weights, fp32).  Afterwards request r holds min(L_r, keep) tokens in dst_tables[r], and goes on
        by resume().  The
        batch must not have been released, and the stream must not be capturing (a graph takes
        evict_select and kv_compact, with tables on the device)."""
        import torch
        plan, n = db.plan, db.plan.n_reqs
        self._check_weights(n, weights)
        if n and int(weights.shape[2]) < int(plan.seq_lens.max()):
            raise ValueError("weights must have an entry for every token of the longest request")
        dst = np.asarray(dst_tables)
        nb = -(-keep // 16)
        if dst.size and dst.dtype.kind not in "iu":
            raise ValueError("dst_tables must hold integers")
        if dst.ndim != 2 or dst.shape[0] != n or dst.shape[1] < nb:
            raise ValueError(f"dst_tables must be [{n}, >= {nb}]")
        own = dst[:, :nb].ravel()
        if own.size:
            lo, hi = int(own.min()), int(own.max())    # of the numbers as given: more than 32 bits would wrap
            if lo < 0 or hi >= self.num_blocks:
                raise ValueError("dst_tables names blocks outside the pool")
            uses = np.bincount(own.astype(np.int64), minlength=self.num_blocks + 1)
            if uses.max() > 1:
                raise ValueError("dst_tables names a block twice")
            # (entries of -1 look at the spare last place)
            if plan.block_tables.size and plan.block_tables.max() >= lo and uses[plan.block_tables].any():
                raise ValueError("dst_tables names a block of the batch")
            if lo < self.num_phys:
                raise ValueError(f"dst_tables names block {lo} of the block cache (private blocks start at {self.num_phys})")
        with contextlib.nullcontext() if stream is None else torch.cuda.stream(self._torch_stream(stream)):
            if torch.cuda.is_current_stream_capturing():
                raise ValueError("evict copies dst_tables from the host and cannot be captured")
            host = torch.empty(dst.shape, dtype=torch.int32, pin_memory=True)
            host.numpy()[:] = dst
            dev = host.to(self.device, non_blocking=True)
            kept = torch.empty((n, self.hkv, keep), dtype=torch.int32, device=self.device)
            kept_weights = torch.empty((n, self.hkv, keep), dtype=torch.float32, device=self.device)
        self._call("arckv_evict_select", stream, weights.data_ptr(), int(weights.shape[2]), db.seq_lens.data_ptr(), n,
                   self.hkv, keep, n_first, n_recent, kept.data_ptr(), kept_weights.data_ptr(), keep)
        args = (db.block_tables.data_ptr(), int(db.block_tables.shape[1]), kept.data_ptr(), keep, dev.data_ptr(),
                int(dst.shape[1]), n, self.num_blocks, self.hkv, self.d)
        if self.kv_format == "mx4":
            self._call("arckv_kv_compact_mx4", stream, self.kv_pool.data_ptr(), *args)
        else:
            self._call("arckv_kv_compact", stream, self.k_pool.data_ptr(), self.v_pool.data_ptr(), *args)
        return kept, kept_weights

    def step(self, token_lists, qkv_for_plan, stream=None, release: bool = True):
        """One batch: plan, upload, scatter, attend, release (release=False: the caller calls
        release()).  qkv_for_plan(plan) returns the computed tokens' (q, k_new, v_new) device
        tensors, ready on `stream`.  Returns (plan, out), out allocated on `stream`."""
        import torch
        db = self.prepare(token_lists, stream)
        plan = db.plan
        try:
            q, k_new, v_new = qkv_for_plan(plan)
            with torch.cuda.stream(self._torch_stream(stream)):
                out = torch.empty_like(q)
            self.scatter(db, k_new, v_new, stream)
            self.attention(db, q, out, stream)
        finally:
            if release:
                self.release()
        return plan, out
