"""The whole compression pass as a user calls it: phase A for every layer, the budget barrier,
phase B for every layer.  Only sequencing and buffer plumbing live here; every step is a C-ABI
call into libmeda.so (see binding.py) and nothing runs on the CPU in between."""
from __future__ import annotations

import torch

from . import binding
from .workloads import Workload


def owned_layers(n_layers: int, rank: int, world: int) -> list[int]:
    """Layers rank `rank` of `world` processes when ONE prompt is sharded by layer: round-robin, so that the
    layers a model's depth makes expensive (large budgets cluster) spread over the ranks."""
    return [l for l in range(n_layers) if l % world == rank]


def exchange_entropies(entropy: torch.Tensor, group=None) -> None:
    """The one exchange step of a layer-sharded pass (Eq. 7's softmax runs over ALL layers): `entropy` holds
    this rank's layers and zeros elsewhere; after the call every rank holds every layer's value (a sum over
    disjoint supports, so the result is exact and the same bits on every rank).  L floats: latency only."""
    import torch.distributed as dist
    if dist.is_available() and dist.is_initialized() and dist.get_world_size(group) > 1:
        dist.all_reduce(entropy, op=dist.ReduceOp.SUM, group=group)


class CompressionPass:
    """Buffers and call sequence of one prompt's pass on one GPU.

    Outputs are packed: layer l's compacted caches occupy rows [offset_l, offset_l + S_l) of
    `k_out` / `v_out` ([n_kv_heads] x rows x head_dim each), with offset_l = l * row_capacity.
    `row_capacity` bounds S_l per layer (n_tokens is always safe; a smaller value saves memory and
    makes a layer whose budget exceeds it report MEDA_ERR_WORKSPACE)."""

    def __init__(self, wl: Workload, row_capacity: int | None = None, device="cuda", n_streams: int = 8,
                 **ctx_overrides):
        self.wl = wl
        self.device = device
        # Layers are independent inside each phase, so they alternate between `n_streams` streams, each
        # with its own context (scratch memory): the short, latency-bound kernels of one layer
        # (selection, sort passes, reductions of partials) then run beside the long kernels of
        # the next instead of leaving the GPU idle.
        self.contexts = [binding.Context.for_workload(wl, **ctx_overrides) for _ in range(max(1, n_streams))]
        self.ctx = self.contexts[0]
        self.streams = [torch.cuda.Stream(device=device) for _ in self.contexts] if len(self.contexts) > 1 else []
        n, hkv, hq, w, d, L = wl.n_tokens, wl.n_kv_heads, wl.n_q_heads, wl.window, wl.head_dim, wl.n_layers
        self.cap = n if row_capacity is None else int(row_capacity)
        f32, i32 = torch.float32, torch.int32
        self.row_stats = [torch.empty((hq, w, 4), dtype=f32, device=device) for _ in self.contexts]
        self.scores = torch.empty((L, hkv, n), dtype=f32, device=device)
        self.entropy = torch.zeros(L, dtype=f32, device=device)
        self.budgets = torch.zeros((L, 3), dtype=i32, device=device)
        self.k_out = torch.empty((L, hkv, self.cap, d), dtype=wl.torch_dtype, device=device)
        self.v_out = torch.empty((L, hkv, self.cap, d), dtype=wl.torch_dtype, device=device)
        self.counts = torch.empty((L, hkv, self.cap), dtype=i32, device=device)
        self.idx_c = torch.empty((L, hkv, self.cap), dtype=i32, device=device)

    def close(self):
        for c in self.contexts:
            c.close()

    def check(self):
        """Synchronises and raises if any context recorded a device-side error."""
        torch.cuda.synchronize()
        for c in self.contexts:
            c.check()

    def launch_count(self) -> int:
        return sum(c.launch_count() for c in self.contexts)

    def _fork(self, main):
        ev = torch.cuda.Event()
        ev.record(main)
        for s in self.streams:
            s.wait_event(ev)

    def _join(self, main):
        for s in self.streams:
            ev = torch.cuda.Event()
            ev.record(s)
            main.wait_event(ev)

    def run(self, q_layers, k_layers, v_layers, stream=None, single_stream=False, qk_ready=None, v_ready=None,
            budgets_done=None, layer_done=None, max_lanes=None, layer_shard=None, exchange=None):
        """Enqueues the whole pass.  Inputs are lists of per-layer device tensors; results stay on the
        device in this object's buffers.  The work is ordered after what `stream` (default: torch's
        current stream) holds and `stream` waits for all of it.  With `single_stream` everything goes to
        `stream` through the first context (used when every launch is timed on its own).  `qk_ready` /
        `v_ready`: optional per-layer events after which a layer's (queries, keys) / values are in
        place (copies still in flight on another stream): phase A of a layer waits for the first,
        phase B for the second.  `budgets_done` (an event) is recorded once the budgets are written,
        `layer_done[l]` (events) once layer l's compressed cache is: a caller can start copying results
        out while later layers are still being compressed.  `max_lanes` limits the streams used.
        `layer_shard=(rank, world)`: this process runs only the layers `owned_layers` deals it (the other
        entries of the input lists are not read and may be None); the L entropies are exchanged between the
        two phases, so every rank computes the same budgets, and each rank's outputs hold its own layers
        only.  `exchange` replaces the collective (a callable taking the entropy tensor; used to emulate the
        other ranks on one GPU)."""
        L = self.wl.n_layers
        mine = list(range(L)) if layer_shard is None else owned_layers(L, *layer_shard)
        main = stream if stream is not None else torch.cuda.current_stream()
        if single_stream or not self.streams:
            lanes = [(self.contexts[0], main, self.row_stats[0])]
        else:
            lanes = list(zip(self.contexts, self.streams, self.row_stats))
            if max_lanes is not None:
                lanes = lanes[: max(1, max_lanes)]
            self._fork(main)
        if layer_shard is not None:
            with torch.cuda.stream(main):
                self.entropy.zero_()                  # the other ranks' layers must read as zero in the exchange
            if len(lanes) > 1:
                self._fork(main)
        for i, l in enumerate(mine):
            c, s, rs = lanes[i % len(lanes)]
            if qk_ready is not None:
                s.wait_event(qk_ready[l])
            c.window_scores(l, q_layers[l], k_layers[l], rs, self.scores[l], self.entropy, s)
        if len(lanes) > 1:
            self._join(main)
        if layer_shard is not None:
            with torch.cuda.stream(main):
                (exchange or exchange_entropies)(self.entropy)
        self.ctx.allocate_budgets(self.entropy, self.budgets, main)      # Eq. 7 needs every layer's entropy
        if budgets_done is not None:
            budgets_done.record(main)
        if len(lanes) > 1:
            self._fork(main)
        for i, l in enumerate(mine):
            c, s, _ = lanes[i % len(lanes)]
            if v_ready is not None:
                s.wait_event(v_ready[l])
            c.compress_layer(l, k_layers[l], v_layers[l], self.scores[l], self.budgets, self.k_out[l], self.v_out[l],
                             self.counts[l], self.idx_c[l], self.cap, s)
            if layer_done is not None:
                layer_done[l].record(s)
        if len(lanes) > 1:
            self._join(main)

    def capture(self, q_layers, k_layers, v_layers):
        """Records the whole pass (every launch of `run` on these buffers) into a CUDA graph, after one
        ordinary run that loads the kernels.  `replay()` then enqueues the pass with a single graph
        launch: no per-kernel launch cost on the host and shorter gaps between kernels on the device.
        Returns the number of kernels in the graph."""
        self.run(q_layers, k_layers, v_layers)
        torch.cuda.synchronize()
        before = self.launch_count()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.run(q_layers, k_layers, v_layers)
        self.graph = graph
        self.graph_kernels = self.launch_count() - before
        return self.graph_kernels

    def replay(self):
        """Enqueues the captured pass on torch's current stream."""
        self.graph.replay()

    def run_from_host(self, q_host, k_host, v_host, staging, out_host):
        """End-to-end variant: per-layer inputs in pinned HOST memory are copied to the device
        staging buffers, the pass runs, and the budgets plus the compacted caches (only the S_l live
        rows of each layer) are copied back to pinned host memory: out_host[name][l] has S_l rows per
        head (see `alloc_host_outputs`).  Returns (h2d_bytes, d2h_bytes)."""
        L = self.wl.n_layers
        h2d = 0
        # Copies run on their own stream, queries and keys of every layer first (phase A needs only
        # those), then the values; each layer's kernels wait for that layer's copies only, so the pass
        # overlaps with the transfer instead of following it.
        main = torch.cuda.current_stream()
        if not hasattr(self, "_copy_stream"):
            self._copy_stream = torch.cuda.Stream(device=self.device)
        cs = self._copy_stream
        cs.wait_stream(main)
        qk_ready, v_ready = [], []
        with torch.cuda.stream(cs):
            for l in range(L):
                for src, dst in ((q_host[l], staging["q"][l]), (k_host[l], staging["k"][l])):
                    dst.copy_(src, non_blocking=True)
                    h2d += src.numel() * src.element_size()
                ev = torch.cuda.Event()
                ev.record(cs)
                qk_ready.append(ev)
            for l in range(L):
                staging["v"][l].copy_(v_host[l], non_blocking=True)
                h2d += v_host[l].numel() * v_host[l].element_size()
                ev = torch.cuda.Event()
                ev.record(cs)
                v_ready.append(ev)
        budgets_done = torch.cuda.Event()
        layer_done = [torch.cuda.Event() for _ in range(L)]
        self.run(staging["q"], staging["k"], staging["v"], qk_ready=qk_ready, v_ready=v_ready,
                 budgets_done=budgets_done, layer_done=layer_done, max_lanes=4)
        # Results leave on a third stream: the budgets as soon as they exist (the live row counts decide
        # what comes back), then each layer's compacted cache as soon as that layer is done, while the
        # values of later layers are still arriving (the link carries both directions at once).
        if not hasattr(self, "_down_stream"):
            self._down_stream = torch.cuda.Stream(device=self.device)
        ds = self._down_stream
        with torch.cuda.stream(ds):
            ds.wait_event(budgets_done)
            out_host["budgets"].copy_(self.budgets, non_blocking=True)
            ds.synchronize()
            d2h = self.budgets.numel() * 4
            for l in range(L):
                s = int(out_host["budgets"][l, 0])
                ds.wait_event(layer_done[l])
                for name, src in (("k", self.k_out), ("v", self.v_out), ("counts", self.counts), ("idx", self.idx_c)):
                    out_host[name][l].copy_(src[l][:, :s], non_blocking=True)
                    d2h += src[l][:, :s].numel() * src.element_size()
        main.wait_stream(ds)
        main.synchronize()
        return h2d, d2h

    def alloc_host_outputs(self):
        """Pinned host buffers sized by the budgets of the last run (budgets are a deterministic
        function of the inputs, so a repeated run of the same prompt fits them exactly)."""
        b = self.budgets.cpu()
        wl = self.wl
        out = dict(budgets=torch.empty_like(b).pin_memory(), k=[], v=[], counts=[], idx=[])
        for l in range(wl.n_layers):
            s = int(b[l, 0])
            out["k"].append(torch.empty((wl.n_kv_heads, s, wl.head_dim), dtype=wl.torch_dtype).pin_memory())
            out["v"].append(torch.empty((wl.n_kv_heads, s, wl.head_dim), dtype=wl.torch_dtype).pin_memory())
            out["counts"].append(torch.empty((wl.n_kv_heads, s), dtype=torch.int32).pin_memory())
            out["idx"].append(torch.empty((wl.n_kv_heads, s), dtype=torch.int32).pin_memory())
        return out


class PagedDecoder:
    """Decoding of many requests over their compressed caches, kept in one pool of pages.

    Sequence `layer * max_requests + request` is one layer of one request, so a layer's batch is a run of
    table rows.  `admit` moves what a CompressionPass left into pages, `begin_step` makes room for one row per layer
    and active request, `attend` (once per layer) rotates and appends the new rows and attends, `release` gives
    a request's pages back.  Everything runs on torch's current stream; nothing is copied to the host, so
    begin_step and the layers' attend calls can be captured into a CUDA graph (the lengths live on the device).
    A request that cannot get its row keeps what it has: see begin_step.

    `keep_pages` > 0: attention reads at most that many pages per sequence and KV head, the ones whose key
    bounds promise the largest logits, the first and the last always among them."""

    def __init__(self, wl: Workload, n_pages: int, max_requests: int, max_rows: int, page_size: int = 16,
                 keep_pages: int = 0, n_first: int = 1, n_last: int = 2, rope_theta: float = 10000.0, rope_sections=None,
                 rope_order: int = 0, rope_pairing: int = 0, device="cuda"):
        L, R, hkv, d = wl.n_layers, int(max_requests), wl.n_kv_heads, wl.head_dim
        self.wl, self.n_layers, self.max_requests = wl, L, R
        self.keep_pages, self.n_first, self.n_last = int(keep_pages), n_first, n_last
        if self.keep_pages < 0 or n_first < 0 or n_last < 0 or (self.keep_pages and n_first + n_last > self.keep_pages):
            raise ValueError("keep_pages has to hold the n_first first and the n_last last pages")
        width = -(-int(max_rows) // page_size)
        with torch.cuda.device(device):
            self.pages = binding.Pages(n_q_heads=wl.n_q_heads, n_kv_heads=hkv, head_dim=d, dtype=wl.dtype, page_size=page_size,
                                       n_pages=n_pages, max_seqs=L * R, max_seq_pages=width, rope_theta=rope_theta,
                                       rope_sections=rope_sections, rope_order=rope_order, rope_pairing=rope_pairing)
        i32 = dict(dtype=torch.int32, device=device)
        dt = dict(dtype=wl.torch_dtype, device=device)
        self.k_pages = torch.empty((n_pages, hkv, page_size, d), **dt)
        self.v_pages = torch.empty((n_pages, hkv, page_size, d), **dt)
        self.bounds = torch.empty((n_pages, hkv, 2, d), **dt) if self.keep_pages else None
        self.table = torch.full((L * R, width), -1, **i32)
        self.lens = torch.zeros(L * R, **i32)              # rows of every sequence
        self.lens_before = torch.zeros(L * R, **i32)       # ... before the step in progress
        self.free_pages = torch.arange(n_pages, **i32)
        self.free_top = torch.zeros(1, **i32)
        self.active = torch.zeros(R, **i32)                # 1: the request takes part in the next step
        self._added = torch.zeros(L * R, **i32)            # rows of every sequence that the last step added
        self.advanced = self._added[:R]                    # 1: the request got a row in the last step (in every layer: they grow together)
        self._stalled = torch.zeros(R, dtype=torch.bool, device=device)    # active requests that got none in it
        self._top_out = torch.zeros(1, **i32)
        self._cu = torch.zeros(L * R + 1, **i32)
        self._new_slots = torch.empty(L * R + 1, dtype=torch.int64, device=device)
        self._no_slots = torch.empty(0, dtype=torch.int64, device=device)
        self.slots = torch.full((L, R), -1, dtype=torch.int64, device=device)
        self.q_rot = torch.zeros((R, wl.n_q_heads, d), **dt)
        self.sel = torch.empty((R, hkv, self.keep_pages), **i32) if self.keep_pages else None

    def close(self):
        self.pages.close()

    def check(self):
        """Synchronises and raises if a device-side error was recorded (a full pool among them) or an active request got no row in
        the last step (the error names them)."""
        status = self.pages.poll_status()
        stalled = self._stalled.nonzero().flatten().tolist()
        self._stalled.zero_()
        if stalled:
            raise binding.MedaError(status or binding.MEDA_ERR_WORKSPACE, f"no room for another row of requests {stalled}")
        binding._check(status, "device status")

    def _move(self, new_lens, slots):
        """Page tables for lens -> new_lens.  A change the pool cannot serve is recorded and changes nothing."""
        self.pages.page_tables(self.lens, new_lens, self.free_pages, self.free_top, self._top_out, self.table, self._cu, slots)
        self.free_top.copy_(self._top_out)

    def _check_request(self, request: int):
        if not 0 <= request < self.max_requests:
            raise IndexError(f"request {request} of {self.max_requests}")

    def admit(self, request: int, cp: CompressionPass):
        """The compacted caches of `cp` (all layers) become request `request`, whose earlier pages are given back.  Caches of another
        number of layers, KV heads, head size, type or device are refused (ValueError); budgets that the pool or the buffers
        of `cp` (its row_capacity) cannot serve are recorded for check(), and the request stays empty."""
        L, R = self.n_layers, self.max_requests
        self._check_request(request)
        _, hkv, _, d = self.k_pages.shape
        for x in (cp.k_out, cp.v_out):
            if x.shape[:2] != (L, hkv) or x.shape[3] != d or x.dtype != self.k_pages.dtype or x.device != self.k_pages.device:
                raise ValueError(f"caches of {tuple(x.shape)} {x.dtype} on {x.device} for a decoder of [{L}][{hkv}][rows][{d}] "
                                 f"{self.k_pages.dtype} on {self.k_pages.device}")
        self.release(request)
        rows = cp.budgets[:, 0]
        over = rows > cp.cap                               # such a layer was not compacted: nothing is admitted then
        new_lens = self.lens.clone()
        new_lens.view(L, R)[:, request] = torch.where(over.any(), 0, rows)
        self._move(new_lens, self._no_slots)               # whole pages are stored: no slot map is needed
        moved = self._cu[-1] > 0                           # stays 0 when the request could not be served
        self.lens.copy_(torch.where(moved, new_lens, self.lens))
        held = torch.where(moved | over, rows, 0).to(torch.int32)      # (page_store records a layer with too many rows, and skips it)
        table = self.table.view(L, R, -1)[:, request].contiguous()
        self.pages.page_store(cp.k_out, cp.v_out, held, table, self.k_pages, self.v_pages, self.bounds)
        self.active[request:request + 1] = moved.to(torch.int32)

    def release(self, request: int):
        """Gives the request's pages back.  Layers of a step in progress that are still to come append nothing of it."""
        self._check_request(request)
        new_lens = self.lens.clone()
        new_lens.view(self.n_layers, self.max_requests)[:, request] = 0
        self._move(new_lens, self._no_slots)
        self.lens.copy_(new_lens)
        self.active[request] = 0
        self.slots[:, request] = -1                        # its pages may be another's before the step ends
        self._stalled[request] = False

    def begin_step(self):
        """Room for one more row in every layer of the active requests.  A request with a layer that is full (max_rows, up to the end of
        its last page) gets none and leaves the others alone; when the pool has too few pages for the rest, nobody gets any, and
        the step can be begun again once a request has left.  `advanced` [R] is 1 for the requests that got their rows.  The query
        of an active one that did not is NaN for this step, and so are its outputs; check() raises for it."""
        L, R = self.n_layers, self.max_requests
        self.lens_before.copy_(self.lens)
        lens = self.lens.view(L, R)
        room = lens.amax(0) < self.table.shape[1] * self.pages.cfg.page_size
        self._move((lens + self.active * room).view(-1), self._new_slots)
        torch.sub(self._cu[1:], self._cu[:-1], out=self._added)            # all 0 when the pool has run out: nothing is appended then
        self.lens.add_(self._added)
        slots = self.slots.view(-1)
        torch.index_select(self._new_slots, 0, self._cu[:-1], out=slots)   # (behind the last sequence cu is at most L * R)
        slots.masked_fill_(self._added == 0, -1)
        torch.gt(self.active, self.advanced, out=self._stalled)
        self.q_rot.masked_fill_(self._stalled[:, None, None], float("nan"))    # attend leaves the rows of tokens without a slot alone

    def attend(self, layer: int, q, k, v, positions, out, lse=None):
        """One layer of the step: q [R][Hq][d], k, v [R][Hkv][d] (any token stride) of the new tokens, positions int32
        [3][R]; out [R][Hq][d], lse fp32 [R][Hq].  Rows of requests that were not active when the step began (or have been
        released or admitted since) attend to what they hold, with the query of an earlier call; their outputs mean nothing."""
        R = self.max_requests
        rows = slice(layer * R, (layer + 1) * R)
        table, lens = self.table[rows], self.lens[rows]
        self.pages.rope_append(q, k, v, positions, self.slots[layer], self.q_rot, self.k_pages, self.v_pages)
        if self.keep_pages:
            self.pages.page_bounds(self.k_pages, table, self.lens_before[rows], lens, self.bounds)
            self.pages.select_pages(self.q_rot, self.bounds, table, lens, self.n_first, self.n_last, self.sel)
        self.pages.paged_attention(self.q_rot, self.k_pages, self.v_pages, table, lens, out, lse, sel=self.sel)
