"""A decode service with continuous batching next to a finetune task, both on one unified pool (Harli Sec. 3-4, the
setting of the evaluation's request trace, Sec. 8.1 / 8.5).  Host orchestration only: every device step runs in
libharli's kernels; this module keeps the request queue, the page tables and the calls in order.

Requests arrive with a prompt whose KV cache is taken as given (the paper serves decode in a prefill/decode
disaggregated deployment: prefill happens elsewhere) and a number of tokens to produce.  Admission allocates the
prompt's KV pages from the pool; every decode step appends one token per running sequence, allocates a page when a
sequence crosses a page boundary and frees the pages of sequences that finish (the pool reuses them once the step
that last read them has completed).  The finetune task allocates its saved activations from the same pool and backs
off when the pool reports pressure or cannot serve it (Sec. 4.4: inference has priority).

Two options: `Sampling` draws the tokens instead of taking the most likely ones, and `KvBudget` keeps every sequence's
cache inside a number of tokens -- steps add up the attention weight each cached token receives, and when a sequence has
grown past the budget its least attended tokens leave, in every layer and KV head by its own choice, and the pages
behind the kept length go back to the pool.
"""
from __future__ import annotations

import collections
import dataclasses
import threading
import time

import numpy as np
import torch

from . import binding as hb

P = 16  # tokens per KV page


@dataclasses.dataclass(frozen=True)
class Sampling:
    """How tokens are drawn (harli_sample); the random numbers come from a generator on the device, seeded here."""
    temperature: float = 1.0
    top_k: int = 0
    top_p: float = 1.0
    min_p: float = 0.0
    seed: int = 0


@dataclasses.dataclass(frozen=True)
class KvBudget:
    """A sequence that holds `keep` + `slack` tokens is cut to `keep` (harli_kv_evict): the first `sink` and the last `recent`
    positions stay, of the others those with the most accumulated attention weight.  `keep` has room for sink + recent."""
    keep: int
    slack: int = P
    sink: int = 4
    recent: int = 64
    decay: float = 1.0

    @classmethod
    def of(cls, keep: int, **kw) -> KvBudget:
        """A budget of `keep` tokens; where that has no room for the usual sink and recent positions, half of it is for the newest ones and
        up to a quarter for the first."""
        if keep < cls.sink + cls.recent:
            kw = dict(dict(sink=min(cls.sink, keep // 4), recent=max(1, keep // 2)), **kw)
        return cls(keep, **kw)


class _SentBack(tuple):
    """The queue's (prompt, out) of a sequence that gave its pages back; `cell`: where the token is that it goes on from."""
    cell = None


class DecodeServer:
    """Continuous batching over `harli_decode_step`.  Not thread-safe: one thread drives it.  A request is a prompt's length and a number of
    tokens; its first step is fed token 0, every other one the sequence's own last token, whatever slot it has moved to and also
    after it was sent back to the queue.  A prompt arrives whole, inside a budget too, and so does a sequence that was sent back: one of
    more tokens than the pool has room for is dropped and counted in `refused`."""

    def __init__(self, ctx, pool, m, *, max_batch: int, max_len: int, stream, slab=None, sampling: Sampling | None = None,
                 budget: KvBudget | None = None):
        """slab: the pool's slab as a torch uint8 tensor; when given, the KV pages of an admitted prompt are cleared on
        the decode stream (standing in for the arrival of the prompt's cache from the prefill instance: the same
        bytes are written once).  Without it the pages keep whatever the pool last held there."""
        self.ctx, self.pool, self.m, self.stream = ctx, pool, m, stream
        self.kv_view = None
        if slab is not None:
            cfg, st = pool.cfg, pool.stats()
            page_w = P * cfg.kv_row_bytes // 8         # in 8-byte words: a byte-wise fill is eight times the work
            chunk_w = 2 * cfg.n_layers * cfg.block_bytes // 8
            self.ppb = st.pages_per_block
            self.kv_view = torch.as_strided(slab.view(torch.int64), (st.n_chunks, 2 * cfg.n_layers, self.ppb, page_w),
                                            (chunk_w, cfg.block_bytes // 8, page_w, 1), cfg.small_pool_bytes // 8)
        self.max_batch, self.max_len = max_batch, max_len
        self.max_pages = (max_len + P - 1) // P + 1
        dev = "cuda:0"
        self.table = np.full((max_batch, self.max_pages), -1, np.int32)   # host truth, updated incrementally
        self.kv = np.zeros(max_batch, np.int32)
        self.ring = [(torch.empty(max_batch, self.max_pages, dtype=torch.int32, pin_memory=True),
                      torch.empty(max_batch, dtype=torch.int32, pin_memory=True), None) for _ in range(4)]
        self.table_dev = torch.empty(max_batch, self.max_pages, dtype=torch.int32, device=dev)
        self.kv_dev = torch.empty(max_batch, dtype=torch.int32, device=dev)
        # The per-step uploads go through a stream of torch's own: for a non-blocking copy out of pinned memory torch's
        # host allocator keeps an event on the stream the copy ran on and asks for it when the buffer is freed --
        # possibly after a restricted stream handed in by the caller has been destroyed.
        self.upload = torch.cuda.Stream()
        # Tokens on the device, by cell: a slot's of the last step and of the next one (the two swap), then those of sequences that wait
        # in the queue to go on (at most max_batch: none are admitted past them), then the one that a new sequence begins with.
        self.cells = torch.zeros(3 * max_batch + 1, dtype=torch.int32, device=dev)
        with torch.cuda.stream(self.upload):
            self.cells.zero_()                 # first use now, not in the middle of a run
        self.upload.synchronize()
        self.tok, self.nxt = self.cells[:max_batch], self.cells[max_batch: 2 * max_batch]
        self.tok_at, self.first_token = 0, 3 * max_batch
        self.waiting_cells = list(range(2 * max_batch, 3 * max_batch))
        # where each slot's token comes from, when not from the slot itself
        self.source_ring = [torch.empty(max_batch, dtype=torch.int32, pin_memory=True) for _ in self.ring]
        self.source_dev = torch.zeros(max_batch, dtype=torch.int32, device=dev)
        self.fed = torch.zeros(max_batch, dtype=torch.int32, device=dev)
        self.logits = torch.empty(max_batch, m.vocab, dtype=torch.float32, device=dev)
        self.x_out = torch.empty(max_batch, m.hidden, dtype=torch.float32, device=dev)
        self.sampling, self.budget = sampling, budget
        if sampling is not None:
            self.gen = torch.Generator(dev).manual_seed(sampling.seed)
            self.uniform = torch.empty(max_batch, device=dev)
            full = lambda v, t: torch.full((max_batch,), v, dtype=t, device=dev)  # noqa: E731
            self.settings = dict(temperature=full(sampling.temperature, torch.float32), top_k=full(sampling.top_k, torch.int32),
                                 top_p=full(sampling.top_p, torch.float32), min_p=full(sampling.min_p, torch.float32))
            self.sample_ws = torch.empty(hb.sample_workspace_bytes(max_batch, m.vocab), dtype=torch.uint8, device=dev)
        if budget is not None:
            if budget.keep < 1 or budget.slack < 1:
                raise ValueError("a budget keeps at least one token and cuts at least one")
            if max_len > 1 << 18:
                raise ValueError("a budget is for sequences of at most 2^18 tokens (harli_kv_evict)")
            if budget.sink < 0 or budget.recent < 0 or not 0 <= budget.decay <= 1:
                raise ValueError("a budget's sink and recent are not negative, and its decay is 0..1")
            if budget.sink + budget.recent > budget.keep:   # the newest tokens would leave: among protected ones the lower slot stays
                raise ValueError("a budget of %d tokens cannot keep %d first and %d last ones" % (budget.keep, budget.sink, budget.recent))
            st = pool.stats()
            self.track = torch.zeros(pool.cfg.n_layers, st.n_chunks * st.pages_per_block, m.n_kv, P, 2, dtype=torch.int32, device=dev)
            self.attend_ws = torch.empty(ctx.kv_attend_workspace_bytes(max_batch, max_len), dtype=torch.uint8, device=dev)
            # per step and slot: position of the new token, tokens of a prompt that has just arrived, tokens after the step,
            # tokens to keep, position of the token after it
            self.marks = np.zeros((5, max_batch), np.int32)
            self.marks_ring = [torch.empty(5, max_batch, dtype=torch.int32, pin_memory=True) for _ in self.ring]
            self.marks_dev = torch.zeros(5, max_batch, dtype=torch.int32, device=dev)
        torch.cuda.current_stream().synchronize()   # the buffers are filled before another stream reads them
        self.evicted = 0           # tokens (of every layer and KV head alike) that have left the cache under a budget
        # per slot: [pages (list), cached tokens, tokens left, tokens it has had, just arrived, cut after this step, cell of its next token]
        self.running = []
        self.queue = collections.deque()
        self.step_no = 0
        self.last_done = None
        self.admitted = self.finished = self.kv_stalls = self.preempted = self.tokens_out = 0
        self.refused = 0           # requests, also ones sent back, that the whole pool could not hold: they leave the queue
        self._held = []            # events handed to the pool with freed pages: alive until the pool has polled them
        self.tag = None            # whatever the caller wants kept with the next step (see completed_steps)
        self._timed = collections.deque()
        self._idle = True          # no step was issued at the last call of step(): the next interval starts at its own start

    def use_stream(self, stream):
        """Later steps run on `stream` (a compute-unit partition); they still follow the steps issued so far."""
        if stream is not self.stream:
            if self.last_done is not None:
                stream.wait_event(self.last_done)
            self.stream = stream

    def submit(self, reqs):
        self.queue.extend(reqs)

    def _admit(self):
        while self.queue and len(self.running) < self.max_batch:
            prompt, out = self.queue[0]
            prompt = min(prompt, self.max_len - 2)
            out = max(1, min(out, self.max_len - 1 - prompt))
            need = (prompt + 1 + P - 1) // P
            st = self.pool.stats()
            if need > st.n_chunks * st.pages_per_block:   # not even an empty pool could take it: it must not hold up those behind it
                cell = getattr(self.queue.popleft(), "cell", None)
                if cell is not None and cell >= 2 * self.max_batch:
                    self.waiting_cells.append(cell)
                self.refused += 1
                continue
            # headroom: besides the prompt, one more page for every sequence that is running (each reaches a page
            # boundary within 16 steps); without it a pool smaller than the KV demand admits, runs out, sends a
            # sequence back to the queue and admits it again, over and over
            free_pages = (st.kv_chunks + st.free_chunks) * st.pages_per_block - st.kv_pages_live
            if self.running and need + len(self.running) > free_pages:
                self.kv_stalls += 1
                break
            try:
                ids = self.pool.alloc_pages(need)
            except hb.HarliError as e:
                if e.status != hb.HARLI_ERR_OOM:
                    raise
                self.kv_stalls += 1            # no room for this prompt now: it stays queued
                break
            cell = getattr(self.queue.popleft(), "cell", None)
            if self.kv_view is not None:       # the prompt's cache "arrives": its pages are written once
                # One fill per run of neighbouring pages, on the decode stream, and no index tensor: copying one to the
                # device would make the host wait for every step it has queued, and anything on the default stream
                # would wait for, and hold up, every restricted stream.
                with torch.cuda.stream(self.stream):
                    srt = sorted(ids)
                    k = 0
                    while k < len(srt):
                        c, s0 = divmod(srt[k], self.ppb)
                        j = k + 1
                        while j < len(srt) and srt[j] == srt[j - 1] + 1 and srt[j] // self.ppb == c:
                            j += 1
                        self.kv_view[c, :, s0:s0 + (j - k), :].zero_()
                        k = j
            b = len(self.running)
            self.table[b, :] = -1
            self.table[b, :need] = ids
            self.kv[b] = prompt
            self.running.append([list(ids), prompt, out, prompt, True, False, self.first_token if cell is None else cell])
            self.admitted += 1

    def _drop(self, b, event):
        """Frees slot b's pages (reusable once `event` has completed) and moves the last slot into its place."""
        self.pool.free_pages(self.running[b][0], event)
        if event is not None and (not self._held or self._held[-1] is not event):
            self._held.append(event)
        last = len(self.running) - 1
        if b != last:
            self.running[b] = self.running[last]
            self.table[b] = self.table[last]
            self.kv[b] = self.kv[last]
        self.running.pop()

    def step(self):
        """Admits what fits, launches one decode step for every running sequence and advances the host state.
        Returns (event recorded after the step, batch size, event recorded before it) or None when nothing is running."""
        self._admit()
        B = len(self.running)
        if B == 0:
            self._idle = True
            return None
        tb, kb, ev = self.ring[self.step_no % len(self.ring)]
        if ev is not None:
            ev.synchronize()                   # the copy that last used this staging buffer is done
        tb[:B].copy_(torch.from_numpy(self.table[:B]))
        kb[:B].copy_(torch.from_numpy(self.kv[:B]))
        source = [seq[6] for seq in self.running]
        moved = source != list(range(self.tok_at, self.tok_at + B))
        if moved:
            staged = self.source_ring[self.step_no % len(self.ring)]
            staged[:B].copy_(torch.tensor(source, dtype=torch.int32))
        if self.budget is not None:
            for b, seq in enumerate(self.running):
                after = seq[1] + 1
                seq[5] = seq[2] > 1 and after >= self.budget.keep + self.budget.slack   # (not for a sequence that ends with this step)
                self.marks[:, b] = seq[3], seq[1] if seq[4] else 0, after, self.budget.keep if seq[5] else after, seq[3] + 1
            marks = self.marks_ring[self.step_no % len(self.ring)]
            marks.copy_(torch.from_numpy(self.marks))
        if self.last_done is not None:
            self.upload.wait_event(self.last_done)   # the previous step still reads the device copies
        with torch.cuda.stream(self.upload):
            self.table_dev[:B].copy_(tb[:B], non_blocking=True)
            self.kv_dev[:B].copy_(kb[:B], non_blocking=True)
            if moved:
                self.source_dev[:B].copy_(staged[:B], non_blocking=True)
            if self.budget is not None:
                self.marks_dev.copy_(marks, non_blocking=True)
            up = torch.cuda.Event()
            up.record()
        self.stream.wait_event(up)
        start = torch.cuda.Event(enable_timing=True)
        start.record(self.stream)
        self._keep_waiting_tokens()
        if moved:
            with torch.cuda.stream(self.stream):
                torch.index_select(self.cells, 0, self.source_dev[:B], out=self.fed[:B])
        self._launch(B, int(self.kv[:B].max()) + 1, self.fed if moved else self.tok)
        done = torch.cuda.Event(enable_timing=True)
        done.record(self.stream)
        self._timed.append((start if self.last_done is None or self._idle else self.last_done, done, self.tag))
        self._idle = False
        self.last_done = done
        self.ring[self.step_no % len(self.ring)] = (tb, kb, up)
        self.tok, self.nxt = self.nxt, self.tok   # the tokens just produced feed the next step
        self.tok_at = self.max_batch - self.tok_at
        for b, seq in enumerate(self.running):
            if 2 * self.max_batch <= seq[6] < self.first_token:
                self.waiting_cells.append(seq[6])
            seq[6] = self.tok_at + b
        self.step_no += 1
        self.tokens_out += B
        if len(self._held) > 256 and self.pool.stats().pending_frees == 0:
            self._held.clear()
        # host state after the step: every sequence holds one more token
        b = 0
        while b < len(self.running):
            seq = self.running[b]
            seq[1] += 1
            seq[2] -= 1
            seq[3] += 1
            seq[4] = False
            if seq[5]:                          # cut: the pages behind the kept tokens and the next one's go back
                self.evicted += seq[1] - self.budget.keep
                seq[1] = self.budget.keep
                held = seq[1] // P + 1
                if len(seq[0]) > held:
                    self.pool.free_pages(seq[0][held:], done)
                    if not self._held or self._held[-1] is not done:
                        self._held.append(done)
                    self.table[b, held: len(seq[0])] = -1
                    del seq[0][held:]
            self.kv[b] = seq[1]
            if seq[2] == 0:
                self._drop(b, done)
                self.finished += 1
                continue                        # slot b now holds another sequence
            if seq[1] + 1 > len(seq[0]) * P:    # the next token starts a new page
                try:
                    pid = self.pool.alloc_pages(1)[0]
                    self.table[b, len(seq[0])] = pid
                    seq[0].append(pid)
                except hb.HarliError as e:
                    if e.status != hb.HARLI_ERR_OOM:
                        raise
                    # the reserve is there to prevent this; if it happens the sequence goes back to the queue
                    self.preempted += 1
                    back = _SentBack((seq[3], seq[2]))   # (as a prompt of all tokens it has had, those that left its cache too)
                    back.cell = seq[6]
                    self.queue.appendleft(back)
                    self._drop(b, done)
                    continue
            b += 1
        return done, B, start

    def _keep_waiting_tokens(self):
        """Tokens of sequences that were sent back and wait on move out of the cells that this step's slots write, on the decode stream."""
        for entry in self.queue:
            if not isinstance(entry, _SentBack):
                break                           # (they are the first in the queue)
            if entry.cell < 2 * self.max_batch:
                cell = self.waiting_cells.pop()
                with torch.cuda.stream(self.stream):
                    self.cells[cell: cell + 1].copy_(self.cells[entry.cell: entry.cell + 1])
                entry.cell = cell

    def _launch(self, B, max_kv, tokens):
        """The step's calls, in order on the decode stream."""
        step = dict(batch=B, kv_len=self.kv_dev, page_table=self.table_dev, max_pages=self.max_pages, max_kv_len=max_kv,
                    token_ids=tokens, x_out=self.x_out, logits=self.logits, next_token=None if self.sampling else self.nxt,
                    stream=self.stream)
        if self.budget is None:
            self.ctx.decode_step(**step)
        else:
            position, arrived, after, keep, following = self.marks_dev
            table = dict(batch=B, page_table=self.table_dev, max_pages=self.max_pages, track=self.track, stream=self.stream)
            if any(seq[4] for seq in self.running):
                self.ctx.kv_record_init(n_tokens=arrived, max_kv_len=max_kv, **table)
            self.ctx.decode_step_tracked(track=self.track, position=position, decay=self.budget.decay, workspace=self.attend_ws, **step)
        if self.sampling is not None:
            with torch.cuda.stream(self.stream):
                self.uniform.uniform_(generator=self.gen)
            hb.sample(self.logits[:B], self.uniform, self.nxt, workspace=self.sample_ws, stream=self.stream, **self.settings)
        if self.budget is not None and any(seq[5] for seq in self.running):
            self.ctx.kv_evict(n_tokens=after, keep=keep, max_kv_len=max_kv, sink=self.budget.sink, recent=self.budget.recent,
                              position=following, **table)

    def completed_steps(self):
        """[(tag, ms)] of the steps that have finished on the device since the last call, oldest first: `tag` is what
        `self.tag` held when the step was issued, ms the time from the end of the step before it to its own end (what a
        request sees as the time per output token: the step itself plus whatever ran on the stream before it, such as
        the arrival of admitted prompts); for the first step, its own time on the device."""
        out = []
        while self._timed and self._timed[0][1].query():
            start, done, tag = self._timed.popleft()
            out.append((tag, start.elapsed_time(done)))
        return out

    def drain(self):
        """Frees every running sequence (end of a run) and lets go of every event recorded on the decode stream, so
        that the caller may destroy that stream afterwards."""
        self.stream.synchronize()
        while self.running:
            self._drop(len(self.running) - 1, None)
        if self.pool.stats().pending_frees == 0:   # the pool has looked at every event it was given
            self._held.clear()
        self.ring = [(tb, kb, None) for tb, kb, _ in self.ring]
        self.last_done = None
        self._timed.clear()


class FinetuneWorker:
    """Host thread stepping a whole-model finetune task.  `step_fn(next_stream)` runs one training step, calling
    `next_stream()` before every layer unit (the paper's scheduling unit, Sec. 6.1) to learn which stream -- which
    compute-unit partition -- the unit goes to; it returns False when the pool could not hold the step.  `target` is the
    stream currently assigned (None: paused; `next_stream` then waits).  Units on a new stream follow the last unit
    on the old one."""

    def __init__(self, pool, step_fn, stream, tokens_per_step):
        self.pool, self.step_fn, self.T = pool, step_fn, tokens_per_step
        self.target = stream
        self.steps = self.oom = self.backoff = self.units = 0
        self.waiting = False            # True while the task has no unit ready to issue (between steps, backing off)
        self.error = None
        self._stop = threading.Event()
        self._last_stream, self._last_ev = None, None
        self.th = threading.Thread(target=self._run, daemon=True)

    def next_stream(self):
        while True:
            st = self.target
            if st is not None or self._stop.is_set():
                break
            time.sleep(1e-4)
        if st is None:
            st = self._last_stream or torch.cuda.current_stream()
        if self._last_ev is not None and st is not self._last_stream:
            st.wait_event(self._last_ev)
        return st

    def unit_done(self, st):
        """Called by step_fn after it has enqueued a unit on `st`: at most two units are in flight, so that a change of
        partition or a pause takes effect within about one unit."""
        ev = torch.cuda.Event()
        ev.record(st)
        prev = self._last_ev
        self._last_stream, self._last_ev = st, ev
        self.units += 1
        if prev is not None:
            prev.synchronize()

    def _run(self):
        try:
            torch.cuda.set_device(0)
            while not self._stop.is_set():
                if self.pool.pressure() > 0:   # inference needs the memory (Sec. 4.4): do not start a step now
                    self.backoff += 1
                    self.waiting = True
                    time.sleep(2e-3)
                    continue
                self.waiting = False
                ok = self.step_fn(self)
                if ok:
                    self.steps += 1
                else:
                    self.oom += 1
                    self.waiting = True
                    time.sleep(2e-3)
        except BaseException as e:             # noqa: BLE001 -- raised again by __exit__
            self.error = e
            self.waiting = True

    def __enter__(self):
        self.th.start()
        return self

    def __exit__(self, *a):
        self._stop.set()
        self.th.join()
        torch.cuda.synchronize()
        self._last_stream, self._last_ev = None, None
        if self.error is not None and a[0] is None:
            raise RuntimeError("the finetune thread failed") from self.error


def replay(server: DecodeServer, arrivals, worker_factory=None, slo_ms=40.0, sample_every=25, log=lambda *a: None, plan=None):
    """Drives `server` through `arrivals` (one list of requests per decode step) with, optionally, a finetune worker
    beside it.  `plan(server, worker)`, when given, is called at the beginning of every decode phase (Sec. 6.2) and may
    move the two tasks to other streams or pause the finetune task; it returns a record that is kept with the step.
    Returns counters, pool snapshots and, per decode step, the batch size, the plan's record and the time per output
    token (`tpot_ms[k]` is the time from the end of step k to the end of step k + 1; `step_ms[k]` is step k's own time
    on the device, from its first kernel to its last)."""
    pool = server.pool
    recs, snaps, plans = [], [], []
    t_start = time.perf_counter()
    box = {"worker": None}

    def run():
        pending = collections.deque()
        for t, reqs in enumerate(arrivals):
            server.submit(reqs)
            decided = plan(server, box["worker"]) if plan is not None else None
            r = server.step()
            if r is not None:
                pending.append(r)
                recs.append(r)
                plans.append(decided)
            if len(pending) > 2:
                pending.popleft()[0].synchronize()     # the host runs at most two steps ahead of the device
            if t % sample_every == 0:
                st = pool.stats()
                snaps.append({"step": t, "batch": len(server.running), "queued": len(server.queue), "free_chunks": st.free_chunks,
                              "kv_chunks": st.kv_chunks, "tensor_chunks": st.tensor_chunks,
                              "pressure": pool.pressure()})
            if t % 200 == 0:
                log("[serve] step %d of %d: batch %d, queued %d, %.1f s" % (t, len(arrivals), len(server.running), len(server.queue),
                                                                       time.perf_counter() - t_start))
        server.stream.synchronize()

    if worker_factory is not None:
        with worker_factory() as worker:
            box["worker"] = worker
            run()
        ft = {"steps": worker.steps, "oom_retries": worker.oom, "pressure_backoffs": worker.backoff, "tokens": worker.steps * worker.T}
    else:
        run()
        ft = None
    elapsed = time.perf_counter() - t_start
    tpot = np.array([recs[i][0].elapsed_time(recs[i + 1][0]) for i in range(len(recs) - 1)]) if len(recs) > 1 else np.array([0.0])
    batches = np.array([r[1] for r in recs])
    busy = np.array([r[2].elapsed_time(r[0]) for r in recs]) if recs else np.array([0.0])
    out = {"steps": len(arrivals), "decode_steps": len(recs), "elapsed_s": elapsed, "tokens_out": server.tokens_out,
           "decode_tokens_per_s": server.tokens_out / elapsed, "tpot_ms_p50": float(np.percentile(tpot, 50)),
           "tpot_ms_p99": float(np.percentile(tpot, 99)), "tpot_ms_max": float(tpot.max()), "within_slo": float(np.mean(tpot <= slo_ms)),
           "batch_mean": float(batches.mean()) if len(batches) else 0.0, "batch_max": int(batches.max()) if len(batches) else 0,
           "admitted": server.admitted, "finished": server.finished, "kv_admission_stalls": server.kv_stalls,
           "preempted": server.preempted, "refused": server.refused, "queued_at_end": len(server.queue), "tokens_evicted": server.evicted, "snapshots": snaps,
           "plans": plans if plan is not None else [], "tpot_ms": tpot, "batches": batches, "step_ms": busy}
    if ft is not None:
        ft["tokens_per_s"] = ft["tokens"] / elapsed
        out["finetune"] = ft
    return out
