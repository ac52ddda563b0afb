"""Multi-step synthetic decode loop: verification steps chained through the KV commit.

Iterative tree decoding (Preliminaries): every step verifies one drafted tree against the prefix,
keeps the accepted path plus one corrected / bonus token, appends the kept tokens' keys and values
to the prefix cache, and repeats until the whole image sequence is formed.  There is no model here:
each step's tree, queries, keys, values, hidden states and uniforms come from a pool of seeded
synthetic step inputs (``workloads.make_config``) that is cycled through, which stands in for a
stochastic drafter and the target's forward pass.  What is real is the chain: the prefix grows by
what the walk accepted, so attention reads what earlier steps committed.

``PagedLoop`` is the same chain for a batch of prompts whose prefixes lie in pages: prompts arrive in chunks, steps verify trees or draw
one token per prompt, and rows take pages as they grow; rows may begin with the pages of another one, and may be held to a budget.

Host logic only; every computation runs in the library's kernels.
"""
from __future__ import annotations

import dataclasses
import time
from typing import List, Optional

import torch

from . import binding


@dataclasses.dataclass
class LoopResult:
    steps: int
    tokens: int                      # emitted tokens (accepted + one correction / bonus per step)
    accept_lens: List[int]
    tvd_used: List[float]
    emitted: List[List[int]]
    seconds: float
    records: Optional[list] = None   # per-step device outputs (only when record=True)

    @property
    def mean_accept_len(self) -> float:
        return sum(self.accept_lens) / max(len(self.accept_lens), 1)

    @property
    def tvd_per_image(self) -> float:
        return float(sum(self.tvd_used))


class DecodeLoop:
    """One prompt (with its guidance row, if any) decoded for ``image_tokens`` tokens."""

    LAG = 2          # steps the host's knowledge of the accepted lengths may trail the device
    RING = 4         # pinned read-back slots (> LAG)

    def __init__(self, pool, image_tokens: int, device: str = "cuda:0", packed_w: bool = True,
                 cfg_mix: int = binding.CFG_MIX_LOGITS):
        first = pool[0]
        if any(p.n_prompts != 1 for p in pool):
            raise ValueError("the decode loop drives one prompt")
        for p in pool[1:]:
            same = (p.dtype, p.cfg, p.n_heads, p.n_kv_heads, p.head_dim, p.hidden, p.vocab) == \
                   (first.dtype, first.cfg, first.n_heads, first.n_kv_heads, first.head_dim, first.hidden, first.vocab)
            if not same:
                raise ValueError("pool entries must share the model shape")
        self.pool = pool
        self.image_tokens = image_tokens
        self.dev = torch.device(device)
        self.dt = torch.bfloat16 if first.dtype == "bf16" else torch.float32
        self.max_depth = max(p.max_depth for p in pool)
        self.max_tree = max(p.n_nodes for p in pool)
        S, P0 = first.n_rows, int(first.prefix_len.max())
        # room for the initial prefix, the image, and the last step's overshoot
        # (the pipelined loop runs up to LAG further steps before it learns that the image is complete)
        self.cap = -(-(P0 + image_tokens + (self.LAG + 1) * (self.max_depth + 1) + 1) // 8) * 8
        self.steps = [binding.DeviceStep(p, device) for p in pool]
        for st in self.steps:
            st.cfg_mix = cfg_mix           # where the projection takes the guidance mix (honoured for packed bf16 weights)
        self.ctx = binding.Context(max_rows=S, max_nodes_total=self.max_tree * S, max_nodes_per_tree=self.max_tree,
                                   max_prefix=self.cap, n_heads=first.n_heads, head_dim=first.head_dim,
                                   hidden=first.hidden, vocab=first.vocab)
        for st in self.steps:      # all steps share one context (one stream, one workspace) and one weight matrix
            st.ctx = self.ctx
            st.w = self.steps[0].w
        self.w_layout = binding.W_ROWMAJOR
        self.w = self.steps[0].w
        if packed_w and first.dtype == "bf16":
            self.w = binding.cascade_pack_lmhead_w(self.ctx, self.steps[0].w)
            self.w_layout = binding.W_PACKED32
        self.k_cache = torch.zeros((1, S, first.n_kv_heads, self.cap, first.head_dim), dtype=self.dt, device=self.dev)
        self.v_cache = torch.zeros_like(self.k_cache)
        self.k_cache[0, :, :, :first.prefix_cap] = self.steps[0].k_cache
        self.v_cache[0, :, :, :first.prefix_cap] = self.steps[0].v_cache
        self.prefix_len = self.steps[0].prefix_len.clone()
        self.prefix_len_next = torch.empty_like(self.prefix_len)
        self.row_prompt = torch.zeros(S, dtype=torch.int32, device=self.dev)
        self.prefix_host = int(first.prefix_len.max())
        self.h_len = torch.empty(self.RING, dtype=torch.int32, pin_memory=True)
        self.h_tvd = torch.empty(self.RING, dtype=torch.float32, pin_memory=True)
        self.h_emit = torch.empty((self.RING, self.max_depth + 1), dtype=torch.int32, pin_memory=True)
        self.done = [torch.cuda.Event() for _ in range(self.RING)]

    def _enqueue_step(self, st, mode: int, max_prefix_len: int, slot: int) -> None:
        """One verification step and its KV commit on the library's stream, then the asynchronous
        read-back of what the host needs into pinned slot `slot` and the event that marks it complete."""
        binding.tree_verify_attn(self.ctx, node_off=st.row_node_off, parent=st.row_parent, prefix_len=self.prefix_len,
                                 q=st.q, k_tree=st.k_tree, v_tree=st.v_tree, k_cache=self.k_cache[0], v_cache=self.v_cache[0],
                                 out=st.attn_out, lse=st.attn_lse, max_nodes_per_tree=st.max_tree,
                                 max_prefix_len=max_prefix_len)
        st.lmhead(self.w, self.w_layout)
        st.accept()
        st.select(mode)
        binding.kv_commit(self.ctx, node_off=st.row_node_off, row_prompt=self.row_prompt, accept_len=st.accept_len,
                          path_nodes=st.path_nodes, k_tree=st.k_tree.unsqueeze(0), v_tree=st.v_tree.unsqueeze(0),
                          k_cache=self.k_cache, v_cache=self.v_cache, prefix_len=self.prefix_len,
                          prefix_len_out=self.prefix_len_next)
        self.prefix_len, self.prefix_len_next = self.prefix_len_next, self.prefix_len
        self.h_len[slot:slot + 1].copy_(st.accept_len, non_blocking=True)
        self.h_tvd[slot:slot + 1].copy_(st.tvd_used, non_blocking=True)
        self.h_emit[slot:slot + 1, :st.emitted.shape[1]].copy_(st.emitted, non_blocking=True)
        self.done[slot].record()

    def run_pipelined(self, mode: int = binding.WALK_SEQUENTIAL) -> LoopResult:
        """The decode loop without a stream wait per step.  The prefix lengths live on the device (the
        commit writes them, the next attention reads them), so the host needs the accepted lengths only
        to know when the image is complete and how large a prefix the next launch must allow for: it
        reads them LAG steps late, passes an upper bound of the prefix (confirmed prefix + a full path
        per unconfirmed step), and discards the at most LAG steps enqueued after the image was complete."""
        accept_lens, tvds, emitted = [], [], []
        tokens, launched, confirmed = 0, 0, 0
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        complete = False
        while not complete:
            st = self.steps[launched % len(self.steps)]
            bound = self.prefix_host + (launched - confirmed) * (self.max_depth + 1)
            self._enqueue_step(st, mode, bound, launched % self.RING)
            launched += 1
            while confirmed < launched and (launched - confirmed > self.LAG or self.done[confirmed % self.RING].query()):
                slot = confirmed % self.RING
                self.done[slot].synchronize()
                a_len = int(self.h_len[slot])
                accept_lens.append(a_len)
                tvds.append(float(self.h_tvd[slot]))
                emitted.append(self.h_emit[slot, :a_len + 1].tolist())
                self.prefix_host += a_len + 1
                tokens += a_len + 1
                confirmed += 1
                if tokens >= self.image_tokens:
                    complete = True
                    break
        torch.cuda.synchronize()   # the discarded steps still run to their end
        seconds = time.perf_counter() - t0
        if self.ctx.device_status() != binding.OK:
            raise binding.CascadeError(binding.ETREE)
        return LoopResult(steps=confirmed, tokens=tokens, accept_lens=accept_lens, tvd_used=tvds, emitted=emitted,
                          seconds=seconds)

    def run(self, mode: int = binding.WALK_SEQUENTIAL, record: bool = False, max_steps: Optional[int] = None) -> LoopResult:
        accept_lens, tvds, emitted, records = [], [], [], [] if record else None
        tokens, n = 0, 0
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        while tokens < self.image_tokens and (max_steps is None or n < max_steps):
            st = self.steps[n % len(self.steps)]
            self._enqueue_step(st, mode, self.prefix_host, 0)
            # the host needs the accepted length to know how far the image has advanced: three small
            # asynchronous copies into pinned memory and one wait for the stream
            torch.cuda.current_stream().synchronize()
            a_len = int(self.h_len[0])
            accept_lens.append(a_len)
            tvds.append(float(self.h_tvd[0]))
            emitted.append(self.h_emit[0, :a_len + 1].tolist())
            if record:
                records.append(dict(pool_index=n % len(self.steps), attn_out=st.attn_out.float().cpu().numpy(),
                                    logits=st.logits.cpu().numpy(), row_thr=st.row_thr.cpu().numpy(),
                                    row_lse=st.row_lse.cpu().numpy(), accept_len=a_len,
                                    path_nodes=st.path_nodes.cpu().numpy().copy(), emitted=st.emitted.cpu().numpy().copy(),
                                    terminal=int(st.terminal.cpu()[0]), prefix_len=self.prefix_len.cpu().numpy().copy()))
            self.prefix_host += a_len + 1
            tokens += a_len + 1
            n += 1
        torch.cuda.synchronize()
        seconds = time.perf_counter() - t0
        if self.ctx.device_status() != binding.OK:
            raise binding.CascadeError(binding.ETREE)
        return LoopResult(steps=n, tokens=tokens, accept_lens=accept_lens, tvd_used=tvds, emitted=emitted, seconds=seconds,
                          records=records)


class PagedLoop:
    """A batch of prompts (with their guidance rows, if any) over a cache in pages.

    The step inputs are one synthetic record, as in ``DecodeLoop``; ``prompt_k`` / ``prompt_v`` of ``admit`` stand for what a model makes of
    the prompts' tokens.  Lengths, tables and free pages live on the device: a step needs nothing from the host but a bound of the prefix lengths.
    A row grows to ``max_len``, rounded up to whole pages; one without room, there or in the pool, stays as it is, and ``ctx.device_status()`` says so.
    Calls run on the stream that was current when the loop was made; inputs have to be ready for it.  What is given under another current stream may be
    dropped at once: its memory is not handed out again before the loop's stream has passed the call.
    ``share`` lets rows begin with the pages of another one; with ``keep_mass`` the loop sums up what attention uses of every position, and ``evict`` holds rows to a budget by it."""

    def __init__(self, inp, page_size: int = 64, n_pages: Optional[int] = None, max_len: int = 4096, max_chunk: int = 1024, device: str = "cuda:0",
                 keep_mass: bool = False):
        width = -(-max_len // page_size)
        self.inp, self.page_size, self.max_len, self.max_chunk, self.keep_mass = inp, page_size, width * page_size, max_chunk, keep_mass
        self.dev = torch.device(device)
        with torch.cuda.device(self.dev):
            self._allocate(inp, page_size, n_pages, width, max_chunk, device)

    def _allocate(self, inp, page_size, n_pages, width, max_chunk, device) -> None:
        self.step_in = binding.DeviceStep(inp, device)
        S = inp.n_rows
        self.n_pages = S * width if n_pages is None else n_pages
        self.ctx = binding.Context(max_rows=max(S, inp.n_prompts), max_nodes_total=max(inp.q.shape[0], S * max_chunk), max_nodes_per_tree=self.step_in.max_tree,
                                   max_prefix=self.max_len, n_heads=inp.n_heads, head_dim=inp.head_dim, hidden=inp.hidden, vocab=inp.vocab)
        self.step_in.ctx = self.ctx
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=self.dev)  # noqa: E731
        dt = self.step_in.q.dtype
        self.k_pages = torch.zeros((1, self.n_pages, inp.n_kv_heads, page_size, inp.head_dim), dtype=dt, device=self.dev)
        self.v_pages = torch.zeros_like(self.k_pages)
        self.block_table = i32(S, width)
        self.free_pages = torch.arange(self.n_pages - 1, -1, -1, dtype=torch.int32, device=self.dev)
        self.free_count, self.free_next = torch.full((1,), self.n_pages, dtype=torch.int32, device=self.dev), i32(1)
        self.seq_len, self.seq_next = i32(S), i32(S)
        self.row_prompt = torch.tensor([s * inp.n_prompts // S if S == inp.n_prompts else s // 2 for s in range(S)], dtype=torch.int32, device=self.dev)
        self.q_off = i32(S + 1)
        self.longest = 0                       # host bound on the rows' lengths
        self.rows = inp.n_rows
        self.admitted: Optional[List[int]] = [0] * S      # tokens that the rows were given; None once steps or evictions have changed how many are there
        self.group_off = self.shared_len = None           # what share has set, for the attention calls
        self.longest_shared = 0
        self.held = i32(S)                                # positions of each row that lie in pages of several rows
        if self.keep_mass:
            self.mass = torch.zeros((1, S, inp.n_kv_heads, self.max_len), dtype=torch.float32, device=self.dev)
            self.mass_next = torch.zeros_like(self.mass)
            self.dropped, self.gone = i32(S), i32(S)      # positions that each row has given up, in all and in the last call
            self.scratch = torch.empty(max(16, binding.paged_evict_workspace(self.ctx, **self._eviction(self.seq_len, self.held, 0))),
                                       dtype=torch.uint8, device=self.dev)

    def _keep(self, *tensors) -> None:
        """Tensors of a caller: tells the allocator that the loop's stream uses them."""
        if torch.cuda.current_stream(self.dev) != self.ctx.stream:
            for t in tensors:
                if t is not None:
                    t.record_stream(self.ctx.stream)

    def _place(self, tokens: int, **lengths):
        """Pages and slots for new tokens; the rows' lengths become those behind them."""
        slot_map, source = (torch.empty(tokens, dtype=torch.int32, device=self.dev) for _ in range(2))
        binding.paged_slots(self.ctx, seq_len=self.seq_len, block_table=self.block_table, free_pages=self.free_pages, free_count=self.free_count,
                            page_size=self.page_size, n_pages=self.n_pages, q_off=self.q_off, slot_map=slot_map, source=source, seq_len_out=self.seq_next,
                            free_count_out=self.free_next, **lengths)
        self.seq_len, self.seq_next = self.seq_next, self.seq_len
        self.free_count, self.free_next = self.free_next, self.free_count
        return slot_map, source

    def _attend(self, prefix_len, **attn) -> None:
        if self.group_off is None:
            binding.paged_attn(self.ctx, prefix_len=prefix_len, **attn)
        else:
            binding.paged_attn_shared(self.ctx, prefix_len=prefix_len, group_off=self.group_off, shared_len=self.shared_len,
                                      max_shared_len=min(self.longest_shared, attn["max_prefix_len"]), **attn)

    def _weigh(self, q, lse, before, max_new: int, source=None) -> None:
        """What the tokens that the last ``_place`` gave slots attended (behind their append); positions that cannot go are left out."""
        binding.paged_mass(self.ctx, q_off=self.q_off, seq_len=self.seq_len, block_table=self.block_table, q=q, lse=lse, k_pages=self.k_pages[0], mass=self.mass[0],
                           source=source, first=self.held, prefix_len=before, max_new=max_new, max_seq_len=self.longest)

    def share(self, group_off, positions) -> None:
        """Rows group_off[g] + 1 .. group_off[g + 1] - 1 (host lists; all rows, in order) get the first positions[g] positions of row group_off[g], in the same pages: whole
        pages that this row was admitted to.  The others must be empty, and no step or eviction may have been made.  Rows of a group give these pages back together.
        Groups are runs of rows: with guidance, whose conditional and unconditional rows alternate, there are none.  Attention reads shared pages once for a group where a call has few
        tokens to a row (up to 16 query rows to a kv head); chunks and large trees share the memory."""
        ok = (len(group_off) == len(positions) + 1 and group_off[0] == 0 and group_off[-1] == self.rows and all(a <= b for a, b in zip(group_off, group_off[1:])))
        if not ok or self.admitted is None or self.group_off is not None:
            raise ValueError(f"groups of rows {list(group_off)}, {self.rows} rows: once, for all rows in order, before the first step or eviction")
        for lo, hi, n in zip(group_off, group_off[1:], positions):
            if n < 0 or n % self.page_size or (hi - lo > 1 and (n > self.admitted[lo] or any(self.admitted[lo + 1:hi]))):
                raise ValueError(f"rows {lo} to {hi - 1} cannot share {n} positions: whole pages of {self.page_size} of what the first has, the others empty")
        with torch.cuda.stream(self.ctx.stream):
            there = []                                    # (the first row may have been refused its pages)
            for lo, hi, n in zip(group_off, group_off[1:], positions):
                pages = n // self.page_size
                n = n if hi - lo > 1 else 0
                there.append(torch.where(self.seq_len[lo] >= n, n, 0).to(torch.int32) if hi > lo else self.seq_len.new_zeros(()))
                self.block_table[lo + 1:hi, :pages] = self.block_table[lo, :pages]
                self.seq_len[lo + 1:hi] = there[-1]
                self.held[lo:hi] = there[-1]
                for s in range(lo + 1, hi):
                    self.admitted[s] = n
            self.shared_len = torch.stack(there) if there else self.seq_len.new_zeros(0)
            self.group_off = torch.tensor(list(group_off), dtype=torch.int32, device=self.dev)
        self.longest_shared = max([n for lo, hi, n in zip(group_off, group_off[1:], positions) if hi - lo > 1], default=0)

    def _eviction(self, budget, n_first, n_recent):
        return dict(seq_len=self.seq_len, budget=budget, n_first=n_first, n_recent=n_recent, block_table=self.block_table, k_pages=self.k_pages, v_pages=self.v_pages, mass=self.mass,
                    mass_out=self.mass_next, free_pages=self.free_pages, free_count=self.free_count, seq_len_out=self.seq_next, free_count_out=self.free_next,
                    dropped=self.gone, max_seq_len=self.max_len)

    def evict(self, budget, n_first: int = 0, n_recent: int = 0) -> None:
        """Rows with more than budget positions (one number, or one for each row) give up those that attention used least, each kv head its own; their last pages go back.
        The first n_first positions, those in shared pages and the last n_recent stay.  ``dropped`` counts what each row has given up."""
        if not self.keep_mass:
            raise ValueError("positions are weighed if the loop is made with keep_mass")
        budgets = [int(budget)] * self.rows if isinstance(budget, int) else [int(b) for b in budget]
        if len(budgets) != self.rows or min(budgets) < 0 or n_first < 0 or n_recent < 0:
            raise ValueError(f"budgets {budgets}, first {n_first}, recent {n_recent}: one budget, or one for each of {self.rows} rows")
        with torch.cuda.stream(self.ctx.stream):
            args = self._eviction(torch.tensor(budgets, dtype=torch.int32, device=self.dev), self.held.clamp(min=n_first), n_recent)
            binding.paged_evict(self.ctx, workspace=self.scratch, **{**args, "max_seq_len": self.longest})
            self.dropped += self.gone
        self.seq_len, self.seq_next = self.seq_next, self.seq_len
        self.free_count, self.free_next = self.free_next, self.free_count
        self.mass, self.mass_next = self.mass_next, self.mass
        self.admitted = None
        self.longest = min(self.longest, max(max(budgets), max(n_first, self.longest_shared) + n_recent))

    def admit(self, q, k_new, v_new, new_len, out, lse=None):
        """A chunk of every row's prompt, packed row by row: its attention over what is there and over itself, then its keys and values go to
        the pages.  new_len: host lengths."""
        if len(new_len) != self.rows or min(new_len) < 0 or sum(new_len) > q.shape[0] or q.shape[0] > self.ctx.limits.max_nodes_total:
            raise ValueError(f"chunks of {list(new_len)} tokens, {q.shape[0]} given: one chunk for each of {self.rows} rows, {self.ctx.limits.max_nodes_total} tokens together")
        if max(new_len) == 0:
            return
        self._keep(q, k_new, v_new, out, lse)
        with torch.cuda.stream(self.ctx.stream):
            if self.keep_mass and lse is None:
                lse = torch.empty(q.shape[:2], dtype=torch.float32, device=self.dev)
            attn = dict(q_off=self.q_off, block_table=self.block_table, q=q, k_new=k_new, v_new=v_new, k_pages=self.k_pages[0], v_pages=self.v_pages[0], out=out, lse=lse,
                        max_new=max(new_len), max_prefix_len=self.longest)
            append = dict(k_new=k_new.unsqueeze(0), v_new=v_new.unsqueeze(0), k_pages=self.k_pages, v_pages=self.v_pages)
            # what the two calls refuse they refuse before rows grow (an append of no tokens looks at everything else)
            binding.paged_attn_workspace(self.ctx, prefix_len=self.seq_len, **attn)
            binding.paged_append(self.ctx, slot_map=self.q_off[:0], **append)
            lens = torch.tensor(new_len, dtype=torch.int32, device=self.dev)
            before = self.seq_len.clone()
            slot_map, _ = self._place(q.shape[0], new_len=lens)
            self._attend(before, **attn)
            binding.paged_append(self.ctx, slot_map=slot_map, **append)
            self.longest = min(self.longest + max(new_len), self.max_len)
            if self.keep_mass:
                self._weigh(q, lse, before, max(new_len))
        if self.admitted is not None:
            self.admitted = [n + more for n, more in zip(self.admitted, new_len)]

    def step(self, mode: int = binding.WALK_SEQUENTIAL) -> None:
        """One verification step of every prompt's tree over the pages, and the commit of what it accepts to them."""
        st = self.step_in
        with torch.cuda.stream(self.ctx.stream):   # and on its device
            self._attend(self.seq_len, q_off=st.row_node_off, parent=st.row_parent, block_table=self.block_table, q=st.q, k_new=st.k_tree, v_new=st.v_tree,
                         k_pages=self.k_pages[0], v_pages=self.v_pages[0], out=st.attn_out, lse=st.attn_lse, max_new=st.max_tree, max_prefix_len=self.longest)
            st.lmhead()
            st.accept()
            st.select(mode)
            slot_map, source = self._place(self.rows * (st.max_depth + 1), node_off=st.row_node_off, row_prompt=self.row_prompt, accept_len=st.accept_len,
                                           path_nodes=st.path_nodes, n_nodes_total=st.q.shape[0])
            binding.paged_append(self.ctx, k_new=st.k_tree.unsqueeze(0), v_new=st.v_tree.unsqueeze(0), slot_map=slot_map, source=source, k_pages=self.k_pages,
                                 v_pages=self.v_pages)
            self.longest = min(self.longest + st.max_depth + 1, self.max_len)
            if self.keep_mass:
                self._weigh(st.q, st.attn_lse, self.seq_next, st.max_depth + 1, source)   # (the lengths before, until the next call)
        self.admitted = None

    def draw(self, u, token, prob=None, **parameters) -> None:
        """Plain decoding: one token of every prompt from the logits of its tree's root (of the last ``step``), with each prompt's own sampling parameters."""
        self._keep(u, token, prob, *parameters.values())
        with torch.cuda.stream(self.ctx.stream):
            roots = self.step_in.node_off[:-1].long()
            binding.sample_tokens(self.ctx, logits=self.step_in.logits.index_select(0, roots), u=u, token=token, prob=prob, **parameters)
