"""The paged 8-bit KV cache of one LLM layer with preallocated buffers (argument marshalling only).

`VScanCache` owns the pool of blocks, the tables and the lengths (and, if asked to, the attention weight that each token has been given), so
that a decode step needs no buffers but its results and can be captured in a CUDA graph.  `VScanReducer.cache_survivors` puts the
survivors of Stage 2 into one.
"""
from __future__ import annotations

import torch

from . import binding as vb


class VScanCache:
    """kv_dtype: "e4m3" or "i8".  `batch` sequences of at most max_blocks * block_size tokens each; `rows`: the most new
    rows of a step over all sequences (their slots are kept in slot_map, their positions in row_pos).  weights: gather the attention weight
    that each cached token is given (`weight`, for `evict`); then every step that writes tokens goes through `prompt`, `step` or `weigh`.
    The calls of a cache follow each other: they go on one stream, or on streams that wait for one another."""

    def __init__(self, *, num_blocks, block_size, kv_heads, head_dim, batch, max_blocks, rows, kv_dtype="e4m3", device="cuda",
                 weights=False):
        dt = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}[kv_dtype]
        shape = (num_blocks, kv_heads, block_size, head_dim)
        self.block_size, self.batch = block_size, batch
        self.k = torch.zeros(shape, dtype=torch.uint8, device=device).view(dt)
        self.v = torch.zeros(shape, dtype=torch.uint8, device=device).view(dt)
        self.k_scale = torch.zeros((num_blocks, kv_heads), device=device)
        self.v_scale = torch.zeros((num_blocks, kv_heads), device=device)
        self.block_table = torch.full((batch, max_blocks), -1, dtype=torch.int32, device=device)
        self.free_ring = torch.arange(num_blocks, dtype=torch.int32, device=device)
        # what a step starts from and what it leaves, in two buffers of one layout: {head, tail} of the ring, lengths
        self._before = torch.zeros(16 + 4 * batch, dtype=torch.uint8, device=device)
        self._after = torch.zeros_like(self._before)
        self._past_state, self._past_len = self._views(self._before)
        self._plan = {"row_offset": torch.zeros(batch + 1, dtype=torch.int32, device=device),
                      "slot_map": torch.full((rows,), -1, dtype=torch.int64, device=device),
                      "row_pos": torch.full((rows,), -1, dtype=torch.int32, device=device),
                      "report": torch.zeros(4, dtype=torch.int32, device=device)}
        self._plan["ring_state_out"], self._plan["kv_len"] = self._views(self._after)
        self._plan["ring_state_out"][1] = num_blocks
        self._workspace, self._outgrown = None, []
        self.weight = torch.zeros(shape[:3], device=device) if weights else None
        self._delta = torch.zeros(batch, dtype=torch.int32, device=device)
        self._spaces = {}                                # of the other calls that need one, as _workspace

    @staticmethod
    def _views(buf):
        return buf[:16].view(torch.int64), buf[16:].view(torch.int32)

    kv_len = property(lambda self: self._plan["kv_len"])
    row_offset = property(lambda self: self._plan["row_offset"])
    slot_map = property(lambda self: self._plan["slot_map"])
    row_pos = property(lambda self: self._plan["row_pos"])
    report = property(lambda self: self._plan["report"])
    arrays = property(lambda self: (self.k, self.v, self.k_scale, self.v_scale))

    def plan(self, new_len):
        """new_len [batch] int32 on the GPU: tokens that each sequence gets, or loses where it is negative (a sequence that
        ends: minus its length).  `report` says whether the step could be planned; if not, nothing changes."""
        self._before.copy_(self._after)
        vb.vscan_kv_plan(self._past_len, new_len, self.block_table, self.free_ring, self._past_state, self.block_size, out=self._plan)

    def _take_back(self):
        """The last plan undone, for a step whose rows are refused afterwards: lengths and ring as before it, no new rows.  The blocks
        that it took lie in front of the ring's head again, those that it put back behind its tail."""
        self._after.copy_(self._before)
        self.row_offset.zero_()

    def write(self, k, v):
        """The new rows of the planned step, packed [rows, kv_heads, head_dim] or padded [batch, kv_heads, rows, head_dim]."""
        vb.vscan_kv_write(k, v, self.kv_len, self.row_offset, self.block_table, *self.arrays)

    def _larger(self, former, work):
        """One workspace serves all calls of a kind: the largest so far.  One that is too small stays where it is, since captured graphs may
        write to it; each is at least twice as large as the one before, so these are less than the last one together."""
        if former is not None:
            work.reserve(2 * former.nbytes)
            self._outgrown.append(former)
            if not (former.buf.is_cuda and torch.cuda.is_current_stream_capturing()):
                former.buf[:4].zero_()           # from here on it says what such graphs leave there
        work.buf[:4].zero_()
        return work

    def _grow(self, q, max_q_len):
        self._workspace = self._larger(self._workspace, vb.vscan_kv_attention_workspace(q, self.block_table, self.k, max_q_len))

    def _in_space(self, kind, make, call):
        """call(workspace) with the workspace of this kind, or a larger one from make() where it is too small."""
        if kind not in self._spaces:
            self._spaces[kind] = self._larger(None, make())
        try:
            return call(self._spaces[kind])
        except vb.VScanError as e:
            if e.status != vb.ERR_WORKSPACE:
                raise
        self._spaces[kind] = self._larger(self._spaces[kind], make())
        return call(self._spaces[kind])

    def attend(self, q, scale, max_q_len=1, causal=True, out=None, lse=None):
        """Attention of the planned step's new rows (vb.vscan_kv_attention).  -> out."""
        if out is None:
            out = torch.zeros_like(q)
        if self._workspace is None:
            self._grow(q, max_q_len)
        args = (q, self.kv_len, self.row_offset, self.block_table, *self.arrays, scale, max_q_len, causal, out, lse)
        try:
            return vb.vscan_kv_attention(*args, workspace=self._workspace)
        except vb.VScanError as e:
            if e.status != vb.ERR_WORKSPACE:
                raise
        self._grow(q, max_q_len)
        return vb.vscan_kv_attention(*args, workspace=self._workspace)

    def weigh(self, q, lse, scale, max_q_len=1, decay=1.0, window=None, causal=True):
        """The planned step's attention weights gathered for each cached token (vb.vscan_kv_weigh), from its queries and what the
        attention left in lse."""
        vb.vscan_kv_weigh(q, lse, self.kv_len, self.row_offset, self.block_table, self.k, self.k_scale, self.weight, scale, max_q_len, decay,
                          window, causal)

    def evict(self, budget, max_keep, keep_first=0, keep_last=0, per_head=True, kept=None):
        """Of each sequence the `budget` [batch] tokens (int32 on the GPU, none counts for more than max_keep) of the most weight stay, among
        them the first and last ones; the blocks left over go back to the ring (vb.vscan_kv_evict and a plan, which leaves no new rows).
        -> minus the number of tokens that left, [batch] int32, until the next call."""
        self._in_space("evict", lambda: vb.vscan_kv_evict_workspace(self.block_table, self.k, max_keep, per_head),
                       lambda work: vb.vscan_kv_evict(self.kv_len, budget, self.block_table, self.weight, *self.arrays, max_keep, keep_first,
                                                      keep_last, per_head, weight_out=self.weight, kept=kept, delta=self._delta, workspace=work))
        self.plan(self._delta)
        return self._delta

    def prompt(self, q, k, v, pos_ids, rope, new_len, scale, pairing=vb.ROPE_HALVES, window=None, out=None):
        """A layer's whole prompts: rotary positions on q and k (rope = (inv_freq, axis)), causal attention from K and V as they are
        (vb.vscan_attention), plan and write; with weights, those that the last `window` rows give (None: all).  q, k, v [batch, heads, rows,
        head_dim] padded, pos_ids [planes, batch, rows], new_len at most `rows`; the cache's sequences must be empty.  -> attention, like q.
        If a tensor is refused, lengths and tables are as they were."""
        q, k = vb.vscan_rope(q, k, pos_ids, *rope, pairing=pairing)
        self.plan(new_len)
        try:
            out = torch.zeros_like(q) if out is None else out
            lse = torch.empty(q.shape[:-1], device=q.device) if self.weight is not None else None
            top = q.shape[2]
            self._in_space("prompt", lambda: vb.vscan_attention_workspace(q, k, self.row_offset, top),
                           lambda work: vb.vscan_attention(q, k, v, self.row_offset, scale, top, out=out, lse=lse, workspace=work))
            self.write(k, v)
            if lse is not None:
                self.weigh(q, lse, scale, max_q_len=top, window=window)
            return out
        except Exception:
            self._take_back()
            raise

    def step(self, q, k, v, pos_ids, rope, new_len, scale, pairing=vb.ROPE_HALVES, out=None, decay=1.0):
        """One step of a layer: rotary positions on q and k (rope = (inv_freq, axis)), plan, write, causal attention; with weights, those
        that the step gives, beside `decay` times the older ones.  q, k, v [batch, heads, rows, head_dim] padded, pos_ids [planes, batch, rows],
        new_len at most `rows`.  -> attention of the new rows, like q.  If a tensor is refused, lengths and tables are as they were."""
        q, k = vb.vscan_rope(q, k, pos_ids, *rope, pairing=pairing)
        self.plan(new_len)
        try:
            self.write(k, v)
            if self.weight is None:
                return self.attend(q, scale, max_q_len=q.shape[2], out=out)
            lse = torch.empty(q.shape[:-1], device=q.device)
            out = self.attend(q, scale, max_q_len=q.shape[2], out=out, lse=lse)
            self.weigh(q, lse, scale, max_q_len=q.shape[2], decay=decay)
            return out
        except Exception:
            self._take_back()
            raise

    def check(self):
        """Synchronises and gives the status of the last attention, prompt and eviction calls (0, or that a block or a length was out of
        range; so of the last replay of a graph that was captured before a larger call), and the code of the last plan."""
        spaces = [w for w in (self._workspace, *self._outgrown, *self._spaces.values()) if w is not None]
        return max([vb.vscan_check(w) for w in spaces], default=0), int(self.report[0])
