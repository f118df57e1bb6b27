"""Device buffers of one attention layer and the call sequence of a decode step.

Plumbing only (allocation and slicing): everything that touches tokens is a call
into libkvr through `binding`.
"""
from __future__ import annotations

import torch

from . import binding as kvr


def _zeros(dev, *shapes):
    """Zero-filled tensors [(shape, dtype), ...], each with a storage of its own, filled by one launch."""
    out = [torch.empty(shape, dtype=dt, device=dev) for shape, dt in shapes]
    torch._foreach_zero_([x.view(torch.int32) for x in out if x.numel()])
    return out


class LayerState:
    """All per-unit buffers of one layer, unit-major [B, Hkv, ...]."""

    def __init__(self, desc, *, n_recent, k_candidate, ret_cap, vague_cap, n_cap, evict_cap=8,
                 device="cuda", ws_attend=None, ws_encode=None, n_ctx=None, slack=0, side=None, empty_slots=True):
        """n_recent, k_candidate: R.budget and C.budget of Algorithm 3; slack: its Slack (the
        Recent queue may outgrow its budget by that many tokens before slack + 1 of them leave at
        once; needs ret_cap >= n_recent + k_candidate + slack + 1 and evict_cap >= slack + 1);
        side: a binding.SideStream lent to every attend call (None: kernels back to back);
        empty_slots: start with every retained slot empty (False: the caller fills k_ret, v_ret and
        ret_pos itself)."""
        self.desc = desc
        self.n_recent, self.k_candidate = int(n_recent), int(k_candidate)
        self.slack = int(slack)
        self.side = side
        self.k_turned = self.q_turned = None
        # R.size after the last update; the queue itself is "the r_size newest positions"
        self.r_size = self.n_recent
        self.ret_cap, self.vague_cap, self.n_cap, self.evict_cap = int(ret_cap), int(vague_cap), int(n_cap), int(evict_cap)
        B, Hkv, Hq, D = desc.batch, desc.n_kv_heads, desc.n_q_heads, desc.head_dim
        dt = torch.float32 if desc.dtype == kvr.KVR_F32 else torch.bfloat16
        dev = torch.device(device)
        self.device, self.dtype = dev, dt
        slots = torch.zeros if empty_slots else torch.empty
        self.k_ret = slots(B, Hkv, self.ret_cap, D, dtype=dt, device=dev)
        self.v_ret = slots(B, Hkv, self.ret_cap, D, dtype=dt, device=dev)
        self.ret_pos = torch.empty(B, Hkv, self.ret_cap, dtype=torch.int32, device=dev)
        if empty_slots:
            self.ret_pos.fill_(-1)
        i32, f32 = torch.int32, torch.float32
        (self.scores, self.sketch_k, self.sketch_v, self.vague_pos, self.n_vague, self.evict_slot, self.evict_pos,
         self.n_evict, self.out) = _zeros(
            dev, ((B, Hkv, self.n_cap), f32), ((B, Hkv, desc.r, desc.w, D), dt), ((B, Hkv, desc.r, desc.w, D), dt),
            ((B, Hkv, self.vague_cap), i32), ((B, Hkv), i32), ((B, Hkv, self.evict_cap), i32),
            ((B, Hkv, self.evict_cap), i32), ((B, Hkv), i32), ((B, Hq, D), f32))
        # several layers may share one n_ctx tensor and one workspace (calls on one
        # stream are ordered, and no workspace content outlives a call)
        self.n_ctx = torch.zeros(B, dtype=torch.int32, device=dev) if n_ctx is None else n_ctx
        self.ws_attend = ws_attend if ws_attend is not None else kvr.alloc_workspace(
            desc, kvr.KVR_OP_ATTEND, self.ret_cap, self.vague_cap, dev)
        self.ws_encode = ws_encode if ws_encode is not None else kvr.alloc_workspace(
            desc, kvr.KVR_OP_ENCODE, self.evict_cap, 0, dev)

    # -- the four calls of a decode step, on this layer's buffers ---------------
    def append(self, k_new, v_new):
        kvr.kvr_append(self.desc, k_new, v_new, self.n_ctx, self.k_ret, self.v_ret, self.ret_pos,
                       self.ret_cap)

    def select(self):
        kvr.kvr_select(self.desc, self.scores, self.n_cap, self.ret_pos, self.ret_cap, self.n_ctx,
                       self.r_size, self.k_candidate, self.evict_slot, self.evict_pos, self.n_evict,
                       self.evict_cap, self.vague_pos, self.n_vague, self.vague_cap)

    def encode(self):
        kvr.kvr_encode(self.desc, self.k_ret, self.v_ret, self.ret_cap, self.evict_slot, self.evict_pos,
                       self.n_evict, self.evict_cap, self.sketch_k, self.sketch_v, None, None,
                       self.ws_encode)

    def attend(self, q, accumulate_scores=True, opts=None):
        kvr.kvr_attend_decode(self.desc, q, self.k_ret, self.v_ret, self.ret_pos, self.ret_cap,
                              self.sketch_k, self.sketch_v, self.vague_pos, self.n_vague, self.vague_cap,
                              self.out, self.scores if accumulate_scores else None, self.n_cap,
                              self.ws_attend, self.side.opts() if self.side is not None and opts is None else opts)
        return self.out

    def attend_multi(self, q, n_q, accumulate_scores=True, ws=None):
        """n_q query tokens per sequence (q [B, n_q, Hq, D]) at the n_q newest
        positions, over one rebuilt cache.  Returns out [B, n_q, Hq, D] float32."""
        if ws is None:
            n = kvr.kvr_attend_multi_workspace_size(self.desc, n_q, self.ret_cap, self.vague_cap)
            ws = torch.empty(max(n, 256), dtype=torch.uint8, device=self.device)
        B, Hq, D = self.desc.batch, self.desc.n_q_heads, self.desc.head_dim
        out = torch.zeros(B, n_q, Hq, D, dtype=torch.float32, device=self.device)
        kvr.kvr_attend_multi(self.desc, q, n_q, self.n_ctx, self.k_ret, self.v_ret, self.ret_pos, self.ret_cap,
                             self.sketch_k, self.sketch_v, self.vague_pos, self.n_vague, self.vague_cap, out,
                             self.scores if accumulate_scores else None, self.n_cap, ws)
        return out

    def step_update(self, k_new, v_new):
        """append + select + encode in one launch (decode steady state)."""
        kvr.kvr_step_update(self.desc, k_new, v_new, self.n_ctx, self.k_ret, self.v_ret, self.ret_pos,
                            self.ret_cap, self.scores, self.n_cap, self.r_size, self.k_candidate,
                            self.evict_slot, self.evict_pos, self.n_evict, self.evict_cap, self.vague_pos,
                            self.n_vague, self.vague_cap, self.sketch_k, self.sketch_v)

    def swap_back(self, replace_rate=1.1, max_swaps=4, n_swapped=None, swap_log=None):
        """The swap loop of Algorithm 3 on this layer's buffers."""
        kvr.kvr_swap_back(self.desc, self.scores, self.n_cap, self.k_ret, self.v_ret, self.ret_pos,
                          self.ret_cap, self.n_ctx, self.r_size, replace_rate, max_swaps, self.sketch_k,
                          self.sketch_v, self.vague_pos, self.n_vague, self.vague_cap, n_swapped, swap_log)

    def check_evictions(self):
        """Synchronises and raises if the last update of some unit could not evict what it had to
        (n_evict < 0: evict_cap or vague_cap too small; the unit then kept everything and its
        retained slots fill up)."""
        worst = int(self.n_evict.min().item())
        if worst < 0:
            raise RuntimeError(f"a unit needed {-worst} evictions but evict_cap = {self.evict_cap}, "
                               f"vague_cap = {self.vague_cap}: nothing was evicted there")

    def rotate(self, k_new, q, rotation):
        """Norm and rotation of one new token per sequence (k_new [B, Hkv, D], q [B, Hq, D] as projected; n_ctx counts
        the token) -> the key that append takes and the query that attend takes, in buffers that the next call reuses."""
        if self.k_turned is None:
            self.k_turned = torch.empty(k_new.shape, dtype=self.dtype, device=self.device)
            self.q_turned = torch.empty(q.shape, dtype=self.dtype, device=self.device)
        kvr.kvr_rotate(self.desc, rotation, q, k_new, None, self.desc.batch, None, self.n_ctx, self.q_turned, self.k_turned)
        return self.k_turned, self.q_turned

    def decode_step(self, k_new, v_new, q, *, bump_n_ctx=True, fused=None, replace_rate=None, max_swaps=4,
                    check=False, opts=None, rotation=None):
        """(rotate, if a binding.make_rotation is given) -> append -> select -> encode -> (swap loop, if replace_rate
        is given) -> attend.  n_ctx counts the new token from here on; pass bump_n_ctx=False when
        several layers share one n_ctx tensor that the caller advances once per
        step.  fused: use kvr_step_update for the first three (default: whenever its
        size limits allow).  check: synchronise after the update and raise if a unit
        could not evict (see check_evictions)."""
        if bump_n_ctx:
            self.n_ctx += 1
        if rotation is not None:
            k_new, q = self.rotate(k_new, q, rotation)
        # Algorithm 3, first branch: does the Recent queue hand its overhang on to the Candidates?
        self.r_size = kvr.kvr_recent_size(self.r_size + 1, self.n_recent, self.slack)
        if fused is None:
            fused = self.ret_cap <= 32768 and self.evict_cap <= 64
        if fused:
            self.step_update(k_new, v_new)
        else:
            self.append(k_new, v_new)
            self.select()
            self.encode()
        if check:
            self.check_evictions()
        if replace_rate is not None and max_swaps > 0:
            self.swap_back(replace_rate, max_swaps)
        return self.attend(q, opts=opts)

    # -- building the state from a prompt ---------------------------------------
    @classmethod
    def from_prefill(cls, desc, K, V, q0, *, n_recent, k_candidate, max_new_tokens, evict_cap=None,
                     init_scores=None, ws_attend=None, ws_encode=None, n_ctx=None, timers=None, slack=0,
                     side=None, q_prompt=None):
        """Compress a prompt's KV cache K, V [B, Hkv, N, D]: cumulative scores are
        initialised with one dense attention pass of q0 (or taken from
        init_scores [B, Hkv, N], or accumulated over the causal attention of all the prompt's
        queries q_prompt [B, N, Hq, D], whose outputs are then info["out"]; q0 may be None), the Recent and Candidate parts are kept raw and
        moved into ret_cap = n_recent + k_candidate + slack + 1 slots, everything else
        goes into the sketch.  Returns (state, info)."""
        B, Hkv, N, D = K.shape
        if init_scores is None and q_prompt is not None and tuple(q_prompt.shape) != (desc.batch, N, desc.n_q_heads, D):
            raise ValueError(f"q_prompt: shape {tuple(q_prompt.shape)}, need {(desc.batch, N, desc.n_q_heads, D)}")
        dev = K.device
        R = n_recent + k_candidate
        ret_cap = R + slack + 1
        n_cap = N + max_new_tokens
        n_vague0 = max(N - R, 0)
        vague_cap = n_vague0 + max_new_tokens
        if evict_cap is None:
            evict_cap = max(8, slack + 1)
        st = cls(desc, n_recent=n_recent, k_candidate=k_candidate, ret_cap=ret_cap, vague_cap=vague_cap,
                 n_cap=n_cap, evict_cap=evict_cap, device=dev, ws_attend=ws_attend, ws_encode=ws_encode,
                 n_ctx=n_ctx, slack=slack, side=side, empty_slots=False)
        st.n_ctx.fill_(N)
        # the whole prompt was pushed into the Recent queue
        st.r_size = kvr.kvr_recent_size(N, n_recent, slack)
        # 1. cumulative scores of the prompt
        if init_scores is not None:
            st.scores[:, :, :N] = init_scores
        elif q_prompt is not None:
            prompt_out = attend_dense_prompt(desc, q_prompt, K, V, st.n_ctx, st.scores)
        else:
            ws = kvr.alloc_workspace(desc, kvr.KVR_OP_ATTEND, N, 0, dev)
            kvr.kvr_attend_decode(desc, q0, K, V, None, N, None, None, None, None, 0, st.out, st.scores,
                                  n_cap, ws)
            del ws
        # 2. partition: every prompt token sits in "slot = position" of the full cache
        full_pos = torch.arange(N, dtype=torch.int32, device=dev).expand(B, Hkv, N).contiguous()
        ev_cap = max(n_vague0, 1)
        lists = ((B, Hkv, ev_cap), torch.int32), ((B, Hkv, ev_cap), torch.int32)
        if n_vague0 > 0 and st.r_size == n_recent:       # exactly n_vague0 tokens leave every unit: no entry stays unwritten
            ev_slot, ev_pos = (torch.empty(shape, dtype=dt, device=dev) for shape, dt in lists)
        else:
            ev_slot, ev_pos = _zeros(dev, *lists)
        ws = kvr.alloc_workspace(desc, kvr.KVR_OP_ENCODE, ev_cap, 0, dev)
        if timers is not None:       # (start, stop) torch events around select + bulk encode
            timers[0].record()
        kvr.kvr_select(desc, st.scores, n_cap, full_pos, N, st.n_ctx, st.r_size, k_candidate,
                       ev_slot, ev_pos, st.n_evict, ev_cap, st.vague_pos, st.n_vague, vague_cap)
        # 3. bulk insert of the evicted tokens
        kvr.kvr_encode(desc, K, V, N, ev_slot, ev_pos, st.n_evict, ev_cap, st.sketch_k, st.sketch_v,
                       None, None, ws)
        if timers is not None:
            timers[1].record()
        del ws
        # 4. the kept rows move into the small slot array (ascending slot order)
        kvr.kvr_compact(desc, K, V, full_pos, N, ev_slot, st.n_evict, ev_cap, st.k_ret, st.v_ret, st.ret_pos,
                        ret_cap, min(st.r_size + k_candidate, N))
        info = {"evict_slot": ev_slot, "evict_pos": ev_pos, "n_evict": st.n_evict.clone()}
        if init_scores is None and q_prompt is not None:
            info["out"] = prompt_out
        return st, info


def attend_dense_prompt(desc, q, K, V, n_ctx, scores=None):
    """Causal attention of all queries q [B, N, Hq, D] of prompts of one length over their dense cache K, V
    [B, Hkv, N, D]; scores [B, Hkv, n_cap] accumulate.  Returns out, shaped as q."""
    B, N = q.shape[0], q.shape[1]
    pages = kvr.make_pages(desc, K, V)
    q_start = torch.arange(0, B * N + 1, N, dtype=torch.int32, device=q.device)
    n = kvr.kvr_attend_prompt_workspace_size(desc, B * N, pages, 0, 0, scores is not None)
    ws = torch.empty(max(n, 256), dtype=torch.uint8, device=q.device)
    out = torch.empty_like(q)
    kvr.kvr_attend_prompt(desc, q, B * N, q_start, n_ctx, pages, 0, 0, out, scores,
                          scores.shape[2] if scores is not None else 0, ws)
    return out


class PagedCache:
    """The uncompressed, paged cache of one layer and the calls over it: what a prompt fills and decode steps extend
    until (or instead of) its compression into a LayerState."""

    def __init__(self, desc, *, n_pages, page_size, table_cap, rotation=None, window=0, n_sink=0, scores=True,
                 device="cuda", n_ctx=None, table=None):
        """table int32 [B, table_cap] (None: made here, with no page assigned; see assign) and n_ctx int32 [B] may be
        shared by layers; rotation: a binding.make_rotation (None: queries and keys are cached as they come);
        scores: accumulate the weights that each token draws.  Tokens past table_cap * page_size are stored nowhere and
        attention takes the sequence to end there: the caller, who advances n_ctx, keeps it within.  A place of the batch
        that passes to another sequence keeps its scores until the caller clears them."""
        B, Hkv, D = desc.batch, desc.n_kv_heads, desc.head_dim
        if table is not None and (table.dim() != 2 or table.shape[1] != table_cap):
            raise ValueError(f"table: shape {tuple(table.shape)}, need [{B}, {table_cap}]")
        self.desc, self.window, self.n_sink = desc, int(window), int(n_sink)
        self.device = torch.device(device)
        self.dtype = torch.float32 if desc.dtype == kvr.KVR_F32 else torch.bfloat16
        self.rotation = kvr.make_rotation(desc) if rotation is None else rotation
        self.k, self.v = (torch.zeros(n_pages, Hkv, page_size, D, dtype=self.dtype, device=self.device) for _ in range(2))
        self.table = torch.full((B, table_cap), -1, dtype=torch.int32, device=self.device) if table is None else table
        self.n_ctx = torch.zeros(B, dtype=torch.int32, device=self.device) if n_ctx is None else n_ctx
        self.pages = kvr.make_pages(desc, self.k, self.v, self.table)
        self.n_cap = table_cap * page_size
        self.scores = torch.zeros(B, Hkv, self.n_cap, dtype=torch.float32, device=self.device) if scores else None
        # one token per sequence: the buffers of every step
        n = kvr.kvr_attend_paged_workspace_size(desc, self.pages, self.window, self.n_sink, scores)
        self.ws = torch.empty(max(n, 256), dtype=torch.uint8, device=self.device)
        self.q = torch.empty(B, desc.n_q_heads, D, dtype=self.dtype, device=self.device)
        self.out = torch.empty_like(self.q)

    def assign(self, b, first, pages):
        """Pages (numbers) of sequence b from its `first`-th page on."""
        if first < 0 or first + len(pages) > self.table.shape[1]:
            raise ValueError(f"pages {first} .. {first + len(pages) - 1} of a sequence that has room for {self.table.shape[1]}")
        self.table[b, first:first + len(pages)] = torch.as_tensor(pages, dtype=torch.int32, device=self.device)

    def prompt(self, q, k, v, q_start):
        """New tokens by q_start int32 [B + 1] (q [n_rows, Hq, D], k, v [n_rows, Hkv, D] as projected; n_ctx counts
        them): into the pages, then attention over all of each sequence.  Returns out [n_rows, Hq, D]."""
        rows = q.shape[0]
        turned = torch.empty(rows, self.desc.n_q_heads, self.desc.head_dim, dtype=self.dtype, device=self.device)
        kvr.kvr_rotate(self.desc, self.rotation, q, k, v, rows, q_start, self.n_ctx, turned, None, self.pages)
        out = torch.zeros_like(turned)
        n = kvr.kvr_attend_prompt_workspace_size(self.desc, rows, self.pages, self.window, self.n_sink, self.scores is not None)
        ws = torch.empty(max(n, 256), dtype=torch.uint8, device=self.device)
        kvr.kvr_attend_prompt(self.desc, turned, rows, q_start, self.n_ctx, self.pages, self.window, self.n_sink, out,
                              self.scores, self.n_cap, ws)
        return out

    def decode_step(self, q, k, v, *, bump_n_ctx=True):
        """One token per sequence (q [B, Hq, D], k, v [B, Hkv, D] as projected) into the pages, then its attention;
        bump_n_ctx as in LayerState.decode_step.  Returns out [B, Hq, D], reused by the next step."""
        if bump_n_ctx:
            self.n_ctx += 1
        kvr.kvr_rotate(self.desc, self.rotation, q, k, v, self.desc.batch, None, self.n_ctx, self.q, None, self.pages)
        kvr.kvr_attend_paged(self.desc, self.q, self.n_ctx, self.pages, self.window, self.n_sink, self.out, self.scores,
                             self.n_cap, self.ws)
        return self.out

    def dense(self, n_tokens):
        """Keys and values of the first n_tokens of every sequence as dense caches [B, Hkv, n_tokens, D], for
        LayerState.from_prefill.  Raises ValueError where a sequence does not have them all, tokens whose page is not there
        among them; looks at the table and n_ctx for that, so it synchronises."""
        ps = self.k.shape[2]
        if n_tokens < 1 or -(-n_tokens // ps) > self.table.shape[1]:
            raise ValueError(f"n_tokens = {n_tokens}: a sequence has room for 1 .. {self.table.shape[1] * ps}")
        B = self.desc.batch
        at = self.table[:B, :-(-n_tokens // ps)].long()
        if not bool(((at >= 0) & (at < self.k.shape[0])).all() & (self.n_ctx[:B] >= n_tokens).all()):
            raise ValueError(f"not every sequence has its first {n_tokens} tokens in the cache")
        return tuple(x[at].transpose(1, 2).flatten(2, 3)[:, :, :n_tokens].contiguous() for x in (self.k, self.v))
