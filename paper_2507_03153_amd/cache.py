"""Plumbing for the KV manager calls: owns the device buffers of one layer's cache state (block pool,
block table, window / pool lengths, moving averages, per-head salient lists) and enqueues the calls of
one decode step in the order of the paper's Alg. 2 (attention) and Alg. 1 (management).  Nothing here
computes: every step is a libhgca call, but for the few lengths that a draft step keeps apart."""
from __future__ import annotations

from dataclasses import replace
from types import SimpleNamespace

import torch

from . import hgca


class LayerCache:
    """Cache state of one attention layer for a batch of B sequences.

    Sequence b owns the blocks block_table[b, :] (here simply b*max_blocks + j); its pool is the first
    first_win_block[b] of them, its window the following ones."""

    def __init__(self, dtype, B: int, Hq: int, Hkv: int, d: int, block_size: int, win_blocks: int, max_blocks: int,
                 k_max: int, sm_scale: float, device="cuda:0", keep_evicted_maw: bool = False,
                 fused_tail: bool = True, win_cap_blocks: int = 0, pool8: bool = False):
        i32 = dict(dtype=torch.int32, device=device)
        f32 = dict(dtype=torch.float32, device=device)
        self.B, self.Hq, self.Hkv, self.d = B, Hq, Hkv, d
        self.block_size, self.win_blocks, self.max_blocks, self.k_max = block_size, win_blocks, max_blocks, k_max
        self.fused_tail = fused_tail      # one fold of all split partials instead of sparse fold + merge
        # capacity of the window range: l_max for decode steps, l_max - 1 + N for prompts of N tokens
        self.win_cap_blocks = win_cap_blocks or win_blocks
        self.win_cap = self.win_cap_blocks * block_size
        self.pool_cap = max_blocks * block_size
        self.k_blocks = torch.zeros(B * max_blocks, Hkv, block_size, d, dtype=dtype, device=device)
        self.v_blocks = torch.zeros_like(self.k_blocks)
        self.block_table = torch.arange(B * max_blocks, **i32).reshape(B, max_blocks).contiguous()
        self.first_win_block = torch.zeros(B, **i32)
        self._lens = torch.zeros(2, B, **i32)
        self.win_lens, self.pool_lens = self._lens[0], self._lens[1]
        self.a_maw = torch.zeros(B, Hq, self.win_cap, **f32)
        self.ctx_idx = torch.full((B, Hq, max(k_max, 1)), -1, **i32)
        self.ctx_cnt = torch.zeros(B, Hq, **i32)
        self.a_evicted = torch.zeros(B, Hq, self.pool_cap, **f32) if keep_evicted_maw else None
        self.plan = torch.zeros(B, 4, **i32)
        self.status = torch.zeros(1, **i32)
        q_like = torch.empty(B, Hq, d, dtype=dtype, device=device)
        self.shape = hgca.make_shape(q_like, Hkv, sm_scale)
        p = lambda t: None if t is None else t.data_ptr()
        self.state = hgca.CacheState(p(self.k_blocks), p(self.v_blocks), p(self.block_table), p(self.first_win_block),
                                     p(self.win_lens), p(self.pool_lens), p(self.a_maw), p(self.ctx_idx),
                                     p(self.ctx_cnt), p(self.a_evicted), p(self.plan), p(self.status),
                                     block_size, max_blocks, win_blocks, k_max, self.pool_cap, self.win_cap_blocks)
        self.window = hgca.Tier(self.k_blocks, self.v_blocks, self.win_cap, self.win_lens, self.block_table,
                                block_size, self.first_win_block)
        self.pool = hgca.Tier(self.k_blocks, self.v_blocks, self.pool_cap, self.pool_lens, self.block_table,
                              block_size, None)
        # the pool's entries once more in 8 bits (E4M3 with scales), for draft_step: same blocks, table and lengths
        self.pool8 = hgca.Kv8Tier.like(self.pool) if pool8 else None
        self.pool8_lens = torch.zeros(B, **i32)          # tokens of the pool that are there already
        self.draft_first = torch.zeros(B, **i32)         # the window's lengths before the drafts of a draft_step
        self.draft_ok = torch.zeros(B, **i32)            # 1: the drafts are in the window, 0: it had no room for them
        self._draft_cnt = torch.zeros(B, **i32)          # what `commit` takes of them
        # the tiers of a draft_step: a sequence without its drafts has no tokens
        self._draft_lens = torch.zeros(2, B, **i32)
        self._draft_window = replace(self.window, seq_lens=self._draft_lens[0])
        self._draft_pool = replace(self.pool8 if pool8 else self.pool, seq_lens=self._draft_lens[1])
        self._drafts = {}
        # per-step outputs and scratch
        self.o_w, self.lse_w = torch.empty(B, Hq, d, **f32), torch.empty(B, Hq, **f32)
        self.o_s, self.lse_s = torch.empty(B, Hq, d, **f32), torch.empty(B, Hq, **f32)
        self.o, self.lse = torch.empty(B, Hq, d, **f32), torch.empty(B, Hq, **f32)
        self.a_gpu = torch.zeros(B, Hq, self.win_cap, **f32)
        self.ws_dense = hgca.alloc_workspace(self.shape, self.win_cap, 0, 0, device)
        self.ws_sparse = hgca.alloc_workspace(self.shape, 0, 0, k_max, device)

    def append(self, k_in, v_in, active=None) -> None:
        hgca.kv_append(self.shape, self.state, k_in, v_in, active)

    def attend(self, q, alpha=None, n_new: int = 1) -> None:
        """Alg. 2, decode branch, on a window that already holds the token being decoded.  With `alpha` the
        moving-average update of Alg. 1 rides along with the window's weights."""
        sh = self.shape
        if alpha is None:
            hgca.dense_window_attn_weights(sh, q, self.window, self.o_w, self.lse_w, self.a_gpu, self.ws_dense)
        else:
            hgca.dense_window_attn_maw(sh, q, self.window, self.o_w, self.lse_w, self.a_gpu, self.a_maw, n_new, alpha,
                                       self.ws_dense)
        if self.fused_tail:        # the window's split partials are still in ws_dense: fold them with the sparse ones
            hgca.sparse_attn(sh, q, self.pool, self.ctx_idx, self.ctx_cnt, self.k_max, None, None, self.ws_sparse)
            hgca.lse_merge_splits(sh, self.win_cap, self.ws_dense, self.k_max, self.ws_sparse, self.o, self.lse)
        else:
            hgca.sparse_attn(sh, q, self.pool, self.ctx_idx, self.ctx_cnt, self.k_max, self.o_s, self.lse_s,
                             self.ws_sparse)
            hgca.lse_merge(sh, self.o_s, self.lse_s, self.o_w, self.lse_w, self.o, self.lse)

    def manage(self, alpha: float, beta: float, n_new: int = 1, maw_done: bool = False) -> None:
        """Alg. 1: moving-average update (unless `attend` did it), then eviction and sparsification where a
        window is full."""
        if not maw_done:
            hgca.maw_update(self.shape, self.a_maw, self.a_gpu, self.win_lens, self.win_cap, n_new, alpha)
        hgca.kv_evict(self.shape, self.state, beta)

    def append_buffers(self, n_q: int):
        """Outputs and scratch of append turns of n_q tokens (allocated once per n_q)."""
        if getattr(self, "_append_n", None) != n_q:
            f32 = dict(dtype=torch.float32, device=self.k_blocks.device)
            self._append_n = n_q
            self.a_cpu = torch.zeros(self.B, self.Hq, max(self.pool_cap, 1), **f32)
            self.o_app = torch.empty(self.B, n_q, self.Hq, self.d, **f32)
            self.lse_app = torch.empty(self.B, n_q, self.Hq, **f32)
            self.ws_append = hgca.managed_append_workspace(self.shape, self.state, n_q, self.k_blocks.device)
            self.ws_attn = hgca.append_workspace(self.shape, n_q, max(self.win_cap, self.pool_cap), self.k_blocks.device)
            self.o_aw, self.lse_aw = torch.empty_like(self.o_app), torch.empty_like(self.lse_app)
            self.o_ap, self.lse_ap = torch.empty_like(self.o_app), torch.empty_like(self.lse_app)

    def append_step(self, q, k_in, v_in, alpha: float, beta: float, one_call: bool = True) -> None:
        """One append turn (Alg. 2 append branch, then Alg. 1 with the re-evaluation): q [B,N,Hq,d], k_in / v_in
        [B,N,Hkv,d].  Results in o_app [B,N,Hq,d], lse_app [B,N,Hq], a_gpu, a_cpu."""
        n_q = int(q.shape[1])
        self.append_buffers(n_q)
        sh = self.shape
        if one_call:
            hgca.managed_append_step(sh, self.state, q, k_in, v_in, alpha, beta, self.a_gpu, self.a_cpu, self.o_app,
                                     self.lse_app, self.ws_append)
            return
        hgca.kv_append_tokens(sh, self.state, k_in, v_in)
        hgca.append_attn(sh, q, self.window, True, self.o_aw, self.lse_aw, self.ws_attn)
        hgca.append_attn(sh, q, self.pool, False, self.o_ap, self.lse_ap, self.ws_attn)
        merged = hgca.Shape(sh.dtype, sh.batch * n_q, sh.n_q_heads, sh.n_kv_heads, sh.head_dim, sh.sm_scale)
        hgca.lse_merge(merged, self.o_ap, self.lse_ap, self.o_aw, self.lse_aw, self.o_app, self.lse_app)
        hgca.append_weights(sh, q, self.window, True, self.lse_aw, self.a_gpu)
        hgca.append_weights(sh, q, self.pool, False, self.lse_ap, self.a_cpu)
        hgca.maw_update(sh, self.a_maw, self.a_gpu, self.win_lens, self.win_cap, n_q, alpha)
        hgca.threshold_select(sh, self.a_cpu, self.pool_lens, self.pool_cap, self.pool_lens, beta, self.k_max,
                              self.ctx_idx, self.ctx_cnt)
        hgca.kv_evict(sh, self.state, beta)

    def decode_step(self, q, k_in, v_in, alpha: float, beta: float, fused_maw: bool = True,
                    one_call: bool = False) -> None:
        if one_call:
            hgca.managed_decode_step(self.shape, self.state, q, k_in, v_in, alpha, beta, self.a_gpu, self.o, self.lse,
                                     self.ws_dense, self.ws_sparse)
            return
        self.append(k_in, v_in)
        self.attend(q, alpha if fused_maw else None)
        self.manage(alpha, beta, maw_done=fused_maw)

    def _draft_buffers(self, n: int) -> SimpleNamespace:
        """Outputs and workspaces of draft steps of n tokens.  Kept for good: a captured graph may hold their addresses."""
        if n not in self._drafts:
            dev = self.k_blocks.device
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError(f"the first draft_step of {n} tokens allocates: make it before the capture")
            f32 = dict(dtype=torch.float32, device=dev)
            o = [torch.empty(self.B, n, self.Hq, self.d, **f32) for _ in range(3)]
            lse = [torch.empty(self.B, n, self.Hq, **f32) for _ in range(3)]
            make = hgca.kv8_workspace if self.pool8 is not None else hgca.append_workspace
            self._drafts[n] = SimpleNamespace(o=o, lse=lse, ws=hgca.tree_workspace(self.shape, n, self.win_cap, dev),
                                              ws_pool=make(self.shape, n, self.pool_cap, dev))
        return self._drafts[n]

    def _device(self) -> int:
        """The cache's GPU, which has to be the current one: some of the calls of a step take that one's stream."""
        dev = self.k_blocks.get_device()
        if torch.cuda.current_device() != dev:
            raise ValueError(f"the cache is on cuda:{dev}, the current device is cuda:{torch.cuda.current_device()}")
        return dev

    def draft_step(self, q, k_in, v_in, mask=None) -> None:
        """Attention of n drafted tokens per sequence, which join the window for the time being: q [B,n,Hq,d], k_in / v_in
        [B,n,Hkv,d]; bit j of mask[b,i] (int64 [B,n]) = draft i sees draft j (None: all).  They see the whole window, and the whole
        pool, in 8 bits if the cache keeps it so.  Results in o_draft [B,n,Hq,d], lse_draft [B,n,Hq]; one `commit` follows.

        A sequence whose table row has no room for n more tokens takes none (status bit CACHE_CONTEXT_FULL, draft_ok[b] = 0): its
        queries see nothing, O = 0 and lse = -inf, and `commit` leaves it as it is."""
        n, sh, dev = int(q.shape[1]), self.shape, self._device()
        # the append is not taken back: what the later calls would refuse is refused before it
        hgca._need("q", q, self.k_blocks.dtype, (self.B, n, self.Hq, self.d), dev)
        for name, t in (("k_in", k_in), ("v_in", v_in)):
            hgca._need(name, t, self.k_blocks.dtype, (self.B, n, self.Hkv, self.d), dev)
        if mask is not None:
            hgca._need("mask", mask, torch.int64, (self.B, n), dev)
        if self.win_cap < (self.win_blocks * self.block_size - 1) + n:
            raise ValueError(f"{n} drafted tokens need win_cap_blocks for l_max - 1 + {n} tokens")
        mine = self._draft_buffers(n)
        (self.o_draft, o_w, o_p), (self.lse_draft, lse_w, lse_p) = mine.o, mine.lse
        self.draft_first.copy_(self.win_lens)
        hgca.kv_append_tokens(sh, self.state, k_in, v_in)
        torch.gt(self.win_lens, self.draft_first, out=self.draft_ok)
        torch.mul(self._lens, self.draft_ok, out=self._draft_lens)
        hgca.tree_attn(sh, q, self._draft_window, mask, o_w, lse_w, mine.ws)
        if self.pool8 is not None:
            self.sync_pool8()
            hgca.kv8_attn(sh, q, self._draft_pool, o_p, lse_p, mine.ws_pool)
        else:
            hgca.append_attn(sh, q, self._draft_pool, False, o_p, lse_p, mine.ws_pool)
        merged = hgca.Shape(sh.dtype, sh.batch * n, sh.n_q_heads, sh.n_kv_heads, sh.head_dim, sh.sm_scale)
        hgca.lse_merge(merged, o_p, lse_p, o_w, lse_w, self.o_draft, self.lse_draft)

    def commit(self, k_in, v_in, path, cnt, beta: float) -> None:
        """Of the last draft_step's tokens (its k_in, v_in) those on the accepted path stay in the window: path int32 [B,n], cnt
        int32 [B] (None: all n).  Then windows that have reached l_max evict (Alg. 1).  The moving averages of the tokens that stay
        start at 0 (attention weights under a tree mask are not averaged): tokens that are evicted before a decode step has seen
        them pass no threshold, so that decode steps attend to them again only from an append_step on, which draws up the lists
        anew.  Draft steps, which attend to the whole pool, lose nothing by that."""
        n, dev = int(k_in.shape[1]), self._device()
        if cnt is not None:
            hgca._need("cnt", cnt, torch.int32, (self.B,), dev)
        torch.mul(self.draft_ok, n if cnt is None else cnt, out=self._draft_cnt)
        hgca.kv_commit(self.shape, self.window, self.draft_first, k_in, v_in, self.win_lens, path=path, cnt=self._draft_cnt,
                       status=self.status)
        hgca.kv_evict(self.shape, self.state, beta)

    def sync_pool8(self) -> None:
        """Stores in 8 bits what the pool has got since the last call; a draft_step begins with it."""
        if self.pool8 is None:
            return
        hgca.kv8_write_tier(self.shape, self.pool8, self.pool8_lens, self.pool, self.pool_cap)
        self.pool8_lens.copy_(self.pool_lens)
