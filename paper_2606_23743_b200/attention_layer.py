"""One self-attention layer of a video transformer with its projections, on one GPU, over the C ABI: the calls around the
attention, in the order in which a denoising loop makes them.

    x -> e4m3 codes -> QKV product -> rotary positions -> K, V into the quantised cache -> K, V of the whole clip read back
      -> routing and block-sparse attention -> e4m3 codes -> output product + residual

ChunkAttentionLayer is such a layer for clips that are generated in chunks, CrossAttentionLayer attends to a prompt's states.

A call gets the tokens that are computed in this step, all of them or a subset (token pruning): the others keep the K and V that an
earlier call wrote.  Weights are quantised once, when the layer is made.  Batch items share the weights and the grid.
"""
from __future__ import annotations

import torch

from . import binding as sva


class _Linear8:
    """y = act(x w^T + bias) + residual with w quantised here, x per call."""

    def __init__(self, w, bias=None):
        n, k = w.shape
        row = -(-k // 16) * 16
        self.n, self.k, self.row, self.bias, self.plan = n, k, row, bias, (None, None)
        self.w8 = torch.empty(n, row, dtype=torch.uint8, device=w.device)
        self.w_scale = torch.empty(-(-n // 128), -(-k // 128), dtype=torch.float32, device=w.device)
        sva.quantize_tiles_fp8(sva.make_linear(w8=self.w8, w_scale=self.w_scale, w=w), w, self.w8, self.w_scale)

    def __call__(self, x, out, status, residual=None):
        x8 = torch.empty(x.shape[0], self.row, dtype=torch.uint8, device=x.device)
        x_scale = torch.empty(-(-self.k // 128), x.shape[0], dtype=torch.float32, device=x.device)
        made_for, p = self.plan                              # (of sizes and strides alone: calls mostly repeat them)
        key = (x.shape, x.stride(), out.stride(), residual is not None and residual.stride())
        if made_for != key:
            p = sva.make_linear(x, x8, x_scale, self.w8, self.w_scale, out, residual=residual)
            self.plan = key, p
        sva.quantize_rows_fp8(p, x, x8, x_scale)
        sva.linear_fp8(p, x8, x_scale, self.w8, self.w_scale, out, self.bias, residual, status)
        return out


class AttentionLayer:
    """w_qkv [3 H d, C] (Q, K, V rows, head by head), w_out [C, H d], biases fp32 or None; `grid` (frames, rows, columns) of the
    clip's tokens, (t, h, w) order; `select` a binding.Select; `batch` items.  `cache` is the format of the K/V cache."""

    def __init__(self, w_qkv, w_out, heads: int, grid, select, batch: int = 1, block: int = 128, bias_qkv=None, bias_out=None,
                 cache: str = "e4m3", page: int = 64, rope_base: float = 10000.0, status=None):
        dev = w_qkv.device
        self.H, self.d, self.B, self.N = heads, w_qkv.shape[0] // (3 * heads), batch, grid[0] * grid[1] * grid[2]
        self.block, self.select = block, select
        self.qkv, self.out = _Linear8(w_qkv, bias_qkv), _Linear8(w_out, bias_out)
        self.status = status if status is not None else torch.zeros(1, dtype=torch.int32, device=dev)
        # rotary positions: a token's frame, row and column, each with its own pairs of channels
        n = torch.arange(self.N, device=dev)
        where = torch.stack((n // (grid[1] * grid[2]), n // grid[2] % grid[1], n % grid[2]))
        self.positions = where.to(torch.int32)[:, None].contiguous()                                   # [3, 1, N]
        side = self.d // 6
        self.pairs = [self.d // 2 - 2 * side, side, side]
        self.steps, _ = sva.rope_steps(self.d, self.pairs, rope_base, device=dev)
        # the cache: a run of pages per batch item
        per = -(-self.N // page)
        pages = batch * per
        row = self.d if cache == "e4m3" else self.d // 2
        arrays = []
        for _ in range(2):
            a = [torch.zeros(pages, heads, page, row, dtype=torch.uint8, device=dev), torch.ones(pages, heads, page, device=dev)]
            if cache == "fp4":
                a.append(torch.zeros(pages, heads, page, self.d // 16, dtype=torch.uint8, device=dev))
            arrays.append(a)
        self.cache = sva.make_kv_cache(*arrays, format=cache)
        self.table = torch.arange(pages, dtype=torch.int32, device=dev).view(batch, per)
        self.slots = (torch.arange(batch, device=dev)[:, None] * (per * page) + n).to(torch.int32).contiguous()      # [B, N]
        # the same by token index, between two places for indices that name no token: those have no slot
        self.positions_of = torch.nn.functional.pad(self.positions[:, 0], (1, 1))
        self.slots_of = torch.nn.functional.pad(self.slots, (1, 1), value=-1)
        self.lengths = torch.full((batch,), self.N, dtype=torch.int32, device=dev)
        self.plan = (None, None)                              # of the rotation
        # Q of the whole clip; tokens that a call leaves out keep theirs, so that routing sees whole blocks
        self.q, self.k, self.v, self.o = (torch.zeros(batch, self.N, heads, self.d, dtype=torch.bfloat16, device=dev).transpose(1, 2)
                                          for _ in range(4))

    def __call__(self, x, token_idx=None):
        """x [B, M, C] bf16, the tokens token_idx [B, M] (integers, ascending; None: all N): x + attention's projection, for them.  An index
        that names no token is reported in `status`; its token stays out of the cache, and its row of the result means nothing."""
        B, M, C = x.shape
        H, d = self.H, self.d
        assert B == self.B and (token_idx is None and M == self.N or token_idx is not None and tuple(token_idx.shape) == (B, M)), \
            "x holds the call's tokens of every batch item"
        if M == 0:
            return torch.empty_like(x)
        x = x.reshape(B * M, C)
        qkv = self.qkv(x, torch.empty(B * M, 3 * H * d, dtype=torch.bfloat16, device=x.device), self.status).view(B, M, 3, H, d)
        q, k, v = (qkv[:, :, i].transpose(1, 2) for i in range(3))
        if token_idx is None:
            positions, slots = self.positions, self.slots
        else:
            token_idx = token_idx.clamp(-1, self.N).int().contiguous()
            at = token_idx.long() + 1
            positions, slots = self.positions_of[:, at].contiguous(), torch.gather(self.slots_of, 1, at).contiguous()
        made_for, p = self.plan
        if made_for != (M, positions.shape):
            p = sva.make_rope(q, k, q, k, positions, d, "interleaved", self.pairs)
            self.plan = (M, positions.shape), p
        sva.rope(p, q, k, self.steps, positions, q, k)
        sva.kv_cache_write(self.cache, k, v, slots, self.status)
        sva.kv_cache_read(self.cache, self.table, self.lengths, self.k, self.v, self.status)
        if token_idx is None:
            self.q.copy_(q)
        else:
            sva.scatter_tokens(q, token_idx, self.q, self.status)
        self._attend()
        o = self.o
        if token_idx is not None:
            o = torch.empty(B, M, H, d, dtype=torch.bfloat16, device=x.device).transpose(1, 2)
            sva.gather_tokens(self.o, token_idx, o, self.status)
        o = o.transpose(1, 2).reshape(B * M, H * d)
        return self.out(o, torch.empty(B * M, C, dtype=torch.bfloat16, device=x.device), self.status, residual=x).view(B, M, C)

    def _attend(self):
        p = sva.make_problem(self.q, self.k, self.v, self.o, self.N, self.block)
        dev, rows = self.q.device, self.B * self.H * (-(-self.N // self.block))
        ws = torch.empty(max(256, sva.select_workspace_bytes(p, self.select)), dtype=torch.uint8, device=dev)
        row_ptr = torch.empty(rows + 1, dtype=torch.int32, device=dev)
        col_idx = torch.empty(sva.select_max_nnz(p, self.select), dtype=torch.int32, device=dev)
        sva.block_select(p, self.select, self.q, self.k, row_ptr, col_idx, ws)
        aws = torch.empty(max(256, sva.attn_one_call_workspace_bytes(p)), dtype=torch.uint8, device=dev)
        sva.block_sparse_attn_fwd(p, self.q, self.k, self.v, row_ptr, col_idx, self.o, None, self.status, workspace=aws)


class ChunkAttentionLayer:
    """The same for a clip that is generated in chunks, or a sequence that grows token by token: the tokens of a call attend to one another (causal: to
    those before them) and to all tokens that their sequence has had, whose K and V lie in a cache with a scale per page and head and are read
    where they lie.

        x -> e4m3 codes -> QKV product -> rotary positions -> pages taken -> K, V appended -> attention over the cache -> output product + residual

    w_qkv [(heads + 2 kv_heads) d, C] (Q rows, K rows, V rows, head by head), w_out [C, heads d]; room for `rows` sequences of up to `tokens`
    tokens in a pool of `pages` pages that they share.  The layer's state (refs, table, lengths) is on the device: no call waits for it."""

    def __init__(self, w_qkv, w_out, heads: int, tokens: int, rows: int = 1, kv_heads: int = 0, bias_qkv=None, bias_out=None, page: int = 64,
                 pages: int = 0, causal: bool = False, rope_base: float = 10000.0, status=None):
        dev = w_qkv.device
        self.Hq, self.H, self.B, self.causal = heads, kv_heads or heads, rows, causal
        self.d = w_qkv.shape[0] // (heads + 2 * self.H)
        self.qkv, self.out = _Linear8(w_qkv, bias_qkv), _Linear8(w_out, bias_out)
        self.status = status if status is not None else torch.zeros(1, dtype=torch.int32, device=dev)
        self.steps, _ = sva.rope_steps(self.d, [self.d // 2], rope_base, device=dev)
        per = -(-tokens // page)
        pages = pages or rows * per
        self.cache = sva.make_kv_cache(*([torch.zeros(pages, self.H, page, self.d, dtype=torch.uint8, device=dev), torch.zeros(pages, self.H, device=dev)]
                                         for _ in range(2)), format="e4m3_page")
        self.refs = torch.zeros(pages, dtype=torch.int32, device=dev)
        self.table = torch.full((rows, per), -1, dtype=torch.int32, device=dev)
        self.lengths = torch.zeros(rows, dtype=torch.int32, device=dev)
        # tokens that each sequence can come to have pages for; None: the pool may run out before
        self.most = torch.full((rows,), per * page, dtype=torch.int32, device=dev) if pages >= rows * per else None
        self.work = torch.empty(sva.kv_pages_compact_workspace_bytes(self.cache), dtype=torch.uint8, device=dev)

    def __call__(self, x, counts=None):
        """x [rows, M, C] bf16, of each sequence's next counts [rows] tokens (int32, outside [0, M] the nearer end; None: M): x + attention's projection, for
        them.  Rows of x behind its count mean nothing, nor do those of the result.  Where the pool or a sequence's table has no more pages the status says
        so, and a sequence goes on by the tokens that it has pages for: `lengths` is what it holds, and the others are as rows behind its count."""
        B, M, C = x.shape
        Hq, H, d = self.Hq, self.H, self.d
        assert B == self.B, "x holds tokens of every sequence"
        if M == 0:
            return torch.empty_like(x)
        x = x.reshape(B * M, C)
        counts = torch.full((B,), M, dtype=torch.int32, device=x.device) if counts is None else counts.clamp(0, M)
        qkv = self.qkv(x, torch.empty(B * M, (Hq + 2 * H) * d, dtype=torch.bfloat16, device=x.device), self.status).view(B, M, Hq + 2 * H, d).transpose(1, 2)
        q, k, v = qkv.split((Hq, H, H), 1)
        positions = (self.lengths[:, None] + torch.arange(M, dtype=torch.int32, device=x.device))[None].contiguous()
        sva.rope(sva.make_rope(q, k, q, k, positions, d), q, k, self.steps, positions, q, k)
        sva.kv_pages_take(self.cache, self.refs, self.table, self.lengths, counts, self.status)
        held = (self.table >= 0).sum(1, dtype=torch.int32) * self.cache.page if self.most is None else self.most
        counts = torch.minimum(counts, held - self.lengths)
        sva.kv_cache_append(self.cache, k, v, self.table, self.lengths, counts, self.status)
        self.lengths += counts
        o = torch.zeros(B, M, Hq, d, dtype=torch.bfloat16, device=x.device).transpose(1, 2)
        p = sva.make_cached_attn(self.cache, q, o, self.table, self.causal)
        space = torch.empty(max(256, sva.cached_attn_workspace_bytes(p)), dtype=torch.uint8, device=x.device)
        sva.cached_attn_fwd(p, q, self.table, self.lengths, o, counts, None, self.status, space)
        o = o.transpose(1, 2).reshape(B * M, Hq * d)
        return self.out(o, torch.empty(B * M, C, dtype=torch.bfloat16, device=x.device), self.status, residual=x).view(B, M, C)

    def fork(self, parents, children):
        """Sequences children (int32) give up what they hold and go on from where sequences parents are, whose full pages they share.  A child comes once
        and is no parent of the call: a parent that is named among the children has given up its pages by then."""
        sva.kv_pages_free(self.cache, self.refs, self.table, self.lengths, children, status=self.status)
        sva.kv_pages_fork(self.cache, self.refs, self.table, self.lengths, parents, children, self.status)

    def forget(self, which, keep=None):
        """Sequences `which` (int32) forget their tokens from keep (int32; None: 0) on.  A sequence that is cut within a page which others share gets a copy
        of it, so that what comes next is its own; where the pool has no page for that the status says so, and its full pages are what is left."""
        sva.kv_pages_free(self.cache, self.refs, self.table, self.lengths, which, keep, self.status)
        if keep is not None:
            self._own_last_pages()

    def _own_last_pages(self):
        """Gives every sequence whose last page is partly filled and shared a copy of it, on a free page of the lowest id, in the order of the rows.  Where nobody
        but such sequences shares a page the last of them keeps it.  (Nothing here waits for the device.)"""
        page, pages = self.cache.page, self.cache.pages
        at = (self.lengths // page).clamp_(max=self.table.shape[1] - 1).long()[:, None]
        src = self.table.gather(1, at)[:, 0]
        held = src.clamp(min=0).long()
        shares = (self.lengths % page != 0) & (src >= 0) & (self.refs[held] > 1)
        same = (src[:, None] == src) & shares
        needs = shares & ((same.sum(1) < self.refs[held]) | same.triu(1).any(1))
        dst = torch.searchsorted((self.refs <= 0).cumsum(0), needs.cumsum(0))       # (pages: there is none)
        gets = needs & (dst < pages)
        none = src.new_full((), -1)
        sva.kv_pages_copy(self.cache, torch.where(gets, src, none), torch.where(gets, dst.int(), none), self.status)
        self.refs.index_add_(0, held, -needs.int()).index_add_(0, dst.clamp(max=pages - 1), gets.int())
        self.table.scatter_(1, at, torch.where(needs, torch.where(gets, dst.int(), none), src)[:, None])
        short = needs & ~gets
        self.lengths -= torch.where(short, self.lengths % page, 0)
        self.status |= short.any().int() * sva.SVA_DEV_NO_PAGES

    def compact(self):
        """Moves the pages in use to the front of the pool."""
        sva.kv_pages_compact(self.cache, self.refs, self.table, self.work, status=self.status)


class CrossAttentionLayer:
    """Attention of a clip's tokens to an encoder's states (a prompt's), with its projections.  w_q [heads d, C], w_kv [2 kv_heads d, E] (K rows, V rows),
    w_out [C, heads d].  K and V of a prompt are the same in every denoising step: states() makes them once."""

    def __init__(self, w_q, w_kv, w_out, heads: int, kv_heads: int = 0, bias_q=None, bias_kv=None, bias_out=None, status=None):
        self.Hq, self.H, self.d = heads, kv_heads or heads, w_q.shape[0] // heads
        self.q, self.kv, self.out = _Linear8(w_q, bias_q), _Linear8(w_kv, bias_kv), _Linear8(w_out, bias_out)
        self.status = status if status is not None else torch.zeros(1, dtype=torch.int32, device=w_q.device)

    def states(self, encoded):
        """encoded [B, S, E] bf16 -> K, V [B, kv_heads, S, d]."""
        B, S, E = encoded.shape
        kv = torch.empty(B * S, 2 * self.H * self.d, dtype=torch.bfloat16, device=encoded.device)
        if S:
            self.kv(encoded.reshape(B * S, E), kv, self.status)
        kv = kv.view(B, S, 2, self.H, self.d)
        return kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2)

    def __call__(self, x, states, lengths=None, key_mask=None):
        """x [B, M, C] bf16: x + the projection of its attention to the states, of which the first lengths [B] (int32) and those that key_mask [B, S] does not
        leave out are there."""
        B, M, C = x.shape
        if M == 0:
            return torch.empty_like(x)
        k, v = states
        x = x.reshape(B * M, C)
        q = self.q(x, torch.empty(B * M, self.Hq * self.d, dtype=torch.bfloat16, device=x.device), self.status).view(B, M, self.Hq, self.d).transpose(1, 2)
        o = torch.empty(B, M, self.Hq, self.d, dtype=torch.bfloat16, device=x.device).transpose(1, 2)
        p = sva.make_cross_attn(q, k, v, o)
        space = torch.empty(max(256, sva.cross_attn_workspace_bytes(p)), dtype=torch.uint8, device=x.device)
        sva.cross_attn_fwd(p, q, k, v, o, lengths, key_mask, None, self.status, space)
        o = o.transpose(1, 2).reshape(B * M, self.Hq * self.d)
        return self.out(o, torch.empty(B * M, C, dtype=torch.bfloat16, device=x.device), self.status, residual=x).view(B, M, C)
