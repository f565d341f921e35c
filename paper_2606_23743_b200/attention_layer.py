"""One self-attention layer of a video transformer with its projections, on one GPU, over the C ABI: the calls around the
attention, in the order in which a denoising loop makes them.

    x -> e4m3 codes -> QKV product -> rotary positions -> K, V into the quantised cache -> K, V of the whole clip read back
      -> routing and block-sparse attention -> e4m3 codes -> output product + residual

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
