"""Decode with the key-value cache in device memory: a stack of attention + MoE layers of one shape, stepped over the fresh tokens of a
batch of requests -- whole prompts, single tokens, or both in one step -- with the seats and pages of requests that are done used again.

    tables of the step (moe_kv_assign, once)
    for each layer:  residual + norm + QKV projection (moe_pre_attention), norm and rotation into the layer's cache
                     (moe_qk_norm_rope), attention over the cache (moe_attn_decode), O projection + residual + norm + MoE layer
                     (moe_post_attention)

With a shape of 8-bit integers the projections and the experts are products of those (moe_pre_attention_i8, moe_post_attention_i8), and every layer
brings the scales of its weights' output channels.

In the paper's decode stage the attention of the middle line runs on the CPU (its section 4.1); here all of a layer is on the GPU.  The
order of the calls and the buffers between them, nothing else: all arithmetic is the library's.
"""
from __future__ import annotations

import dataclasses
from typing import List, Optional, Sequence, Tuple

import torch

from . import binding as B


@dataclasses.dataclass
class LayerScales:
    """Scales of one layer's 8-bit weights, device float32: of the rows of Wqkv and Wo, and of the experts'."""
    qkv: torch.Tensor                    # [rows of Wqkv, padded to a multiple of 128]
    o: torch.Tensor                      # [H]
    experts: B.ExpertScales


@dataclasses.dataclass
class LayerWeights:
    """One layer's weights in device memory: Wqkv, Wo and the experts in pages of one pool."""
    page_pool: torch.Tensor              # uint8 [pool_pages, page_bytes]
    qkv_table: torch.Tensor              # int32 [pages of Wqkv]
    o_table: torch.Tensor                # int32 [pages of Wo]
    page_table: torch.Tensor             # int32 [E, pages per expert]
    Wr: torch.Tensor                     # bf16 [E, H]
    norm_attn: torch.Tensor              # float32 [H], before the QKV projection
    norm_moe: torch.Tensor               # float32 [H], before the MoE layer
    bias: Optional[torch.Tensor] = None
    q_gamma: Optional[torch.Tensor] = None
    k_gamma: Optional[torch.Tensor] = None
    scales: Optional[LayerScales] = None         # with 8-bit weights


class DecodeLayers:
    """``shape``: the MoE layer (its T is ignored), ``kv``: heads and cache; ``n_requests`` seats, each with a row of the block
    table.  The requests' lengths, the pages they hold and the caches of all layers are kept here from step to step."""

    def __init__(self, shape: B.MoEShape, kv: B.KvShape, layers: Sequence[LayerWeights], inv_freq: torch.Tensor, n_requests: int,
                 eps: float = 1e-5, window: int = 0, device="cuda"):
        if kv.dtype != B.DTYPE_BF16 or shape.dtype not in (B.DTYPE_BF16, B.DTYPE_I8):
            raise ValueError("DecodeLayers: cache and MoE layer have to be bf16, the type of the projections beside them (or layer and projections 8-bit integers)")
        for i, w in enumerate(layers):
            if (w.scales is not None) != (shape.dtype == B.DTYPE_I8):
                raise ValueError(f"DecodeLayers: layer {i}: scales go with 8-bit weights, and with no others")
        if not 0 <= n_requests <= B.MAX_REQUESTS:
            raise ValueError(f"n_requests: at most {B.MAX_REQUESTS}, got {n_requests}")
        self.shape, self.kv, self.layers, self.n_requests = shape, kv, list(layers), int(n_requests)
        self.inv_freq, self.eps, self.window = inv_freq, float(eps), int(window)
        width = (kv.n_q + 2 * kv.n_kv) * kv.head_dim
        self.qkv_width, self.attn_width = -(-width // 128) * 128, kv.n_q * kv.head_dim
        norm = B._lib().moe_add_rmsnorm(0, shape.H, None, None, None, self.eps, None, None, None)          # no rows: the sizes alone
        for status in (B.kv_validate(kv), B.validate_shape(shape), norm):
            B._check(status, "DecodeLayers")
        for K, N in ((shape.H, self.qkv_width), (self.attn_width, shape.H)):
            B.linear_pages_required(B.make_linear_shape(1, K, N, shape.page_bytes, shape.dtype))         # raises where the projections do not take such sizes
        self.caches: List[Tuple[torch.Tensor, torch.Tensor]] = [
            (torch.empty(kv.cache_shape, dtype=kv.torch_dtype, device=device), torch.empty(kv.cache_shape, dtype=kv.torch_dtype, device=device)) for _ in self.layers]
        self.block_table = torch.full((self.n_requests, kv.max_pages), -1, dtype=torch.int32, device=device)
        self.free_pages = torch.arange(kv.pool_pages, dtype=torch.int32, device=device)
        self.lengths = torch.zeros(self.n_requests, dtype=torch.int32, device=device)
        self.free_head = torch.zeros(1, dtype=torch.int32, device=device)
        self.status = torch.zeros(4, dtype=torch.int32, device=device)
        self._rows, self._pair, self._turn = -1, (), 0    # two KvSteps for the number of rows of the step before, taken in turn
        self._workspace: Optional[B.AttnWorkspace] = None

    def step(self, embedded: torch.Tensor, fresh: torch.Tensor) -> Tuple[torch.Tensor, B.KvStep]:
        """embedded float32 [T, H]: the fresh tokens of all requests, in the order of the requests; fresh int32 [n_requests].
        -> (hidden states float32 [T, H] after the last layer, the step's tables).  Nothing waits for the device: a request that does
        not fit (bits 1 and 2 of status[0]) keeps its length, and its rows of the result mean nothing.  Entries of page tables outside their
        pool set bit 0, of the weights' tables with 8-bit weights only.  The tables are written again two steps later.  A call that raises leaves the requests as they were, and the step can be taken again."""
        kv, T = self.kv, embedded.shape[0]
        if T != self._rows:
            self._rows, self._pair = T, [B.KvStep(kv, self.n_requests, T, embedded.device) for _ in range(2)]
        if self._workspace is None or self._workspace.buf.numel() < B.attn_workspace_bytes(kv, T):
            self._workspace = B.AttnWorkspace(kv, T, embedded.device)
        tables = self._pair[self._turn]              # not the one that holds self.lengths: _turn goes on with them
        B.moe_kv_assign(kv, self.lengths, fresh, self.free_pages, self.free_head, self.block_table, step=tables, status=self.status)
        seen = torch.where(tables.slots >= 0, tables.positions + 1, 0)          # rows without a slot attend to nothing
        s = self.shape.with_tokens(T)
        qkv_proj = B.make_linear_shape(T, s.H, self.qkv_width, s.page_bytes, s.dtype)
        o_proj = B.make_linear_shape(T, self.attn_width, s.H, s.page_bytes, s.dtype)
        space = None
        if s.dtype == B.DTYPE_I8:
            # One buffer for the layers' workspaces, each of which begins 256 bytes behind the one before: a layer writes over what is behind the beginnings of
            # those before it, whose status words so stay until the end of the step, where they are looked at all at once.  Before them four words for the QKV
            # projections, which beside the errors leave a reading of the clock in their status.
            need = B.post_attention_i8_workspace_bytes(s, o_proj)
            space = B._scratch(need + 256 * (len(self.layers) + 1), embedded.device)
            words = space.view(torch.int32)
            projections = words[:4].zero_()
        hidden, delta = None, embedded
        for i, (w, (k_cache, v_cache)) in enumerate(zip(self.layers, self.caches), 1):
            if w.scales is None:
                hidden, _, qkv, _ = B.moe_pre_attention(qkv_proj, hidden, delta, w.norm_attn, self.eps, w.qkv_table, w.page_pool, want_bf16=False)
            else:
                hidden, _, _, qkv = B.moe_pre_attention_i8(qkv_proj, hidden, delta, w.norm_attn, self.eps, w.qkv_table, w.page_pool, w.scales.qkv, status=projections)
            q = B.moe_qk_norm_rope(kv, qkv, self.inv_freq, tables.positions, tables.slots, k_cache, v_cache, w.q_gamma, w.k_gamma, self.eps, status=self.status)
            attn, _ = B.moe_attn_decode(kv, q, seen, self.block_table, k_cache, v_cache, window=self.window, table_row=tables.request,
                                        workspace=self._workspace, status=self.status)
            attn = attn.view(T, self.attn_width)
            if w.scales is None:
                hidden, _, delta, _ = B.moe_post_attention(s, o_proj, attn, hidden, w.o_table, w.norm_moe, self.eps, w.Wr, w.page_table, w.page_pool, bias=w.bias)
            else:
                hidden, _, delta, _ = B.moe_post_attention_i8(s, o_proj, attn, hidden, w.o_table, w.scales.o, w.norm_moe, self.eps, w.Wr, w.page_table, w.page_pool,
                                                              w.scales.experts, bias=w.bias, workspace=space[256 * i:256 * i + need])
        out = hidden + delta
        if space is not None and T:                  # without rows no layer has written there
            self.status[:1].bitwise_or_(words[:64 * (len(self.layers) + 1):64].amax())          # bit 0 is the only one that a layer sets
        self.lengths, self.free_head, self._turn = tables.seq_len, tables.free_head, self._turn ^ 1
        return out, tables

    def retire(self, seats: torch.Tensor) -> None:
        """seats bool [n_requests]: these requests are done.  Their pages are free again, and their seats are of length 0 for others to take with the
        next step's fresh tokens.  Nothing waits for the device, as in a step."""
        if seats.dtype is not torch.bool or seats.shape != (self.n_requests,):
            raise ValueError(f"seats: expected torch.bool [{self.n_requests}], got {seats.dtype} {list(seats.shape)}")
        # The pages that are taken are those before free_head: the freed ones go to the last places of these, one after another.
        held = torch.where(seats, (self.lengths.long() + self.kv.page_tokens - 1) // self.kv.page_tokens, 0)
        freed = (torch.arange(self.kv.max_pages, device=seats.device) < held[:, None]).flatten()
        count = held.sum()
        to = torch.where(freed, self.free_head.long() - count + freed.cumsum(0) - 1, self.kv.pool_pages)         # what stays goes behind the list, and is cut off
        free_pages = torch.cat([self.free_pages, self.free_pages[:1]]).scatter_(0, to, self.block_table.flatten())[:-1]
        free_head, lengths = (self.free_head - count).to(torch.int32), self.lengths.masked_fill(seats, 0)
        self.block_table.masked_fill_(seats[:, None], -1)
        self.free_pages, self.free_head, self.lengths = free_pages, free_head, lengths
