"""The two halves of a served model's layer on one rank.

MoELayer: the norm before the block, the router, this rank's experts, and the norm after it with the block's gate, the residual
sum and the next block's norm.  Attention: what lies between the projections, norm and rotation of the heads, the append to a paged
cache held in 4 bits, and attention over it.

MoELayer's batches of up to `few_tokens` (FEW_TOKENS, fewer above 16 choices per token) run in four kernels (norm, router, few-token
experts, norm); larger ones take the four-step block between the norms (dispatch, permute, grouped FFN, combine).  Both read
the same packed weights.  Marshalling and buffers only; every step runs in the library's kernels."""
from __future__ import annotations

import torch

from . import binding as B

# The few-token kernel takes at most 64 tokens and is the faster form of all of them: 16 experts of d = 4096, f = 1536 on a
# rank, top-8 of 128: 56 us against 76 of the four-step block at 64 tokens, 27 against 46 at 8, 14 against 29 at 1 (either way
# every chosen expert's weights are read once; the block pads each instance to 128 rows and runs four kernels).
FEW_TOKENS = 64
FEW_PAIRS = 1024            # and at most so many (token, expert) pairs: fewer tokens above 16 choices each


class MoELayer:
    """Weights of one layer and the buffers of its calls.

    max_tokens   largest batch (rows of the buffers)
    w_router     bf16 [E, d]; bias f32 [E] or None; score B.ROUTE_SOFTMAX or B.ROUTE_SIGMOID
    replica_map  i32 [E, R]; quota i32 [E, R] or None (uniform over an expert's replicas; the few-token path uses the first)
    packed       the blob of tempo_pack_weights, or of tempo_pack_weights_bf16 with bf16=True
    norm_w, post_w, next_w   weights [d] of the norm before the block, after it (None: not normed) and of the next block;
                 norm_b, post_b, next_b their biases or None; kind B.NORM_RMS or B.NORM_LAYER
    count        every batch's pairs per expert are written to `counts` (i32 [E]) and added to `cum_counts` (u32 counters in
                 an i32 tensor, mod 2^32), which the dispatch solver works from.  The block counts as it dispatches; a
                 few-token batch takes one more kernel for it, the block's first step (6 us).  Without it both are None.

    A layer has one set of buffers and one workspace: its calls must follow one another on one stream (or be ordered by events).
    `status` collects the STATUS_* bits of every call.  After STATUS_TIMEOUT zero `workspace` and, where there is one,
    `block.workspace`.
    """

    def __init__(self, max_tokens, k, G_max, f, w_router, replica_map, packed, norm_w, post_w=None, next_w=None, bias=None,
                 quota=None, gate=None, kind=B.NORM_RMS, eps=1e-6, score=B.ROUTE_SOFTMAX, renormalise=True, scale=1.0,
                 r_scale=1.0, y_scale=1.0, count=False, norm_b=None, post_b=None, next_b=None, bf16=False):
        E, d = w_router.shape
        dev = w_router.device
        self.k, self.E, self.G_max, self.R, self.d, self.f = k, E, G_max, replica_map.shape[1], d, f
        self.w_router, self.bias, self.replica_map, self.packed = w_router, bias, replica_map, packed
        self.quota = torch.zeros_like(replica_map) if quota is None else quota
        self.norm_w, self.post_w, self.next_w, self.gate = norm_w, post_w, next_w, gate
        self.norm_b, self.post_b, self.next_b = norm_b, post_b, next_b
        self.kind, self.eps, self.r_scale, self.y_scale = kind, eps, r_scale, y_scale
        self.score, self.renormalise, self.scale = score, renormalise, scale
        self.bf16 = bf16
        self.x = torch.empty(max_tokens, d, dtype=torch.bfloat16, device=dev)
        self.y = torch.empty_like(self.x)
        self.topk_ids = torch.empty(max_tokens, k, dtype=torch.int32, device=dev)
        self.topk_w = torch.empty(max_tokens, k, dtype=torch.float32, device=dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.few_tokens = min(FEW_TOKENS, FEW_PAIRS // max(k, 1))
        few = B.make_shape(min(max_tokens, self.few_tokens), k, E, G_max, self.R, d, f, 128)
        self.workspace = torch.zeros(B.tempo_few_workspace_bytes(few), dtype=torch.uint8, device=dev)
        self.block = B.RankBuffers(max_tokens, k, E, G_max, self.R, d, f, device=dev) if max_tokens > self.few_tokens else None
        if self.block is not None:                       # the block reads this layer's tables and tensors
            self.block.replica_map, self.block.quota = self.replica_map, self.quota
            if bf16:
                self.block.packed_bf16 = packed
                self.block.alloc_bf16()
            else:
                self.block.packed = packed
            self.block.x, self.block.topk_ids, self.block.topk_w = self.x, self.topk_ids, self.topk_w
            self.block.out, self.block.status = self.y, self.status
        self.counts = self.cum_counts = None
        if count:
            i32 = dict(dtype=torch.int32, device=dev)
            self.counts, self.cum_counts = torch.zeros(E, **i32), torch.zeros(E, **i32)
            if self.block is not None:
                self.block.counts, self.block.cum_counts = self.counts, self.cum_counts
            cap = B.tempo_m_cap_bound(few)               # the dispatch of a few-token batch, of which only the counts are used
            self.few_dispatch = [torch.empty(n, **i32) for n in (G_max, G_max + 1, few.T * k, cap, cap // 128, 1)]

    def forward(self, r, r_out, x_next=None, gate=None, n_valid=None):
        """r_out = the residual stream after the block; x_next = its norm for the next block (with next_w).  r, r_out [T, d]
        bf16 or f32 (r_out may be r), x_next bf16.  gate: of this batch, e.g. [T, 1] (None: the layer's).  n_valid i32 [1]: rows
        behind it are padding and stay as they are in r_out and x_next (None: every row is live).  Enqueues kernels only: the
        call can be captured in a CUDA graph."""
        T = r.shape[0]
        if T > self.x.shape[0]:
            raise B.TempoError(f"a batch of {T} tokens exceeds the layer's {self.x.shape[0]}")
        x, y, ids, w = self.x[:T], self.y[:T], self.topk_ids[:T], self.topk_w[:T]
        shape = B.make_shape(T, self.k, self.E, self.G_max, self.R, self.d, self.f, 128)
        B.tempo_norm_in(r, self.norm_w, x, b=self.norm_b, kind=self.kind, eps=self.eps, n_valid=n_valid)
        B.tempo_route(shape, x, self.w_router, self.bias, n_valid, ids, w, self.status, score=self.score,
                      renormalise=self.renormalise, scale=self.scale)
        if T <= self.few_tokens:
            if self.counts is not None:
                shape.M_cap = B.tempo_m_cap_bound(shape)
                B.tempo_count_dispatch(shape, ids, n_valid, self.replica_map, self.quota, self.cum_counts, self.counts,
                                       *self.few_dispatch, self.status)
            ffn = B.tempo_few_ffn_bf16 if self.bf16 else B.tempo_few_ffn
            ffn(shape, x, ids, w, n_valid, self.replica_map, self.packed, y, self.status, self.workspace)
        else:
            self.block.n_valid = n_valid
            (self.block.run_block_bf16 if self.bf16 else self.block.run_block)(T=T)
        next_w, next_b = (self.next_w, self.next_b) if x_next is not None else (None, None)
        B.tempo_norm_out(y, r, r_out, post_w=self.post_w, post_b=self.post_b, gate=self.gate if gate is None else gate,
                         next_w=next_w, next_b=next_b, x_out=x_next, kind=self.kind, eps=self.eps, r_scale=self.r_scale,
                         y_scale=self.y_scale, n_valid=n_valid)
        return r_out


class Attention:
    """One layer's 4-bit cache of keys and values, and the buffers of its calls.

    n_pages, page_size   the cache: pages of 16, 32, 64, 128 or 256 tokens
    Hq, Hkv, D           query heads, key heads (a divisor of Hq), elements of a head (64 or 128)
    max_tokens           largest batch (rows of the buffers)
    cos_sin              f32 [positions, rot]: cos, then sin, of rot / 2 pairs' angles; None: heads are not rotated
    q_w, k_w             weights [D] of the heads' RMS norms (one dtype) or None: not normed
    interleaved          pairs are neighbours instead of (i, i + rot / 2)
    scale                of the scores; None: D ** -0.5

    A layer has one query buffer and one workspace: its calls must follow one another on one stream (or be ordered by events).
    `status` collects the STATUS_* bits of every call; after STATUS_TIMEOUT `workspace` has to be zeroed.
    """

    def __init__(self, n_pages, page_size, Hq, Hkv, D, max_tokens, cos_sin=None, q_w=None, k_w=None, eps=1e-6, interleaved=False,
                 scale=None, device="cuda"):
        self.Hq, self.Hkv, self.D, self.eps, self.interleaved, self.scale = Hq, Hkv, D, eps, interleaved, scale
        self.cos_sin, self.q_w, self.k_w = cos_sin, q_w, k_w
        self.shape = B.make_cache(n_pages, page_size, Hkv, D)
        u8 = dict(dtype=torch.uint8, device=device)
        self.cache = torch.empty(B.tempo_cache_bytes(self.shape), **u8)
        self.workspace = torch.zeros(B.tempo_attend_workspace_bytes(self.shape, Hq), **u8)
        self.q = torch.empty(max_tokens, Hq, D, dtype=torch.bfloat16, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)

    def forward(self, qkv, positions, slots, page_table, lens, out, q_start=None, max_q=None, n_valid=None):
        """out = attention of this batch's tokens, which are appended to the cache first.

        qkv bf16 [T, (Hq + 2 Hkv) * D]: a projection's rows (queries, keys, values); out bf16 [T, Hq, D] or [T, Hq * D].
        positions, slots i32 [T]: of the rotation, and where in the cache (page * page_size + offset; below zero: not appended).
        page_table i32 [B, pages], lens i32 [B]: the sequences with this batch's tokens; q_start i32 [B + 1]: their rows (None: one
        each), max_q the most of one (None: 1 without q_start, else by the sizes).  n_valid i32 [1]: rows behind it are neither
        appended nor read, and their rows of out stay as they are.  Enqueues kernels only: the call can be captured in a CUDA graph."""
        T = qkv.shape[0]
        if T > self.q.shape[0]:
            raise B.TempoError(f"a batch of {T} tokens exceeds the layer's {self.q.shape[0]}")
        q, k, v = qkv.unflatten(1, (-1, self.D)).split([self.Hq, self.Hkv, self.Hkv], dim=1)
        turned = self.q[:T]
        turn = dict(positions=positions, cos_sin=self.cos_sin) if self.cos_sin is not None else {}
        B.tempo_kv_append(self.shape, k, v, slots, self.cache, self.status, k_w=self.k_w, q=q, q_w=self.q_w, q_out=turned, eps=self.eps,
                          interleaved=self.interleaved, n_valid=n_valid, **turn)
        B.tempo_attend(self.shape, turned, self.cache, page_table, lens, out.view(T, self.Hq, self.D), self.status, self.workspace,
                       scale=self.scale, q_start=q_start, max_q=max_q, n_valid=n_valid)
        return out

    def read(self, slots):
        """The cache's tokens at slots i32 [n] as fp16 [n, Hkv, D] keys and values: to move a sequence, or to keep its prefix."""
        k, v = (torch.empty(slots.shape[0], self.Hkv, self.D, dtype=torch.float16, device=self.cache.device) for _ in range(2))
        B.tempo_kv_read(self.shape, self.cache, slots, k, v, self.status)
        return k, v
