"""A Llama-shaped decoder stack driven through the C-ABI binding: per layer, the model steps around the path
(RMSNorm, Q/K/V projection with RoPE, output projection, SwiGLU feed-forward) for the recomputed rows only,
with the selective-prefill calls in between.  Argument marshalling and buffer management only: every step runs
in the library's kernels.  Weights are random (there are no checkpoints here); the shapes are the model's."""
from __future__ import annotations

import dataclasses
from typing import List, Optional

import torch

from . import binding as B


@dataclasses.dataclass
class LayerWeights:
    g1: torch.Tensor          # [hidden]
    w_qkv: torch.Tensor       # [(Hq + 2 Hkv) d, hidden]: query heads, key heads, value heads
    w_o: torch.Tensor         # [hidden, Hq d]
    g2: torch.Tensor          # [hidden]
    w_gate_up: torch.Tensor   # [2 ffn, hidden]: gate and up rows interleaved
    w_down: torch.Tensor      # [hidden, ffn]


def random_layer(hidden: int, ffn: int, Hq: int, Hkv: int, d: int, gen: torch.Generator, std: float = 0.02,
                 device: str = "cuda") -> LayerWeights:
    def w(n, k):
        return (torch.randn((n, k), generator=gen, device=device, dtype=torch.float32) * std).to(torch.bfloat16)
    ones = torch.ones(hidden, dtype=torch.bfloat16, device=device)
    return LayerWeights(ones.clone(), w((Hq + 2 * Hkv) * d, hidden), w(hidden, Hq * d), ones.clone(),
                        w(2 * ffn, hidden), w(hidden, ffn))


class SelectivePrefillStack:
    """Runs `layers` decoder layers over the rows listed in a Q index.  Per layer (the order of the full-stack
    configuration): Q/K/V projection of the rows, fr_rope_shift of that layer's cached keys, optionally
    fr_score_select on the layer's own question queries (result discarded: the row set of a sparse prefill is
    fixed before the first layer), fr_sparse_prefill_attn, fr_kv_scatter, output projection and feed-forward."""

    def __init__(self, ctx: B.Context, layers: List[LayerWeights], hidden: int, ffn: int, eps: float = 1e-5):
        self.ctx, self.layers, self.hidden, self.ffn, self.eps = ctx, layers, hidden, ffn, eps
        d = ctx.desc
        self.Hq, self.Hkv, self.d = d.n_q_heads, d.n_kv_heads, d.head_dim
        self._buf = {}

    def _scratch(self, R: int):
        if self._buf.get("R") != R:
            dev, bf = "cuda", torch.bfloat16
            self._buf = dict(
                R=R, x=torch.empty((R, self.hidden), dtype=bf, device=dev),
                q=torch.empty((R, self.Hq, self.d), dtype=bf, device=dev),
                k=torch.empty((R, self.Hkv, self.d), dtype=bf, device=dev),
                v=torch.empty((R, self.Hkv, self.d), dtype=bf, device=dev),
                attn=torch.empty((R, self.Hq, self.d), dtype=bf, device=dev),
                act=torch.empty((R, self.ffn), dtype=bf, device=dev))
        return self._buf

    def forward(self, h: torch.Tensor, q_index: torch.Tensor, k_cached: List[torch.Tensor], k_cache: List[torch.Tensor],
                v_cache: List[torch.Tensor], chunk_offsets, src_pos0, nq: int, L: int, select_every_layer: bool = False,
                k_select: int = 0, q_index_scratch: Optional[torch.Tensor] = None,
                capture: Optional[dict] = None) -> torch.Tensor:
        """h [R, hidden] is updated in place and returned; k_cache / v_cache [L, Hkv, d] per layer end up holding
        the stitched cache with the recomputed rows written back.  `capture`, if given, maps layer numbers to dicts
        that receive copies of the layer's input and output rows ("h_in", "h_out"): tests feed the input to the oracle."""
        c, R = self.ctx, h.shape[0]
        s = self._scratch(R)
        for l, w in enumerate(self.layers):
            if capture is not None and l in capture:
                capture[l]["h_in"] = h.clone()
            c.fr_rmsnorm(h, w.g1, R, self.hidden, self.eps, s["x"])
            c.fr_qkv_rope(s["x"], w.w_qkv, R, self.hidden, q_index, s["q"], s["k"], s["v"])
            c.fr_rope_shift(k_cached[l], k_cache[l], chunk_offsets, src_pos0)
            if select_every_layer:
                c.fr_score_select(s["q"][R - nq:], nq, k_cache[l], chunk_offsets, k_select, B.FR_NORM_PER_CHUNK, None,
                                  q_index_scratch)
            c.fr_sparse_prefill_attn(s["q"], q_index, R, k_cache[l], v_cache[l], L, s["k"], s["v"], s["attn"])
            c.fr_kv_scatter(s["k"], s["v"], q_index, R, k_cache[l], v_cache[l], L)
            c.fr_linear(s["attn"], w.w_o, R, self.hidden, self.Hq * self.d, h, h)
            c.fr_rmsnorm(h, w.g2, R, self.hidden, self.eps, s["x"])
            c.fr_linear_swiglu(s["x"], w.w_gate_up, R, self.ffn, self.hidden, s["act"])
            c.fr_linear(s["act"], w.w_down, R, self.hidden, self.ffn, h, h)
            if capture is not None and l in capture:
                capture[l]["h_out"] = h.clone()
        return h


class PagedCache:
    """K/V of up to `n_requests` requests in pages of `page_rows` rows, for every layer; one free list and one block table serve all layers.
    Lengths and tables stay on the device (a captured step serves other lengths).  A step that asks for more pages than the list has
    leaves the rows without one out of the cache: `free_start` is beyond `n_pages` then.  A request that ends is taken out by its
    length 0 and new entries of `free_pages`; the list may be rewritten between steps."""

    def __init__(self, n_layers: int, n_requests: int, n_pages: int, page_rows: int, max_blocks: int, Hkv: int, d: int,
                 dtype=torch.bfloat16):
        i32 = dict(dtype=torch.int32, device="cuda")
        shape = (n_pages, page_rows, Hkv, d)
        self.k = [torch.zeros(shape, dtype=dtype, device="cuda") for _ in range(n_layers)]
        self.v = [torch.zeros(shape, dtype=dtype, device="cuda") for _ in range(n_layers)]
        self.n_requests, self.n_pages, self.page_rows, self.max_blocks = n_requests, n_pages, page_rows, max_blocks
        self.block_table = torch.full((n_requests, max_blocks), -1, **i32)
        self.cached_len = torch.zeros(n_requests, **i32)
        self.free_pages = torch.arange(n_pages, **i32)
        self.free_start, self.pages_needed = torch.zeros(1, **i32), torch.zeros(1, **i32)


class PagedStack:
    """Decoder layers over a paged cache: a step appends new_len[b] rows to every request b (a decoding step, drafted tokens, a chunk of
    a prompt, a whole prompt, side by side) and computes them.  Per layer: RMSNorm, Q/K/V projection with each row's own position,
    fr_paged_append, fr_paged_attn, output projection and feed-forward."""

    def __init__(self, ctx: B.Context, layers: List[LayerWeights], hidden: int, ffn: int, eps: float = 1e-5):
        self.ctx, self.layers, self.hidden, self.ffn, self.eps = ctx, layers, hidden, ffn, eps
        d = ctx.desc
        self.Hq, self.Hkv, self.d = d.n_q_heads, d.n_kv_heads, d.head_dim
        # fr_qkv_rope rotates rows of this layout itself; others are projected part by part and rotated on the way into the pages
        self.fused_rope = d.head_dim == 128 and d.rope_layout == B.FR_ROPE_INTERLEAVED
        if not self.fused_rope and (self.Hq * self.d % 128 or self.Hkv * self.d % 128):
            raise ValueError(f"{self.Hq} / {self.Hkv} heads of {self.d}: queries, keys and values are projected by themselves, and fr_linear takes multiples of 128 features")
        self._buf, self._captured = {}, {}

    def _scratch(self, T: int, n: int):
        capturing = torch.cuda.is_current_stream_capturing()
        key = T, n, torch.cuda.current_stream().cuda_stream   # (freed buffers go back to the stream that they were taken on: a step on another one takes its own)
        if not capturing and self._buf.get("key") == key:
            return self._buf
        if capturing and (T, n) in self._captured:
            return self._captured[T, n]
        mk = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        i32 = lambda m: torch.empty(m, dtype=torch.int32, device="cuda")
        buf = dict(key=key, x=mk(T, self.hidden), q=mk(T, self.Hq, self.d), k=mk(T, self.Hkv, self.d), v=mk(T, self.Hkv, self.d),
                   attn=torch.zeros((T, self.Hq, self.d), dtype=torch.bfloat16, device="cuda"), act=mk(T, self.ffn),
                   offsets=i32(n + 1), positions=i32(T), slots=i32(T))
        if capturing:
            self._captured[T, n] = buf   # the graphs' of this size (the context's calls are in order, so they never run at once): steps of other sizes do not free it
        else:
            self._buf = buf
        return buf

    def release(self):
        """Gives back the buffers of all steps, captured ones too: for when no graph of this stack will be replayed again."""
        self._buf, self._captured = {}, {}

    def forward(self, h: torch.Tensor, new_len: torch.Tensor, max_new: int, cache: PagedCache) -> torch.Tensor:
        """h [T, hidden] is updated in place and returned: the requests' rows one after the other, rows behind them hold nothing of use.
        A captured step holds its buffers until release(); graphs of one size share them.
        new_len [n_requests] int32 on the device, none beyond max_new.  With head_dim 128 and interleaved pairs T is at most the
        context's max_tokens (fr_qkv_rope).  The cache's lengths and free list move on."""
        c, T, n = self.ctx, h.shape[0], cache.n_requests
        s = self._scratch(T, n)
        c.fr_page_tables(cache.cached_len, new_len, n, cache.page_rows, cache.free_pages, cache.n_pages, cache.free_start, cache.block_table,
                         cache.max_blocks, T, s["offsets"], s["positions"], s["slots"], cache.pages_needed)
        nq, nk = self.Hq * self.d, self.Hkv * self.d
        for l, w in enumerate(self.layers):
            kp, vp = cache.k[l], cache.v[l]
            c.fr_rmsnorm(h, w.g1, T, self.hidden, self.eps, s["x"])
            if self.fused_rope:
                c.fr_qkv_rope(s["x"], w.w_qkv, T, self.hidden, s["positions"], s["q"], s["k"], s["v"])
                c.fr_paged_append(None, s["k"], s["v"], None, s["slots"], T, kp, vp, cache.n_pages, cache.page_rows)
            else:
                for out, at, rows in ((s["q"], 0, nq), (s["k"], nq, nk), (s["v"], nq + nk, nk)):
                    c.fr_linear(s["x"], w.w_qkv[at: at + rows], T, rows, self.hidden, None, out)
                c.fr_paged_append(s["q"], s["k"], s["v"], s["positions"], s["slots"], T, kp, vp, cache.n_pages, cache.page_rows, s["q"])
            c.fr_paged_attn(s["q"], s["offsets"], cache.cached_len, n, T, max_new, kp, vp, cache.n_pages, cache.page_rows, cache.block_table,
                            cache.max_blocks, s["attn"])
            c.fr_linear(s["attn"], w.w_o, T, self.hidden, nq, h, h)
            c.fr_rmsnorm(h, w.g2, T, self.hidden, self.eps, s["x"])
            c.fr_linear_swiglu(s["x"], w.w_gate_up, T, self.ffn, self.hidden, s["act"])
            c.fr_linear(s["act"], w.w_down, T, self.hidden, self.ffn, h, h)
        cache.cached_len += s["offsets"][1:] - s["offsets"][:-1]
        cache.free_start += cache.pages_needed
        return h
