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
    q_norm: Optional[torch.Tensor] = None   # [d]: gains of layers that normalise queries and keys per head, both or neither
    k_norm: Optional[torch.Tensor] = None


@dataclasses.dataclass
class HeadWeights:
    g: torch.Tensor           # [hidden]: the norm behind the last layer
    w: torch.Tensor           # [vocabulary, hidden]


def random_layer(hidden: int, ffn: int, Hq: int, Hkv: int, d: int, gen: torch.Generator, std: float = 0.02,
                 device: str = "cuda", qk_norm: bool = False) -> LayerWeights:
    def w(n, k):
        return (torch.randn((n, k), generator=gen, device=device, dtype=torch.float32) * std).to(torch.bfloat16)
    ones = torch.ones(hidden, dtype=torch.bfloat16, device=device)
    gains = [(torch.rand(d, generator=gen, device=device) + 0.5).to(torch.bfloat16) for _ in range(2)] if qk_norm else [None, None]
    return LayerWeights(ones.clone(), w((Hq + 2 * Hkv) * d, hidden), w(hidden, Hq * d), ones.clone(),
                        w(2 * ffn, hidden), w(hidden, ffn), *gains)


def random_head(hidden: int, vocab: int, gen: torch.Generator, std: float = 0.02, device: str = "cuda") -> HeadWeights:
    w = (torch.randn((vocab, hidden), generator=gen, device=device, dtype=torch.float32) * std).to(torch.bfloat16)
    return HeadWeights(torch.ones(hidden, dtype=torch.bfloat16, device=device), w)


def _int32(**arrays: Optional[torch.Tensor]):
    for name, t in arrays.items():
        if t is not None and t.dtype != torch.int32:
            raise ValueError(f"{name} is of {t.dtype}: the library reads int32")


def _sized(**arrays):
    """(tensor or None, its length) each."""
    for name, (t, n) in arrays.items():
        if t is not None and t.shape != (n,):
            raise ValueError(f"{name} has shape {tuple(t.shape)}, not ({n},)")


def _rows(h: torch.Tensor, hidden: int, **beside: Optional[torch.Tensor]):
    """h [T, hidden] as the library reads it, and what stands on the same device."""
    if h.dim() != 2 or h.shape[1] != hidden:
        raise ValueError(f"h has shape {tuple(h.shape)}, not (rows, {hidden})")
    if h.dtype != torch.bfloat16:
        raise ValueError(f"h is of {h.dtype}: the library reads bfloat16")
    for name, t in beside.items():
        if t is not None and t.device != h.device:
            raise ValueError(f"{name}: on {t.device}, h on {h.device}")
    if not h.is_cuda or h.device.index != torch.cuda.current_device():
        raise ValueError(f"h: on {h.device}, not on the current GPU")


def _normed(layers: List[LayerWeights]) -> bool:
    """Whether layers normalise queries and keys per head."""
    if any((w.q_norm is None) != (w.k_norm is None) for w in layers):
        raise ValueError("q_norm and k_norm: both or neither")
    return any(w.q_norm is not None for w in layers)


class SelectivePrefillStack:
    """Runs `layers` decoder layers over the rows listed in a Q index.  Per layer (the order of the full-stack
    configuration): Q/K/V projection of the rows, fr_rope_shift of that layer's cached keys, optionally
    fr_score_select on the layer's own question queries (result discarded: the row set of a sparse prefill is
    fixed before the first layer), fr_sparse_prefill_attn, fr_kv_scatter, output projection and feed-forward."""

    def __init__(self, ctx: B.Context, layers: List[LayerWeights], hidden: int, ffn: int, eps: float = 1e-5):
        self.ctx, self.layers, self.hidden, self.ffn, self.eps = ctx, layers, hidden, ffn, eps
        d = ctx.desc
        self.Hq, self.Hkv, self.d = d.n_q_heads, d.n_kv_heads, d.head_dim
        self.normed = _normed(layers)
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
            if self.normed:
                self._buf["qkv"] = torch.empty((R, self.Hq + 2 * self.Hkv, self.d), dtype=bf, device=dev)
        return self._buf

    def _project(self, w: LayerWeights, R: int, positions: torch.Tensor, s: dict):
        """The rows' queries, keys and values at their positions."""
        if w.q_norm is None:
            self.ctx.fr_qkv_rope(s["x"], w.w_qkv, R, self.hidden, positions, s["q"], s["k"], s["v"])
            return
        heads = [self.Hq, self.Hkv, self.Hkv]
        self.ctx.fr_linear(s["x"], w.w_qkv, R, sum(heads) * self.d, self.hidden, None, s["qkv"])
        q, k, v = s["qkv"].split(heads, 1)
        self.ctx.fr_qk_norm_append(q, k, v, w.q_norm, w.k_norm, self.eps, positions, None, R, s["k"], s["v"], R, 1, s["q"])   # (rows, one to a "page")

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
            self._project(w, R, q_index, s)
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
    leaves the rows without one out of the cache: `free_start` is beyond `n_pages` then (verify() gives pages back and returns how far it was).  A request that ends is taken out by its
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


class Head:
    """What stands behind the last layer: its norm, the projection to the vocabulary and the log probabilities of tokens.  The logits of `rows_at_once` rows are held at a time."""

    def __init__(self, ctx: B.Context, w: HeadWeights, eps: float = 1e-5, rows_at_once: int = 4096):
        self.ctx, self.w, self.eps, self.rows_at_once = ctx, w, eps, rows_at_once
        self.vocab, self.hidden = w.w.shape
        if self.vocab % 128 or self.hidden % 64:
            raise ValueError(f"{self.vocab} tokens, {self.hidden} features: fr_linear takes multiples of 128 and of 64")
        if rows_at_once < 1:
            raise ValueError(f"rows_at_once = {rows_at_once} is not positive")
        _sized(g=(w.g, self.hidden))

    def check(self, h: torch.Tensor, **beside: Optional[torch.Tensor]):
        """Refuses rows that are not the head's, and arrays of another device (the library takes addresses)."""
        if self.w.w.dtype != torch.bfloat16 or self.w.g.dtype != torch.bfloat16:
            raise ValueError(f"the head's weights are of {self.w.w.dtype}, its norm of {self.w.g.dtype}: the library reads bfloat16")
        _rows(h, self.hidden, weights=self.w.w, norm=self.w.g, **beside)

    def logprobs(self, h: torch.Tensor, tokens: Optional[torch.Tensor] = None, n_top: int = 1, scale: float = 1.0) -> dict:
        """Of the rows h [T, hidden] (fr_token_logprobs): "logprobs" [T] of the tokens, if any are given, "entropy" and "lse" [T], "top_ids" and "top_logprobs" [T, n_top];
        scale = 1 / temperature."""
        _int32(tokens=tokens)
        T = h.shape[0]
        _sized(tokens=(tokens, T))
        self.check(h, tokens=tokens)
        f32 = lambda *shape: torch.empty(shape, dtype=torch.float32, device=h.device)
        out = dict(logprobs=f32(T) if tokens is not None else None, entropy=f32(T), lse=f32(T),
                   top_ids=torch.empty((T, n_top), dtype=torch.int32, device=h.device), top_logprobs=f32(T, n_top))
        n = min(T, self.rows_at_once)
        x, logits = torch.empty((n, self.hidden), dtype=h.dtype, device=h.device), torch.empty((n, self.vocab), dtype=h.dtype, device=h.device)
        for at in range(0, T, max(n, 1)):
            m = min(n, T - at)
            part = lambda t: None if t is None else t[at: at + m]
            self.ctx.fr_rmsnorm(part(h), self.w.g, m, self.hidden, self.eps, x)
            self.ctx.fr_linear(x, self.w.w, m, self.vocab, self.hidden, None, logits)
            self.ctx.fr_token_logprobs(logits, B.FR_BF16, self.vocab, m, self.vocab, scale, part(tokens), n_top, part(out["logprobs"]), part(out["entropy"]), part(out["lse"]),
                                       part(out["top_ids"]), part(out["top_logprobs"]))
        return out


class PagedStack:
    """Decoder layers over a paged cache: a step appends new_len[b] rows to every request b (a decoding step, drafted tokens, a chunk of
    a prompt, a whole prompt, side by side) and computes them.  Per layer: RMSNorm, Q/K/V projection with each row's own position,
    fr_paged_append (fr_qk_norm_append in layers with norms of queries and keys), fr_paged_attn, output projection and feed-forward.
    verify() is a step whose rows are trees of drafted tokens, of which those stay in the cache that the model agrees with."""

    def __init__(self, ctx: B.Context, layers: List[LayerWeights], hidden: int, ffn: int, eps: float = 1e-5):
        self.ctx, self.layers, self.hidden, self.ffn, self.eps = ctx, layers, hidden, ffn, eps
        d = ctx.desc
        self.Hq, self.Hkv, self.d = d.n_q_heads, d.n_kv_heads, d.head_dim
        # fr_qkv_rope rotates rows of this layout itself; others are projected part by part and rotated on the way into the pages
        self.normed = _normed(layers)
        self.fused_rope = d.head_dim == 128 and d.rope_layout == B.FR_ROPE_INTERLEAVED
        plain = not layers or any(w.q_norm is None for w in layers)
        if self.normed and (self.Hq + 2 * self.Hkv) * self.d % 128:
            raise ValueError(f"{self.Hq} + 2 x {self.Hkv} heads of {self.d}: they are projected at once, and fr_linear takes multiples of 128 features")
        if plain and not self.fused_rope and (self.Hq * self.d % 128 or self.Hkv * self.d % 128):
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
        if self.normed:
            buf["qkv"] = mk(T, self.Hq + 2 * self.Hkv, self.d)
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
        _int32(new_len=new_len)
        _sized(new_len=(new_len, n))
        _rows(h, self.hidden, new_len=new_len)
        s = self._scratch(T, n)
        self._tables(new_len, T, cache, s)

        def attend(kp, vp):
            c.fr_paged_attn(s["q"], s["offsets"], cache.cached_len, n, T, max_new, kp, vp, cache.n_pages, cache.page_rows, cache.block_table, cache.max_blocks, s["attn"])
        self._layers(h, s["positions"], cache, s, attend)
        cache.cached_len += s["offsets"][1:] - s["offsets"][:-1]
        cache.free_start += cache.pages_needed
        return h

    def verify(self, h: torch.Tensor, parents: torch.Tensor, tokens: torch.Tensor, new_len: torch.Tensor, max_new: int, cache: PagedCache, head: Head,
               given: Optional[torch.Tensor] = None) -> dict:
        """A step whose rows are trees: row 0 of a request is its last token, every other one a drafted token behind its parent (fr_tree_tables), or with `given` [n_requests]
        the first given[b] rows are not drafts but a chunk, each behind the one before.  h [T, hidden] as in forward; parents and tokens [T], new_len [n_requests] int32 on the device, none beyond
        max_new <= FR_TREE_MAX_ROWS.  The drafts stay that the model agrees with (its likeliest token after a row is a draft behind it), in every layer's pages at
        consecutive positions; the cache's lengths and free list move on by them alone.
        Returns "kept" [n_requests] rows that stay, "path" [T] which ones they are, "next_token" [n_requests] the model's token behind them, "free_end" [1] the index in the
        free list behind the pages that the step took (beyond cache.n_pages: the list was too short.  Rows without a page are not in the cache and do not see themselves, and where one of
        them stays its position may hold another draft's row: such a request is best computed again), and of every row "choice", its likeliest token, "logprob" of it and "entropy"."""
        c, T, n = self.ctx, h.shape[0], cache.n_requests
        if max_new > B.FR_TREE_MAX_ROWS:
            raise ValueError(f"max_new = {max_new}: a tree has at most {B.FR_TREE_MAX_ROWS} rows")
        _int32(parents=parents, tokens=tokens, new_len=new_len, given=given)
        _sized(parents=(parents, T), tokens=(tokens, T), new_len=(new_len, n), given=(given, n))
        if len(cache.k) > B.FR_TREE_MAX_LAYERS:
            raise ValueError(f"the cache has {len(cache.k)} layers: fr_tree_keep moves the rows of {B.FR_TREE_MAX_LAYERS} at most")
        if head.hidden != self.hidden:
            raise ValueError(f"a head of {head.hidden} features behind layers of {self.hidden}")
        head.check(h, parents=parents, tokens=tokens, new_len=new_len, given=given)
        s = self._scratch(T, n)
        words = max(1, -(-max_new // 32))
        i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device=h.device)
        positions, mask, kept, path, next_token = i32(T), i32(T, words), i32(n), torch.full((T,), -1, dtype=torch.int32, device=h.device), i32(n)
        self._tables(new_len, T, cache, s)
        c.fr_tree_tables(parents, s["offsets"], cache.cached_len, n, T, max_new, positions, mask, words)

        def attend(kp, vp):
            c.fr_paged_tree_attn(s["q"], s["offsets"], cache.cached_len, n, T, max_new, mask, words, kp, vp, cache.n_pages, cache.page_rows, cache.block_table, cache.max_blocks,
                                 s["attn"])
        self._layers(h, positions, cache, s, attend)
        answer = head.logprobs(h)
        choice = answer["top_ids"].view(T)
        free_end = cache.free_start + cache.pages_needed
        c.fr_tree_keep(parents, tokens, choice, s["offsets"], cache.cached_len, given, n, T, max_new, cache.k, cache.v, cache.n_pages, cache.page_rows, cache.block_table,
                       cache.max_blocks, cache.free_pages, cache.n_pages, free_end, cache.free_start, kept, path, next_token)
        cache.cached_len += kept
        return dict(kept=kept, path=path, next_token=next_token, free_end=free_end, choice=choice, logprob=answer["top_logprobs"].view(T), entropy=answer["entropy"])

    def _tables(self, new_len: torch.Tensor, T: int, cache: PagedCache, s: dict):
        self.ctx.fr_page_tables(cache.cached_len, new_len, cache.n_requests, cache.page_rows, cache.free_pages, cache.n_pages, cache.free_start, cache.block_table,
                                cache.max_blocks, T, s["offsets"], s["positions"], s["slots"], cache.pages_needed)

    def _layers(self, h: torch.Tensor, positions: torch.Tensor, cache: PagedCache, s: dict, attend):
        c, T = self.ctx, h.shape[0]
        nq, nk = self.Hq * self.d, self.Hkv * self.d
        for l, w in enumerate(self.layers):
            kp, vp = cache.k[l], cache.v[l]
            c.fr_rmsnorm(h, w.g1, T, self.hidden, self.eps, s["x"])
            if w.q_norm is not None:
                c.fr_linear(s["x"], w.w_qkv, T, nq + 2 * nk, self.hidden, None, s["qkv"])
                q, k, v = s["qkv"].split([self.Hq, self.Hkv, self.Hkv], 1)
                c.fr_qk_norm_append(q, k, v, w.q_norm, w.k_norm, self.eps, positions, s["slots"], T, kp, vp, cache.n_pages, cache.page_rows, s["q"])
            elif self.fused_rope:
                c.fr_qkv_rope(s["x"], w.w_qkv, T, self.hidden, positions, s["q"], s["k"], s["v"])
                c.fr_paged_append(None, s["k"], s["v"], None, s["slots"], T, kp, vp, cache.n_pages, cache.page_rows)
            else:
                for out, at, rows in ((s["q"], 0, nq), (s["k"], nq, nk), (s["v"], nq + nk, nk)):
                    c.fr_linear(s["x"], w.w_qkv[at: at + rows], T, rows, self.hidden, None, out)
                c.fr_paged_append(s["q"], s["k"], s["v"], positions, s["slots"], T, kp, vp, cache.n_pages, cache.page_rows, s["q"])
            attend(kp, vp)
            c.fr_linear(s["attn"], w.w_o, T, self.hidden, nq, h, h)
            c.fr_rmsnorm(h, w.g2, T, self.hidden, self.eps, s["x"])
            c.fr_linear_swiglu(s["x"], w.w_gate_up, T, self.ffn, self.hidden, s["act"])
            c.fr_linear(s["act"], w.w_down, T, self.hidden, self.ffn, h, h)
