"""Decoder layers over a paged cache against the 64-bit oracle's layer, and what captured steps hold."""
import numpy as np
import pytest
import torch

from oracle import fusionrag_oracle as orc
from paper_2601_12904_amd import stack as S
from paper_2601_12904_amd import synth
from tests import harness as H
from tests.test_gpu_paged import i32, make_ctx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,d,half", [(8, 2, 128, False), (8, 2, 128, True), (6, 2, 64, True), (8, 4, 64, False)])
def test_steps_against_the_oracles_layer(Hq, Hkv, d, half):
    """Three steps of three requests through two layers, prompts, chunks and single rows: every request's rows, and the keys and values in its pages, against the oracle, which
    takes each request by itself and follows the steps store by store.  Both layouts, fused rotary embedding and three projections."""
    hidden, ffn, L, page, base, eps = 256, 384, 2, 8, 5e5, 1e-5
    gen = torch.Generator(device="cuda").manual_seed(11)
    layers = [S.random_layer(hidden, ffn, Hq, Hkv, d, gen, std=0.08) for _ in range(L)]
    for w in layers:   # (gains of ones would hide where they are taken)
        w.g1.copy_((torch.rand(hidden, generator=gen, device="cuda") + 0.5).bfloat16())
        w.g2.copy_((torch.rand(hidden, generator=gen, device="cuda") + 0.5).bfloat16())
    weights = [{n: H.host(getattr(w, n)) for n in ("g1", "w_qkv", "w_o", "g2", "w_gate_up", "w_down")} for w in layers]
    ctx = make_ctx((Hq, Hkv, d, "bf16"), half, base=base, tokens=128)
    stack = S.PagedStack(ctx, layers, hidden, ffn, eps)
    cache = S.PagedCache(L, 3, 40, page, 12, Hkv, d)
    rnd = lambda t: synth.round_to_storage(np.asarray(t, dtype=np.float32), "bf16").astype(np.float64)
    held = [[(np.zeros((0, Hkv, d)), np.zeros((0, Hkv, d))) for _ in range(L)] for _ in range(3)]
    turn = lambda x, pos: orc.rope_rotate(x, pos, base, "half" if half else "interleaved")
    for new in ([20, 7, 0], [1, 30, 5], [33, 1, 1]):
        h0 = torch.randn((sum(new) + 2, hidden), generator=gen, device="cuda").bfloat16()
        start = H.host(h0)
        h = stack.forward(h0.clone(), i32(new), max(new), cache)
        got = H.host(h)
        at = 0
        for b, n in enumerate(new):
            if n == 0:
                continue
            rows, c = start[at: at + n], len(held[b][0][0])
            pos = np.arange(c, c + n)
            for l, w in enumerate(weights):
                x = rnd(orc.rmsnorm(rows, w["g1"], eps))
                y = rnd(orc.linear(x, w["w_qkv"]))      # (both ways are within a rounding of this one: the unfused one stores the projection before it is rotated)
                q, k, v = (y[:, lo: hi].reshape(n, -1, d) for lo, hi in ((0, Hq * d), (Hq * d, (Hq + Hkv) * d), ((Hq + Hkv) * d, (Hq + 2 * Hkv) * d)))
                K, V = np.concatenate([held[b][l][0], rnd(turn(k, pos))]), np.concatenate([held[b][l][1], v])
                held[b][l] = (K, V)
                full = np.concatenate([np.zeros((c, Hq, d)), rnd(turn(q, pos))])
                attn = rnd(orc.full_causal_attention(full, K, V)[c:]).reshape(n, Hq * d)
                h1 = rnd(orc.linear(attn, w["w_o"], rows))
                act = rnd(orc.linear_swiglu(rnd(orc.rmsnorm(h1, w["g2"], eps)), w["w_gate_up"]))
                rows = rnd(orc.linear(act, w["w_down"], h1))
                blocks = cache.block_table[b, : -(-(c + n) // page)].long()
                for name, pages, want in (("keys", cache.k[l], K), ("values", cache.v[l], V)):
                    H.assert_close(H.host(pages[blocks]).reshape(-1, Hkv, d)[: c + n], want, "bf16", f"request {b}, layer {l}: {name}")
            H.assert_close(got[at: at + n], rows, "bf16", f"request {b}: rows")
            at += n
    ctx.close()


def test_captures_of_one_size_share_their_buffers():
    """A server that captures its step again and again holds one set of buffers for each size, and none after release()."""
    Hq, Hkv, d, hidden, ffn, L, n = 8, 2, 128, 512, 256, 1, 2
    gen = torch.Generator(device="cuda").manual_seed(5)
    layers = [S.random_layer(hidden, ffn, Hq, Hkv, d, gen, std=0.05) for _ in range(L)]
    ctx = make_ctx((Hq, Hkv, d, "bf16"), tokens=4096)
    stack = S.PagedStack(ctx, layers, hidden, ffn)
    cache = S.PagedCache(L, n, 60, 8, 16, Hkv, d)
    T, rows = 4096, torch.randn((3, hidden), generator=gen, device="cuda").bfloat16()
    new = i32([0] * n)
    h = torch.zeros((T, hidden), device="cuda").bfloat16()
    stack.forward(h, new, 8, cache)          # (once outside)
    torch.cuda.synchronize()
    held, results = [], []
    for _ in range(4):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            stack.forward(h, new, 8, cache)
        for _ in range(2):
            cache.cached_len.zero_(); cache.free_start.zero_()
            new.copy_(i32([2, 1]))
            h[:3] = rows
            graph.replay()
            torch.cuda.synchronize()
            results.append(h[:3].clone())
            new.zero_()
            stack.forward(torch.zeros((5, hidden), device="cuda").bfloat16(), new, 5, cache)      # another size between the replays
        held.append(torch.cuda.memory_allocated())
        if len(held) < 4:
            del graph
    assert all(torch.equal(r, results[0]) for r in results) and bool(torch.isfinite(results[0].float()).all())
    one = T * (hidden + Hq * d) * 2          # less than a set of buffers takes
    assert held[-1] - held[0] < one, "captures of one size add up"
    del graph
    stack.release()
    assert torch.cuda.memory_allocated() < held[0] - one
    ctx.close()


def test_steps_on_two_streams_take_buffers_of_their_own():
    """Steps on a second stream, behind one on the first: the first one's buffers, which go back to the first stream when they are dropped, are not among those that they use."""
    Hq, Hkv, d, hidden, ffn, n = 8, 2, 128, 512, 256, 2
    gen = torch.Generator(device="cuda").manual_seed(5)
    layers = [S.random_layer(hidden, ffn, Hq, Hkv, d, gen, std=0.05)]
    ctx = make_ctx((Hq, Hkv, d, "bf16"), tokens=64)
    stack = S.PagedStack(ctx, layers, hidden, ffn)
    rows = torch.randn((3, hidden), generator=gen, device="cuda").bfloat16()
    seen, append = {}, ctx.fr_paged_append

    def spy(q, k_new, *rest):
        seen.setdefault(torch.cuda.current_stream().cuda_stream, set()).add(k_new.data_ptr())
        return append(q, k_new, *rest)
    ctx.fr_paged_append = spy
    got = []
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for i in (0, 1, 1, 0):
        torch.cuda.synchronize()
        with torch.cuda.stream(streams[i]):
            cache = S.PagedCache(1, n, 20, 8, 8, Hkv, d)
            got.append(stack.forward(rows.clone(), i32([2, 1]), 2, cache))
    torch.cuda.synchronize()
    assert all(torch.equal(g, got[0]) for g in got)
    one, two = seen.values()
    assert len(seen) == 2 and not one & two
    ctx.close()
