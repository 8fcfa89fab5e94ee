"""Which kernels an attention call over a paged cache runs: every branch of the choice, each against the 64-bit oracle.

`branch` repeats the library's rule (its constants and both sides' measurements stand beside the kernels), so that a test that means a branch notices when its
sizes no longer reach it."""
import numpy as np
import pytest
import torch

from paper_2601_12904_amd import binding as B
from tests.test_gpu_paged import U32, UBF, check_attn, i32, make_batch, make_ctx, run_attn

LAYER = (32, 8, 128, "bf16")
NEAR, FAR, SHORT, KEY, NEAR_BYTES = 100e6, 35e6, 24e6, 29e3, 8 << 20


def branch(lens, n_tokens, max_new, positions, captured=False, layer=LAYER, n_cu=256):
    """(who decides, what runs): "stream" (everything), "tiled" (everything), "together" (the same, requests with few columns among them), "split" (requests with few columns apart)."""
    Hq, Hkv, d, _ = layer
    G = Hq // Hkv
    few = max(64, G)
    B_, rows = len(lens), min(n_tokens, len(lens) * max_new)
    if max_new * G <= few or rows * Hq * positions <= FAR:
        return "host", "stream"
    together = (B_ - 1) * Hkv <= n_cu // 4
    has_few = any(0 < n * G <= few for _, n in lens)
    tiled = "together" if together and has_few else "tiled" if together or not has_few else "split"
    least = 0.0 if captured or max_new > positions else (rows * rows / B_ - B_ * (few / G) ** 2) * Hq
    if least > min(NEAR, SHORT + KEY * B_ * positions):
        return "host", tiled
    many = [(min(n, max_new) * G, min(c + n, positions)) for c, n in lens if min(n, max_new) * G > few]
    pairs, keys = sum(c * k for c, k in many) * Hkv, sum(k for _, k in many)
    return "device", tiled if pairs > (min(NEAR, SHORT + KEY * keys) if keys * 4 * d <= NEAR_BYTES else FAR) else "stream"


CASES = {
    "short": ([(700, 100), (300, 1)], 0, ("host", "stream")),
    "middle": ([(700, 400), (300, 1)], 600, ("device", "stream")),
    "long_chunk": ([(6000, 900)], 0, ("device", "tiled")),
    "chunk_with_single_rows": ([(6000, 900)] + [(40 * i, 1) for i in range(8)], 0, ("device", "together")),
    "prompt_beside_many_single_rows": ([(500 + i, 1) for i in range(20)] + [(0, 8000)], 0, ("device", "split")),
    "chunks_beside_many_few_rows": ([(90 * i, 1 + i % 16) for i in range(12)] + [(4000, 600), (7, 0), (3000, 1200)], 100, ("device", "split")),
    "prompt": ([(0, 2300)], 0, ("host", "tiled")),
    "prompt_with_single_rows": ([(0, 6000), (300, 1), (0, 1), (44, 16)], 0, ("host", "together")),
    "long_prompt_beside_many_single_rows": ([(500 + i, 1) for i in range(20)] + [(0, 16000)], 0, ("host", "split")),
}


@pytest.mark.parametrize("case", list(CASES))
def test_the_rule(case):
    lens, wider, want = CASES[case]
    T = sum(n for _, n in lens)
    positions = (max(-(-(c + n) // 16) for c, n in lens) + 1 + wider) * 16
    assert branch(lens, T, max(n for _, n in lens), positions) == want


@pytest.mark.gpu
@pytest.mark.parametrize("case", list(CASES))
def test_every_branch(case):
    """Rows of both kinds of request (first and last ones, around the tiles' borders, where items are cut) against the oracle."""
    lens, wider, _ = CASES[case]
    assert torch.cuda.get_device_properties(0).multi_processor_count == 256
    bt = make_batch(LAYER, lens, 16, seed=len(lens), extra_blocks=1 + wider, pad=3)
    ctx = make_ctx(LAYER)
    out, lse = run_attn(ctx, bt)
    rng = np.random.default_rng(1)
    rows = set()
    for b, (c, n) in enumerate(lens):
        lo = int(bt["offs"][b])
        if n > 16:
            rows |= {lo + t for t in (0, 1, 63, 64, n // 2, n - 65, n - 1)} | {lo + int(t) for t in rng.integers(0, n, 5)}
        elif n:
            rows |= {lo, lo + n - 1}
    check_attn(bt, out, lse, rows)
    assert bool((out[-3:] == 7).all()) and bool((lse[-3:] == 7).all())
    assert bool(torch.isfinite(out.float()).all()) and bool(torch.isfinite(lse).all())
    again, _ = run_attn(ctx, bt, lse=False)
    assert torch.equal(out, again)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("n_requests,T,live", [(1, 2304, [(16000, 1)]), (8, 8192, [(3000 + 500 * i, 1) for i in range(8)])])
def test_a_captured_step_of_fixed_size_with_few_live_rows(n_requests, T, live):
    """A step captured in buffers for a long chunk, replayed for single rows: the streaming kernel has them (the same bits as when it is asked for), and
    replayed for a long chunk of its first request the same as eagerly."""
    chunk = [(300, T - 200)] + [(20, 1)] * (n_requests - 1)
    bt = make_batch(LAYER, [(16000, 1)] + [(c, max(n, m)) for (c, n), (_, m) in zip(live[1:], chunk[1:])], 16, seed=2)
    rng = np.random.default_rng(4)
    q = torch.from_numpy(rng.standard_normal((T, 32, 128)).astype(np.float32)).bfloat16().cuda()
    dev = dict(q=q, kp=torch.nan_to_num(torch.from_numpy(bt["kp"])).bfloat16().cuda(), vp=torch.nan_to_num(torch.from_numpy(bt["vp"])).bfloat16().cuda(), table=i32(bt["table"]))
    bt["q"] = q.float().cpu().numpy()

    def lengths(lens):
        return i32(np.concatenate([[0], np.cumsum([n for _, n in lens])])), i32([c for c, _ in lens])

    def call(ctx, offs, cached, out, lse):
        ctx.fr_paged_attn(dev["q"], offs, cached, n_requests, T, T, dev["kp"], dev["vp"], len(bt["kp"]), 16, dev["table"], bt["table"].shape[1], out, lse)

    fresh = lambda: (torch.full_like(q, 7), torch.full((T, 32), 7.0, device="cuda"))
    ctx, stream = make_ctx(LAYER), make_ctx(LAYER, kernel="stream")
    offs, cached = lengths(live)
    out, lse = fresh()
    call(ctx, offs, cached, out, lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(ctx, offs, cached, out, lse)
    for lens in (live, chunk, live, live):
        o, c = lengths(lens)
        offs.copy_(o); cached.copy_(c)
        for x in (out, lse):
            x.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        n = sum(m for _, m in lens)
        want, want_lse = fresh()
        if lens is live:
            call(stream, o, c, want, want_lse)
            assert torch.equal(out, want) and torch.equal(lse, want_lse)
        else:
            part = dict(bt, offs=o.cpu().numpy(), cached=c.cpu().numpy())
            check_attn(part, out, lse, {0, 1, 255, 256, T - 201, n - 1})
        assert bool((out[n:] == 7).all()) and bool((lse[n:] == 7).all())
    ctx.close()
    stream.close()
