"""What paged attention needs of a context's workspace, and what it shares there."""
import numpy as np
import pytest
import torch

from paper_2601_12904_amd import binding as B
from tests.test_gpu_paged import check_attn, make_batch, make_ctx, run_attn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 128), (1, 1, 64), (4, 4, 64), (32, 8, 128)])
def test_bf16_contexts_hold_no_memory_for_it(Hq, Hkv, d):
    """The partial results lie over those of decoding (4096 pieces) and of the projections (256 parts of a tile of 256 x 256), 68 MB of them at the most."""
    ctx = make_ctx((Hq, Hkv, d, "bf16"))
    others = 16 << 20                            # selection, maps, normalisers, pieces of the sparse attention of a context of 64 tokens
    assert ctx.workspace_bytes() <= 4096 * Hq * (d + 2) * 4 + 256 * 256 * 256 * 4 + others
    ctx.close()


def test_calls_that_share_the_workspace_in_turn():
    """Cut items of both attention kernels, projections that are split along K, a decoding step: one after the other, each as by itself."""
    Hq, Hkv, d = 8, 2, 128
    ctx = make_ctx((Hq, Hkv, d, "bf16"), tokens=512)
    tiled = make_batch((Hq, Hkv, d, "bf16"), [(6000, 200)], 16, seed=1)
    few = make_batch((Hq, Hkv, d, "bf16"), [(5000, 1), (300, 2)], 16, seed=2)
    gen = torch.Generator(device="cuda").manual_seed(3)
    f = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()
    a, w, out = f(300, 6144), f(384, 6144), torch.empty((300, 384), dtype=torch.bfloat16, device="cuda")
    k, v, q = f(4000, Hkv, d), f(4000, Hkv, d), f(2, Hq, d)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    got = torch.empty_like(q)

    def paged(bt, kernel):
        ctx.fr_set_option(B.FR_OPT_PAGED_KERNEL, kernel)
        return run_attn(ctx, bt)

    def linear():
        ctx.fr_linear(a, w, 300, 384, 6144, None, out)
        return out.clone(), out[:0]

    pages = f(2, 8, Hkv, d)
    segments = [i32(x) for x in ([0, 1, 2], [0, 500], [3900, 3500], [0, 0])]

    def decode():
        ctx.fr_decode_attn(q, 2, k, v, 4000, *segments, 2, None, 0, pages, pages, 8, i32([8, 5]), got)
        return got.clone(), got[:0]

    calls = [lambda: paged(tiled, B.FR_PAGED_KERNEL_TILED), lambda: paged(few, B.FR_PAGED_KERNEL_STREAM), linear, decode]
    want = [c() for c in calls]
    check_attn(tiled, *want[0], {0, 1, 63, 64, 130, 199})
    check_attn(few, *want[1])
    for i in np.random.default_rng(4).integers(0, len(calls), 24):
        o, l = calls[i]()
        assert torch.equal(o, want[i][0]) and torch.equal(l, want[i][1]), i
    ctx.close()
