"""The largest sizes that the paged step's calls take, and queries that are not finite beside ones that are."""
import numpy as np
import pytest
import torch

from paper_2601_12904_amd import binding as B
from tests.test_gpu_paged import FEW, LAYERS, check_attn, down, i32, make_batch, make_ctx, run_attn, up

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kernel", ["auto", "stream", "tiled"])
def test_the_most_requests(kernel):
    """FR_PAGED_MAX_REQUESTS of them, many without rows, one with a chunk near the end."""
    rng = np.random.default_rng(8)
    lens = [(int(rng.integers(0, 30)), int(rng.integers(0, 3))) for _ in range(B.FR_PAGED_MAX_REQUESTS)]
    lens[4000] = (200, 300)
    bt = make_batch((4, 2, 64, "bf16"), lens, 8, seed=4)
    ctx = make_ctx(bt["layer"], kernel=kernel)
    out, lse = run_attn(ctx, bt)
    first = int(bt["offs"][4000])
    check_attn(bt, out, lse, set(range(0, len(bt["q"]), 29)) | {0, first - 1, first, first + 127, first + 128, first + 299, first + 300, len(bt["q"]) - 1})
    ctx.close()


@pytest.mark.parametrize("kernel", ["stream", "tiled"])
def test_elements_beyond_32_bits(kernel):
    """Pages at the end of a cache of more than 2^32 elements."""
    layer = (8, 8, 128, "bf16")
    n_pages, page = 270000, 16                                        # 8.8 GB each
    assert n_pages * page * 8 * 128 > 2 ** 32
    kp, vp = (torch.empty((n_pages, page, 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bt = make_batch(layer, [(300, 1), (20, 100)], page, seed=1)
    used = bt["kp"].shape[0]
    kp[-used:], vp[-used:] = up(bt["kp"], "bf16"), up(bt["vp"], "bf16")
    table = np.where(bt["table"] >= 0, bt["table"] + n_pages - used, -1)
    ctx = make_ctx(layer, kernel=kernel)
    q, out = up(bt["q"], "bf16"), torch.zeros(bt["q"].shape, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(bt["q"].shape[:2], device="cuda")
    ctx.fr_paged_attn(q, i32(bt["offs"]), i32(bt["cached"]), 2, 101, 100, kp, vp, n_pages, page, i32(table), table.shape[1], out, lse)
    check_attn(bt, out, lse, {0, 1, 50, 100})
    rows = up(np.random.default_rng(0).standard_normal((2, 8, 128)), "bf16")
    ctx.fr_paged_append(None, rows, rows, None, i32([n_pages * page - 1, n_pages * page]), 2, kp, vp, n_pages, page)      # the last row, and one that is none
    assert torch.equal(kp[-1, -1], rows[0]) and torch.equal(vp[-1, -1], rows[0])
    ctx.close()


@pytest.mark.parametrize("kernel,layer", FEW)
def test_queries_that_are_not_finite(kernel, layer):
    """They are their own row's and head's alone."""
    bt = make_batch(LAYERS[layer], [(100, 40), (700, 1), (200, 300)], 16, seed=12)
    Hq, _, d, _ = LAYERS[layer]
    bad = {(3, 0): np.nan, (17, 1): np.inf, (39, Hq - 1): -np.inf, (40, 0): np.nan, (41, 0): np.inf, (200, 1): np.nan, (340, Hq - 1): np.nan}
    clean = {t for t in (0, 1, 2, 4, 16, 18, 38, 42, 100, 199, 201, 250, 339)}
    for (t, h), what in bad.items():
        bt["q"][t, h, d // 3] = what
    ctx = make_ctx(LAYERS[layer], kernel=kernel)
    out, lse = run_attn(ctx, bt)
    check_attn(bt, out, lse, clean)
    got = down(out)
    for t, h in bad:
        others = np.arange(Hq) != h
        assert np.isnan(got[t, h]).any() and np.isfinite(got[t, others]).all(), (t, h)
    ctx.close()
