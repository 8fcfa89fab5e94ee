"""Attention of a step with trees at the ends of its range: logits beyond what an exponential can take, values as large as their sums allow, masks of all ones.

The masks of paths are a chunk's causal ones, so a batch of paths is held to the bounds of fr_paged_attn's own extremes (there: what fp32 makes of such logits)."""
import numpy as np
import pytest
import torch

import tests.test_gpu_paged_extremes as ext
import tests.test_gpu_tree as trees
from oracle import fusionrag_oracle as orc
from tests.test_gpu_paged import LAYERS, U32, UBF, down, make_batch, make_ctx, stored
from tests.test_gpu_tree import FEW, check_tree, make_tree, run_tree, some

pytestmark = pytest.mark.gpu


def paths(bt, lens):
    """The masks that make a chunk of each request's rows."""
    words = -(-bt["max_new"] // 32)
    parents = np.concatenate([np.arange(n) - 1 for _, n in lens])
    bt["sees"] = orc.tree_tables(parents, bt["offs"], bt["cached"], len(bt["q"]), bt["max_new"], words)[1]
    return bt


@pytest.mark.parametrize("kernel,layer", FEW)
@pytest.mark.parametrize("where,sign", [("all", 0), ("all", 1), ("all", -1), ("late", 0), ("late", -1), ("early", -1)])
@pytest.mark.parametrize("exponent", [30, 60, 100, 112])
def test_logits_far_apart(kernel, layer, exponent, where, sign):
    """Logits of 1e9 to 1e35."""
    bt = paths(ext.batch(LAYERS[layer], exponent, sign, where), ext.LENS)
    ctx = make_ctx(LAYERS[layer], kernel=kernel)
    out, lse = run_tree(ctx, bt)
    T = len(bt["q"])
    rows = {0, 1, 2, 30, 77, 80, 81, 82, 85, 100, 113, 114, 115, 116, 117, 120, 150, T - 2, T - 1}
    assert bool(torch.isfinite(out.float()).all()) and bool(torch.isfinite(lse).all())
    decided, total = ext.check(bt, out, lse, rows)
    assert decided > 0.9 * total, (decided, total)
    ctx.close()


@pytest.mark.parametrize("kernel,layer", [x for x in FEW if x[1] != "g7"])
@pytest.mark.parametrize("size", [2.0 ** 44, 2.0 ** 57])
def test_exact_logits_of_any_size(kernel, layer, size):
    """Up to 9 x 2^114 / sqrt(d) = 2e34, each of them exact, and shared by several keys."""
    trees.test_logits_of_any_size(kernel, layer, size)


@pytest.mark.parametrize("kernel,layer", FEW)
def test_logits_of_minus_infinity(kernel, layer):
    """Rows all of whose logits are -infinity, and rows with one finite logit among such."""
    dt = LAYERS[layer][3]
    lens = [(300, 70), (40, 1), (0, 20), (900, 1)]
    bt = paths(make_batch(LAYERS[layer], lens, 16, seed=8), lens)
    bt["q"] = stored(np.abs(bt["q"]) + 0.5, dt)
    for b, (c, n) in enumerate(lens):
        for j in range(c + n):
            if (b, j) not in ((0, 310), (2, 5), (3, 33)):
                bt["kp"][bt["table"][b, j // 16], j % 16] = -np.inf
    ctx = make_ctx(LAYERS[layer], kernel=kernel)
    out, lse = (down(x) for x in run_tree(ctx, bt))
    blind = [*range(0, 10), 70, *range(71, 76)]
    assert np.all(out[blind] == 0) and np.all(np.isneginf(lse[blind]))
    for b, (rows, j) in {0: (range(10, 70), 310), 2: (range(76, 91), 5), 3: (range(91, 92), 33)}.items():
        v = bt["vp"][bt["table"][b, j // 16], j % 16].repeat(LAYERS[layer][0] // LAYERS[layer][1], axis=0)
        assert np.all(np.abs(out[list(rows)] - v) <= (UBF if dt == "bf16" else 4 * U32) * np.abs(v)) and np.all(np.isfinite(lse[list(rows)]))
    ctx.close()


@pytest.mark.parametrize("kernel,layer", FEW)
@pytest.mark.parametrize("words", [None, 8])
def test_masks_of_all_ones(kernel, layer, words):
    """Every row sees all rows of its request; the bits behind those are set too, and mean nothing."""
    bt = make_tree(LAYERS[layer], [(40, 64), (0, 50), (333, 37), (31, 96), (1, 20), (64, 1)], 16, seed=4, words=words)
    bt["sees"][:] = True
    ctx = make_ctx(LAYERS[layer], kernel=kernel)
    out, lse = run_tree(ctx, bt)
    check_tree(bt, out, lse, some(bt, 5))
    ctx.close()


@pytest.mark.parametrize("kernel,layer", FEW)
@pytest.mark.parametrize("growing", [False, True])
def test_values_as_large_as_their_sums_allow(kernel, layer, growing):
    """Values of 2^119 / (keys of the request) in magnitude: with weights of up to 2^8 no sum of them passes fp32.  Growing logits raise the weights before the references follow."""
    lens = [(400, 40), (70, 9)]                                     # at most 440 keys: 2^110
    bt = make_tree(LAYERS[layer], lens, 16, seed=8, q_scale=2.0)
    rng = np.random.default_rng(5)
    bt["vp"] = (np.sign(bt["vp"]) * np.where(rng.random(bt["vp"].shape) < 0.9, np.float32(2.0 ** 110), np.float32(1))).astype(np.float32)   # (NaN where no position is)
    if growing:
        for b, (c, n) in enumerate(lens):
            for j in range(c + n):
                bt["kp"][bt["table"][b, j // 16], j % 16] *= np.float32(1 + j // 32)
        bt["kp"] = stored(np.nan_to_num(bt["kp"], nan=0.0), LAYERS[layer][3])
    ctx = make_ctx(LAYERS[layer], kernel=kernel)
    out, lse = run_tree(ctx, bt)
    check_tree(bt, out, lse, some(bt, 7))
    ctx.close()
