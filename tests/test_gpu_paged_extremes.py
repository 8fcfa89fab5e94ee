"""Paged attention of logits so large that the steps of fp32 between them are larger than what an exponential can take, against the 64-bit oracle's logits.

At such sizes a softmax is the value of the key with the largest logit, and that logit is the normaliser.  fp32 forms a logit off by at most
e = 2 (d + 6) 2^-24 spread, spread = sum of |q_c k_c| / sqrt(d) (the sum's d roundings and the scale's, each twice over): where no other key comes within 2 e of the largest, the
row has to be that key's value (to half a step of the output) and the normaliser the largest logit to e and its own rounding.  Rows whose largest logits are of ordinary size are
held to the bounds of ordinary attention."""
import numpy as np
import pytest

from tests.test_gpu_paged import FEW, LAYERS, U32, UBF, down, make_batch, make_ctx, run_attn, stored

import torch

pytestmark = pytest.mark.gpu

LENS = [(900, 1), (300, 80), (0, 33), (31, 2), (3000, 70)]


def batch(layer, exponent, sign, where):
    """Logits scaled by 2^exponent: all of a request's keys, those behind its first 40, or its first 20.  sign: of all logits, or 0: of both."""
    bt = make_batch(layer, LENS, 16, seed=abs(exponent) + 3)
    half = exponent // 2
    if sign:
        bt["q"], bt["kp"] = np.abs(bt["q"]), sign * np.abs(bt["kp"])
    # (powers of two: everything stays exact in either type)
    bt["q"] = stored(bt["q"] * 2.0 ** half, layer[3])
    for b, (c, n) in enumerate(LENS):
        lo, hi = {"all": (0, c + n), "late": (40, c + n), "early": (0, 20)}[where]
        for j in range(c + n):
            bt["kp"][bt["table"][b, j // 16], j % 16] *= np.float32(2.0 ** ((exponent - half) if lo <= j < hi else -half))
    return bt


def check(bt, out, lse, rows):
    Hq, Hkv, d, dt = bt["layer"]
    out, lse = down(out), down(lse)
    decided = total = 0
    for b, (c, n) in enumerate(LENS):
        for t in (t for t in rows if bt["offs"][b] <= t < bt["offs"][b + 1]):
            j = np.arange(c + t - bt["offs"][b] + 1)
            k, v = (x[bt["table"][b, j // 16], j % 16].astype(np.float64) for x in (bt["kp"], bt["vp"]))
            for h in range(Hq):
                x, kh = bt["q"][t, h].astype(np.float64), k[:, h // (Hq // Hkv)]
                s, spread = kh @ x / np.sqrt(d), np.abs(kh) @ np.abs(x) / np.sqrt(d)
                e = 2 * (d + 6) * U32 * spread
                best = int(np.argmax(s))
                others = np.delete(s + e, best)
                total += 1
                assert np.all(np.isfinite(out[t, h])), f"row {t}, head {h}"
                assert abs(lse[t, h] - s[best]) <= e.max() + 4 * U32 * abs(s[best]) + np.log(len(j)), f"row {t}, head {h}: normaliser {lse[t, h]}, largest logit {s[best]}"
                # 120: what the others leave is below 2^-24 of a value by far, whatever the sum of them
                if len(others) and others.max() > s[best] - e[best] - 120:
                    near = s >= s[best] - 200
                    if spread[near].max() < 1000:      # keys of ordinary size beside those that nothing is left of: as any attention
                        decided += 1
                        w = np.exp(s[near] - s[best])
                        vh = v[near, h // (Hq // Hkv)]
                        want, mass = w / w.sum() @ vh, w / w.sum() @ np.abs(vh)
                        weight = 2 * (d + 6) * U32 * (spread[near].max() + 1) + (len(j) + 64) * U32
                        assert np.all(np.abs(out[t, h] - want) <= weight * 2 * mass + U32 * np.abs(want) + (UBF * 1.01 * (mass + np.abs(want)) if dt == "bf16" else 0)), f"row {t}, head {h}"
                        assert abs(lse[t, h] - s[best] - np.log(w.sum())) <= weight + 4 * U32 * abs(s[best]), f"row {t}, head {h}: normaliser"
                    continue
                decided += 1
                want = v[best, h // (Hq // Hkv)]
                assert np.all(np.abs(out[t, h] - want) <= (UBF if dt == "bf16" else 4 * U32) * np.abs(want)), f"row {t}, head {h}"
    return decided, total


@pytest.mark.parametrize("kernel,layer", FEW)
@pytest.mark.parametrize("where,sign", [("all", 0), ("all", 1), ("all", -1), ("late", 0), ("late", 1), ("late", -1), ("early", 1), ("early", -1)])
@pytest.mark.parametrize("exponent", [30, 60])
def test_logits_far_apart(kernel, layer, exponent, where, sign):
    bt = batch(LAYERS[layer], exponent, sign, where)
    ctx = make_ctx(LAYERS[layer], kernel=kernel)
    out, lse = run_attn(ctx, bt)
    T = len(bt["q"])
    rows = {0, 1, 2, 30, 77, 80, 81, 82, 85, 100, 113, 114, 115, 116, 117, 120, 150, T - 2, T - 1}
    assert bool(torch.isfinite(out[:T].float()).all()) and bool(torch.isfinite(lse).all())
    decided, total = check(bt, out, lse, rows)
    assert decided > 0.9 * total, (decided, total)
    ctx.close()


@pytest.mark.parametrize("kernel,layer", FEW)
@pytest.mark.parametrize("where,sign", [("all", 0), ("all", 1), ("all", -1), ("late", 0), ("late", -1), ("early", -1)])
@pytest.mark.parametrize("exponent", [100, 112])
def test_logits_beyond_1e30(kernel, layer, exponent, where, sign):
    """A finite logit is seen, however low it is."""
    test_logits_far_apart(kernel, layer, exponent, where, sign)


@pytest.mark.parametrize("kernel,layer", FEW)
def test_logits_of_minus_infinity(kernel, layer):
    """Rows all of whose logits are -infinity, and rows with one finite logit among such."""
    dt = LAYERS[layer][3]
    bt = make_batch(LAYERS[layer], [(300, 70), (40, 1), (0, 20), (900, 1)], 16, seed=8)
    bt["q"] = stored(np.abs(bt["q"]) + 0.5, dt)
    for b, (c, n) in enumerate([(300, 70), (40, 1), (0, 20), (900, 1)]):
        for j in range(c + n):
            if (b, j) not in ((0, 310), (2, 5), (3, 33)):
                bt["kp"][bt["table"][b, j // 16], j % 16] = -np.inf
    ctx = make_ctx(LAYERS[layer], kernel=kernel)
    out, lse = (down(x) for x in run_attn(ctx, bt))
    blind = [*range(0, 10), 70, *range(71, 76)]
    assert np.all(out[blind] == 0) and np.all(np.isneginf(lse[blind]))
    seen = {0: (range(10, 70), 310), 2: (range(76, 91), 5), 3: (range(91, 92), 33)}
    for b, (rows, j) in seen.items():
        v = bt["vp"][bt["table"][b, j // 16], j % 16].repeat(LAYERS[layer][0] // LAYERS[layer][1], axis=0)
        assert np.all(np.abs(out[list(rows)] - v) <= (UBF if dt == "bf16" else 4 * U32) * np.abs(v)) and np.all(np.isfinite(lse[list(rows)]))
    ctx.close()
