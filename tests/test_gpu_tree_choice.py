"""Steps with trees whose table has far more room than their requests hold, and on both sides of where the kernel changes: right by whichever they go to, eager and captured."""
import numpy as np
import pytest
import torch

from oracle import fusionrag_oracle as orc
from tests.test_gpu_paged import i32, make_ctx, up
from tests.test_gpu_tree import check_tree, make_tree, run_tree

pytestmark = pytest.mark.gpu


def widened(bt, width):
    table = np.full((len(bt["table"]), width), -1, dtype=np.int64)
    table[:, : bt["table"].shape[1]] = bt["table"]
    return dict(bt, table=table)


def on_device(bt):
    return dict(q=up(bt["q"], "bf16"), kp=up(bt["kp"], "bf16"), vp=up(bt["vp"], "bf16"), offs=i32(bt["offs"]), cached=i32(bt["cached"]), table=i32(bt["table"]),
                mask=torch.from_numpy(orc.pack_bits(bt["sees"])).cuda())


# heads; rows behind positions; blocks of the table in pages of 16 (0: what the requests hold and one more)
SIDES = [
    ((32, 8, 128, "bf16"), [(100, 24)] * 16, 0),         # 96 columns; 384 rows x 32 heads x 144 positions = 1.8 M
    ((32, 8, 128, "bf16"), [(100, 24)] * 16, 8192),      # the same requests, a table with room for 131072 positions
    ((32, 8, 128, "bf16"), [(100, 8)] * 16, 8192),       # 32 columns
    ((32, 8, 128, "bf16"), [(1000, 24)] * 3, 0),         # 2.4 M
    ((32, 8, 128, "bf16"), [(1000, 24)] * 4, 0),         # 3.2 M
    ((32, 8, 128, "bf16"), [(1000, 100)] + [(300 + b, 1) for b in range(30)], 8192),   # one wide tree, single rows beside it
    ((16, 8, 64, "bf16"), [(100, 32)] * 4, 8192),        # 64 columns
    ((16, 8, 64, "bf16"), [(100, 33)] * 4, 8192),
    ((16, 8, 64, "bf16"), [(100, 33)] * 4, 0),           # 132 rows x 16 heads x 160 positions
]


@pytest.mark.parametrize("layer,lens,width", SIDES)
def test_right_by_whichever_kernel(layer, lens, width):
    bt = make_tree(layer, lens, 16, seed=2)
    bt = widened(bt, width or bt["table"].shape[1])
    bt["kp"], bt["vp"] = np.nan_to_num(bt["kp"]), np.nan_to_num(bt["vp"])
    rows = set(range(0, len(bt["q"]), 29)) | {0, len(bt["q"]) - 1}
    for kernel in ("auto", "stream", "tiled"):
        ctx = make_ctx(layer, kernel=kernel)
        out, lse = run_tree(ctx, bt)
        check_tree(bt, out, lse, rows)
        ctx.close()


@pytest.mark.parametrize("width", [10, 8192])
def test_a_captured_call_serves_other_lengths(width):
    """Replayed for other lengths it gives the bits that an eager call gives for them."""
    layer = (32, 8, 128, "bf16")
    steps = [widened(make_tree(layer, lens, 16, seed=k), width) for k, lens in enumerate(([(100, 24)] * 16, [(3, 24)] * 16, [(117 - b, 24) for b in range(16)]))]
    ctx = make_ctx(layer)
    most = max(len(bt["kp"]) for bt in steps)
    for bt in steps:   # one cache for all of them
        for name in ("kp", "vp"):
            bt[name] = np.concatenate([np.nan_to_num(bt[name]), np.zeros((most - len(bt[name]), *bt[name].shape[1:]), dtype=np.float32)])
    held = on_device(steps[0])
    run_tree(ctx, steps[0], dev=held)                              # (once outside)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = run_tree(ctx, steps[0], dev=held)
    for bt in (steps[1], steps[0], steps[2], steps[1]):
        dev = on_device(bt)
        for name in held:
            held[name].copy_(dev[name])
        graph.replay()
        torch.cuda.synchronize()
        check_tree(bt, out, lse, {0, 23, 24, 200, 383})
        want = run_tree(ctx, bt, dev=dev)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    ctx.close()
