"""GPU parity of the paged step (tables, append, attention) against the 64-bit oracle, through the C ABI.

Bounds.  A value rounded to bf16 is off by at most 2^-8 of it, one rounded to fp32 by 2^-24.  Attention keeps its weights in bf16 on the
way into the second product and rounds its output once: 2^-8 (mass + |out|), mass = sum of weight x |value|.  Below that lies fp32: a logit
sums d products, off by (d + 2) 2^-24 spread, spread = sum of |q_c k_c| / sqrt(d); that and the scale's and exponent's roundings move a
weight by exp of it, the sums of up to n weights add n 2^-24."""
import numpy as np
import pytest
import torch

from oracle import fusionrag_oracle as orc
from paper_2601_12904_amd import binding as B
from paper_2601_12904_amd import stack as S
from paper_2601_12904_amd import synth

pytestmark = pytest.mark.gpu

U32, UBF = 2.0 ** -24, 2.0 ** -8
TD = {"f32": torch.float32, "bf16": torch.bfloat16}
# Hq, Hkv, d, dtype
LAYERS = {
    "g4": (8, 2, 128, "bf16"), "g7": (14, 2, 128, "bf16"), "g1": (3, 3, 128, "bf16"), "g8_d64": (16, 2, 64, "bf16"), "g2_d64": (4, 2, 64, "bf16"),
    "g16": (16, 1, 128, "bf16"), "g33": (33, 1, 64, "bf16"), "f32_d64": (4, 4, 64, "f32"), "f32_g5_d128": (10, 2, 128, "f32"), "g80_d64": (80, 1, 64, "bf16"),
}


def make_ctx(layer, half=False, base=5e5, tokens=64, kernel="auto"):
    Hq, Hkv, d, dt = layer
    c = B.Context(Hq, Hkv, d, B.FR_BF16 if dt == "bf16" else B.FR_F32, base, max_tokens=tokens, max_chunks=1, max_question_tokens=1,
                  rope_layout=B.FR_ROPE_HALF if half else B.FR_ROPE_INTERLEAVED)
    c.fr_set_option(B.FR_OPT_PAGED_KERNEL, {"auto": B.FR_PAGED_KERNEL_AUTO, "stream": B.FR_PAGED_KERNEL_STREAM, "tiled": B.FR_PAGED_KERNEL_TILED}[kernel])
    return c


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def stored(x, dt):
    return synth.round_to_storage(np.asarray(x, dtype=np.float32), dt)


def up(x, dt):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(TD[dt]).cuda()


def down(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


# ---- tables --------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("seed,n,page,width,spare_rows,short", [
    (0, 1, 16, 40, 0, 0), (1, 3, 1, 700, 5, 0), (2, 64, 16, 30, 0, 0), (3, 64, 7, 20, -40, 0), (4, 300, 32, 9, 13, 4), (5, 1025, 8, 5, 3, 20),
    (6, B.FR_PAGED_MAX_REQUESTS, 24, 3, 700, 0), (7, 5, 128, 1, 0, 0), (8, 2, 3, 0, 0, 0), (9, 1024, 16, 40, -5000, 3)])
def test_tables(seed, n, page, width, spare_rows, short):
    rng = np.random.default_rng(seed)
    cached = rng.integers(-2, 300, n)
    new = np.where(rng.random(n) < 0.3, rng.integers(0, 200, n), rng.integers(-1, 3, n))
    T = max(int(np.maximum(new, 0).sum()) + spare_rows, 1)
    need = sum(-(-(max(c, 0) + max(m, 0)) // page) for c, m in zip(cached, new))
    ids = rng.permutation(need + 50)
    table = rng.choice(ids, (n, width)) if width else np.zeros((n, 0), dtype=np.int64)
    start = int(rng.integers(0, 4))
    free = ids[: max(0, need // 2 if short else len(ids))]
    want = orc.page_tables(cached, new, page, free, start, table, T)
    ctx = make_ctx(LAYERS["g4"])
    tab, off, pos, slot, needed = i32(table), i32(np.full(n + 1, -9)), i32(np.full(T + 3, -9)), i32(np.full(T + 3, -9)), i32([-9])
    args = (i32(cached), i32(new), n, page, i32(free), len(free), i32([start]), tab, width, T, off, pos, slot, needed)
    for _ in range(2):                                   # the second call finds its own table: the same again
        ctx.fr_page_tables(*args)
        for name, got, exp in (("table", tab, want[0]), ("offsets", off, want[1]), ("positions", pos[:T], want[2]), ("slots", slot[:T], want[3]),
                               ("needed", needed, [want[4]])):
            assert np.array_equal(got.cpu().numpy(), np.asarray(exp)), name
        assert bool((pos[T:] == -9).all()) and bool((slot[T:] == -9).all())
    ctx.close()


def test_tables_without_requests_or_optional_arrays():
    ctx = make_ctx(LAYERS["g4"])
    off, pos, slot = i32([5]), i32([5, 5]), i32([5, 5])
    ctx.fr_page_tables(None, None, 0, 16, None, 0, None, None, 4, 2, off, pos, slot)
    assert off.tolist() == [0] and pos.tolist() == [0, 0] and slot.tolist() == [-1, -1]
    tab, off = i32([[-1, -1]]), i32([0, 0])
    ctx.fr_page_tables(i32([0]), i32([2]), 1, 16, i32([3]), 1, None, tab, 2, 2, off, pos, slot)
    assert tab.tolist() == [[3, -1]] and slot.tolist() == [48, 49] and pos.tolist() == [0, 1]
    big = 2 ** 31 - 1                                    # lengths whose sums pass 32 bits, a position at the end of the range
    ctx.fr_page_tables(i32([big]), i32([big]), 1, 16, i32([3]), 1, None, tab, 2, 1, off, pos[:1], slot[:1])
    assert off.tolist() == [0, 1] and pos[0].item() == big and slot[0].item() == -1 and tab.tolist() == [[3, -1]]
    ctx.close()


# ---- append --------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("layer", ["g4", "g7", "g2_d64", "f32_d64", "f32_g5_d128", "g80_d64"])
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("T,mode", [(1, "all"), (5, "in_place"), (70, "keys"), (700, "copy"), (601, "all")])
def test_append(layer, half, T, mode):
    Hq, Hkv, d, dt = LAYERS[layer]
    rng = np.random.default_rng(T)
    n_pages, page = T // 5 + 3, 7
    rows = n_pages * page
    ctx = make_ctx(LAYERS[layer], half)
    q, k, v, kp, vp = (stored(rng.standard_normal(s), dt) for s in ((T, Hq, d), (T, Hkv, d), (T, Hkv, d), (n_pages, page, Hkv, d), (n_pages, page, Hkv, d)))
    slots = rng.permutation(rows)[:T]
    slots[rng.random(T) < 0.2] = -1
    if T > 4:
        slots[2:5] = (rows, 2 ** 31 - 1, -2 ** 31)
    pos = rng.integers(-5, 200000, T)
    dk, dv, dq, dkn, dvn = up(kp, dt), up(vp, dt), up(q, dt), up(k, dt), up(v, dt)
    q_out = None if mode in ("keys", "copy") else dq if mode == "in_place" else torch.full_like(dq, 7)
    ctx.fr_paged_append(None if q_out is None else dq, dkn, dvn, None if mode == "copy" else i32(pos), i32(slots), T, dk, dv, n_pages, page, q_out)
    wq, wk, wv = orc.paged_append(q, k, v, None if mode == "copy" else pos, slots, kp, vp, 5e5, "half" if half else "interleaved")
    gk, gv = down(dk), down(dv)
    hit = np.zeros(rows, dtype=bool)
    hit[[s for s in slots if 0 <= s < rows]] = True
    assert np.array_equal(gv, wv)
    assert np.array_equal(gk.reshape(rows, Hkv, d)[~hit], kp.reshape(rows, Hkv, d)[~hit])     # other rows as they were
    u = UBF if dt == "bf16" else U32

    def near(got, want, size):   # the output's rounding; cos, sin and two products and a sum in fp32 on pairs of `size`
        assert np.all(np.abs(got - want) <= u * np.abs(want) + 6 * U32 * size)
    if mode == "copy":
        assert np.array_equal(gk, wk)
    else:
        near(gk, wk, np.abs(kp).max() + np.abs(k).max())
    if q_out is not None:
        near(down(q_out), wq, 2 * np.abs(q).max())
        assert mode == "in_place" or np.array_equal(down(dq), q)
    ctx.close()


# ---- attention -----------------------------------------------------------------------------------------------------------

def make_batch(layer, lens, page, seed, q_scale=1.5, extra_blocks=1, pad=0):
    """Requests of (cached, new) positions in pages in no order; unused pages hold NaN, and so do rows behind a request's last."""
    Hq, Hkv, d, dt = layer
    rng = np.random.default_rng(seed)
    need = [-(-max(c + n, 0) // page) for c, n in lens]
    n_pages = sum(need) + 3
    ids = rng.permutation(n_pages)
    table = np.full((len(lens), max(need + [0]) + extra_blocks), -1)
    kp, vp = np.full((n_pages, page, Hkv, d), np.nan, dtype=np.float32), np.full((n_pages, page, Hkv, d), np.nan, dtype=np.float32)
    at = 0
    for b, (c, n) in enumerate(lens):
        table[b, : need[b]] = ids[at: at + need[b]]
        at += need[b]
        for x in (kp, vp):
            rows = stored(rng.standard_normal((max(c + n, 0), Hkv, d)), dt)
            full = np.full((need[b] * page, Hkv, d), np.nan, dtype=np.float32)
            full[: len(rows)] = rows
            x[table[b, : need[b]]] = full.reshape(need[b], page, Hkv, d)
    offs = np.concatenate([[0], np.cumsum([n for _, n in lens])]).astype(np.int64)
    q = stored(rng.standard_normal((int(offs[-1]) + pad, Hq, d)) * q_scale, dt)
    return dict(layer=layer, page=page, table=table, kp=kp, vp=vp, offs=offs, cached=np.array([c for c, _ in lens]), q=q,
                max_new=max([n for _, n in lens] + [1]))


def run_attn(ctx, bt, lse=True, stream=None, dev=None, **kw):
    dt = bt["layer"][3]
    dev = dev or dict(q=up(bt["q"], dt), kp=up(bt["kp"], dt), vp=up(bt["vp"], dt), offs=i32(bt["offs"]), cached=i32(bt["cached"]), table=i32(bt["table"]))
    T = bt["q"].shape[0]
    out, l = torch.full_like(dev["q"], 7), torch.full((T, bt["q"].shape[1]), 7.0, device="cuda")
    ctx.fr_paged_attn(dev["q"], dev["offs"], dev["cached"], len(bt["cached"]), T, kw.get("max_new", bt["max_new"]), dev["kp"], dev["vp"], bt["kp"].shape[0],
                      bt["page"], dev["table"], bt["table"].shape[1], out, l if lse else None, stream)
    return out, l


def check_attn(bt, out, lse, rows=None):
    d, dt = bt["layer"][2], bt["layer"][3]
    n = bt["table"].shape[1] * bt["page"]
    want = orc.paged_attn(bt["q"], bt["offs"], bt["cached"], bt["kp"], bt["vp"], bt["table"], rows)
    out, lse = down(out), down(lse)
    for t, (o, l, mass, spread) in want.items():
        weight = 2 * (d + 6) * U32 * (spread + 1) + (n + 16) * U32      # relative, of a weight and of the sum
        bound = weight[:, None] * 2 * mass + U32 * np.abs(o) + (UBF * 1.01 * (mass + np.abs(o)) if dt == "bf16" else 0)
        assert np.all(np.abs(out[t] - o) <= bound), f"row {t}: off by {np.max(np.abs(out[t] - o) - bound)} more than it may be"
        none = np.isneginf(l)
        assert np.array_equal(none, np.isneginf(lse[t])) and np.all(out[t][none] == 0)
        assert np.all(np.abs(lse[t][~none] - l[~none]) <= weight[~none] + 4 * U32 * np.abs(l[~none])), f"row {t}: lse"


FORMS = {
    "decode": [(0, 1), (1, 1), (30, 1), (31, 1), (32, 1), (63, 1), (64, 1), (127, 1), (128, 1), (700, 1), (1999, 1)],
    "one_long": [(4095, 1)],
    "verify": [(5, 3), (900, 8), (61, 5), (64, 2), (250, 7)],
    "chunk": [(777, 65), (0, 33)],
    "prompt": [(0, 300)],
    "mixed": [(90, 1), (200, 130), (0, 1), (3, 0), (1000, 2), (0, 0), (64, 64)],
    "long_chunk": [(1500, 200)],
    "few_behind_many": [(6000, 70)],      # (the tiled kernel cuts it)
}
BOTH = [(k, l) for k in ("auto", "tiled") for l in LAYERS if k == "auto" or LAYERS[l][3] == "bf16"]


@pytest.mark.parametrize("kernel,layer", BOTH)
@pytest.mark.parametrize("form", list(FORMS))
def test_attention(kernel, layer, form):
    page = {"decode": 16, "one_long": 16, "verify": 8, "chunk": 64, "prompt": 32, "mixed": 24, "long_chunk": 128, "few_behind_many": 16}[form]
    bt = make_batch(LAYERS[layer], FORMS[form], page, seed=len(layer) + len(form))
    ctx = make_ctx(LAYERS[layer], kernel=kernel)
    out, lse = run_attn(ctx, bt)
    rows = None if len(bt["q"]) < 60 else {int(t) for o in bt["offs"] for t in (o - 2, o - 1, o, o + 1)} | set(range(0, len(bt["q"]), 13))
    check_attn(bt, out, lse, rows)
    again, _ = run_attn(ctx, bt, lse=False)
    assert torch.equal(out, again)                     # the same bits, with and without the normalisers
    ctx.close()


FEW = [("auto", "g4"), ("auto", "g2_d64"), ("auto", "f32_d64"), ("tiled", "g4"), ("tiled", "g2_d64")]


@pytest.mark.parametrize("kernel,layer", FEW)
@pytest.mark.parametrize("form", ["decode", "one_long", "verify", "mixed", "long_chunk", "few_behind_many"])
def test_what_an_earlier_call_left_in_the_workspace(kernel, layer, form):
    """Partial results of a batch that is NaN throughout lie where the next call's go: nothing of them is read."""
    ctx = make_ctx(LAYERS[layer], kernel=kernel)
    for lens in ([(900, 1)] * 40, [(1000, 300), (500, 200)], [(6000, 1)], [(3000, 70)]):
        nan = make_batch(LAYERS[layer], lens, 16, seed=1)
        nan["kp"][:], nan["vp"][:] = np.nan, np.nan
        run_attn(ctx, nan)
    bt = make_batch(LAYERS[layer], FORMS[form], 16, seed=3)
    out, lse = run_attn(ctx, bt)
    check_attn(bt, out, lse, None if len(bt["q"]) < 60 else set(range(0, len(bt["q"]), 13)) | {len(bt["q"]) - 1} | {131, 132, 133})
    ctx.close()


@pytest.mark.parametrize("page", [1, 2, 3, 5, 8, 12, 16, 20, 31, 100, 256, 5000])
@pytest.mark.parametrize("kernel,layer", FEW)
def test_page_sizes(kernel, layer, page):
    bt = make_batch(LAYERS[layer], [(333, 1), (64, 70), (0, 3)], page, seed=page)
    ctx = make_ctx(LAYERS[layer], kernel=kernel)
    out, lse = run_attn(ctx, bt)
    check_attn(bt, out, lse, set(range(0, 74, 5)) | {0, 1, 70, 71, 73})
    ctx.close()


@pytest.mark.parametrize("kernel,layer", [(k, l) for k in ("auto", "tiled") for l in ("g4", "g7", "g8_d64", "f32_g5_d128") if (k, l) != ("tiled", "f32_g5_d128")])
def test_what_a_row_does_not_see(kernel, layer):
    """Values and keys of later rows of the chunk that are not finite, pages that are not there, rows that see nothing."""
    bt = make_batch(LAYERS[layer], [(100, 40), (37, 1), (-3, 6), (-9, 4), (200, 90)], 16, seed=5, pad=4)
    Hq, Hkv, d, dt = LAYERS[layer]
    for x, at, what in ((bt["vp"], 120, np.inf), (bt["vp"], 127, np.nan), (bt["kp"], 130, np.nan), (bt["vp"], 139, -np.inf), (bt["kp"], 125, 3e38)):
        x[bt["table"][0, at // 16], at % 16] = what
    bt["vp"][bt["table"][4, 250 // 16], 250 % 16] = np.nan
    bt["table"][4, 2], bt["table"][4, 7], bt["table"][4, 0] = -1, len(bt["kp"]), -2 ** 31
    bt["table"][1, :] = -1
    ctx = make_ctx(LAYERS[layer], kernel=kernel)
    out, lse = run_attn(ctx, bt)
    o = [int(x) for x in bt["offs"]]
    clean = {t for t in range(o[0], o[1]) if 100 + t < 120} | set(range(o[1], o[4])) | {o[4] + t for t in range(90) if 200 + t < 250}
    check_attn(bt, out, lse, clean)
    got = down(out)
    assert np.all(got[o[5]:] == 7) and np.all(down(lse)[o[5]:] == 7)        # rows of no request
    assert np.all(np.isinf(got[o[0] + 20: o[0] + 25]) | np.isnan(got[o[0] + 20: o[0] + 25]))   # and those that see the infinity show it
    assert np.all(np.isnan(got[o[4] + 50: o[5]]))
    assert np.all(got[o[1]] == 0) and np.all(np.isneginf(down(lse)[o[1]]))
    ctx.close()


@pytest.mark.parametrize("kernel,layer", FEW)
def test_large_and_growing_logits(kernel, layer):
    """The largest logits come late, hundreds above the first: whatever reference the weights have, they keep their size."""
    Hq, Hkv, d, dt = LAYERS[layer]
    bt = make_batch(LAYERS[layer], [(900, 1), (300, 80), (2000, 1), (500, 300)], 16, seed=9, q_scale=4.0)
    for b, (c, n) in enumerate([(900, 1), (300, 80), (2000, 1), (500, 300)]):
        for j in range(c + n):
            bt["kp"][bt["table"][b, j // 16], j % 16] *= 1 + 9.0 * (j / (c + n)) ** 3
    bt["kp"] = stored(np.nan_to_num(bt["kp"], nan=0.0), dt) + np.where(np.isnan(bt["kp"]), np.float32(np.nan), np.float32(0))
    ctx = make_ctx(LAYERS[layer], kernel=kernel)
    out, lse = run_attn(ctx, bt)
    check_attn(bt, out, lse, set(range(0, 382, 11)) | {0, 1, 80, 81, 82, 381})
    ctx.close()


@pytest.mark.parametrize("kernel,layer", [("auto", "g4"), ("tiled", "g4"), ("auto", "f32_d64")])
def test_rows_beyond_max_new_and_a_narrow_table(kernel, layer):
    bt = make_batch(LAYERS[layer], [(10, 50), (5, 1)], 16, seed=2)
    ctx = make_ctx(LAYERS[layer], kernel=kernel)
    want, _ = run_attn(ctx, bt)
    out, _ = run_attn(ctx, bt, max_new=20)
    assert torch.equal(out[:20], want[:20]) or np.allclose(down(out[:20]), down(want[:20]), atol=2 * UBF * 4)   # (another kernel may take them)
    assert bool((out[20:50] == 7).all()) and not bool((out[50] == 7).any())
    narrow = dict(bt, table=bt["table"][:, :2])                       # positions from 32 on are invisible
    out, lse = run_attn(ctx, narrow)
    check_attn(narrow, out, lse)
    ctx.close()


@pytest.mark.parametrize("kernel", ["stream", "tiled"])
def test_offsets_beyond_32_bits(kernel):
    """Pages at the end of a cache of more than 2^32 bytes, and a row index beyond 2^31 elements."""
    layer = (8, 8, 128, "bf16")
    n_pages, page = 150000, 16                                        # 4.9 GB each
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
    k = up(np.random.default_rng(0).standard_normal((1, 8, 128)), "bf16")
    ctx.fr_paged_append(None, k, k, None, i32([n_pages * page - 1]), 1, kp, vp, n_pages, page)
    assert torch.equal(kp[-1, -1], k[0]) and torch.equal(vp[-1, -1], k[0])
    ctx.close()


@pytest.mark.parametrize("kernel,layer", FEW)
@pytest.mark.parametrize("form", ["decode", "one_long", "mixed", "few_behind_many"])
def test_outputs_in_the_place_of_the_queries(kernel, layer, form):
    """Whole items, cut ones and (logits that outgrow the first keys') items that are taken twice."""
    bt = make_batch(LAYERS[layer], FORMS[form], 16, seed=3)
    ctx = make_ctx(LAYERS[layer], kernel=kernel)
    for scale in (1.0, 100.0):
        dt = LAYERS[layer][3]
        dev = dict(q=up(bt["q"] * scale, dt), kp=up(bt["kp"], dt), vp=up(bt["vp"], dt), offs=i32(bt["offs"]), cached=i32(bt["cached"]), table=i32(bt["table"]))
        want, _ = run_attn(ctx, bt, dev=dev)
        q = dev["q"]
        ctx.fr_paged_attn(q, dev["offs"], dev["cached"], len(bt["cached"]), len(bt["q"]), bt["max_new"], dev["kp"], dev["vp"], len(bt["kp"]), bt["page"], dev["table"],
                          bt["table"].shape[1], q)
        n = int(bt["offs"][-1])
        assert torch.equal(q[:n], want[:n])
    ctx.close()


@pytest.mark.parametrize("kernel", ["auto", "tiled"])
@pytest.mark.parametrize("heads", [(130, 1), (320, 320), (96, 2)])
def test_wide_groups_and_many_heads(kernel, heads):
    """A group wider than a tile of the streaming kernel and than half of the tiled one's, more KV heads than compute units."""
    layer = heads + (64, "bf16")
    bt = make_batch(layer, [(300, 3), (0, 1), (70, 9)], 16, seed=heads[0])
    ctx = make_ctx(layer, kernel=kernel)
    out, lse = run_attn(ctx, bt)
    check_attn(bt, out, lse)
    ctx.close()


@pytest.mark.parametrize("kernel", ["auto", "tiled"])
def test_many_requests_and_empty_ones(kernel):
    rng = np.random.default_rng(8)
    lens = [(int(rng.integers(0, 40)), int(rng.integers(0, 3))) for _ in range(1500)]
    bt = make_batch((2, 1, 64, "bf16"), lens, 8, seed=4)
    ctx = make_ctx(bt["layer"], kernel=kernel)
    out, lse = run_attn(ctx, bt)
    check_attn(bt, out, lse, set(range(0, len(bt["q"]), 17)) | {len(bt["q"]) - 1})
    ctx.close()


@pytest.mark.parametrize("kernel", ["auto", "tiled"])
def test_a_prompt_in_one_call_and_in_chunks(kernel):
    """2500 positions at once, and the same as chunks of 900 behind one another: sampled rows against the oracle, the two against each other."""
    layer = (8, 2, 128, "bf16")
    bt = make_batch(layer, [(0, 2500)], 64, seed=6)
    ctx = make_ctx(layer, kernel=kernel)
    out, lse = run_attn(ctx, bt)
    check_attn(bt, out, lse, {0, 1, 63, 64, 65, 255, 256, 257, 1000, 1777, 2498, 2499})
    for c in range(0, 2500, 900):
        n = min(900, 2500 - c)
        part = dict(bt, cached=np.array([c]), offs=np.array([0, n]), q=bt["q"][c: c + n], max_new=n)
        o, l = run_attn(ctx, part)
        assert np.allclose(down(o), down(out[c: c + n]), atol=2 * UBF * 4, rtol=0) and np.allclose(down(l), down(lse[c: c + n]), atol=1e-4)
    ctx.close()


@pytest.mark.parametrize("lens,pad_blocks", [([(700, 400), (300, 1)], 600), ([(100, 300)] * 3 + [(2000, 1)] * 30, 0), ([(6000, 900)], 0), ([(3000, 700), (9, 1)], 400)])
def test_both_kernels_in_a_call(lens, pad_blocks):
    """Sizes on both sides of the rule, tables as wide as they need to be and wider (the kernels then find out which of them works): the
    same rows as either kernel alone gives, up to their roundings, whatever the rule says."""
    layer = (32, 8, 128, "bf16")
    rng = np.random.default_rng(0)
    need = [-(-(c + n) // 16) for c, n in lens]
    n_pages, T = sum(need) + 1, sum(n for _, n in lens)
    ids, at = rng.permutation(n_pages), 0
    table = np.full((len(lens), max(need) + pad_blocks), -1)
    for b, k in enumerate(need):
        table[b, :k] = ids[at: at + k]
        at += k
    f = lambda *s: torch.randn(s, generator=torch.Generator(device="cuda").manual_seed(len(s) * sum(s)), device="cuda").bfloat16()
    dev = dict(q=f(T, 32, 128), kp=f(n_pages, 16, 8, 128), vp=f(n_pages, 16, 8, 128) * 0.5, offs=i32(np.concatenate([[0], np.cumsum([n for _, n in lens])])),
               cached=i32([c for c, _ in lens]), table=i32(table))
    bt = dict(layer=layer, page=16, table=table, kp=dev["kp"], cached=lens, q=np.empty((T, 32, 0)), max_new=max(n for _, n in lens))
    got = {}
    for kernel in ("auto", "stream", "tiled"):
        ctx = make_ctx(layer, kernel=kernel)
        got[kernel] = [x.clone() for x in run_attn(ctx, bt, dev=dev)]
        ctx.close()
    for kernel in ("stream", "tiled"):
        # two roundings of each weight, two of each output, of values of at most 3 (the weights' mean of |value| is 0.4)
        assert float((got["auto"][0].float() - got[kernel][0].float()).abs().max()) <= 4 * UBF * 3
        assert float((got["auto"][1] - got[kernel][1]).abs().max()) <= 1e-4


# ---- the step ------------------------------------------------------------------------------------------------------------

def _step_case(layer, seed):
    Hq, Hkv, d, dt = layer
    rng = np.random.default_rng(seed)
    n, page, n_pages = 5, 8, 120
    f = lambda *s: up(rng.standard_normal(s), dt)
    st = dict(n=n, page=page, n_pages=n_pages, T=64, table=i32(np.full((n, 20), -1)), free=i32(rng.permutation(n_pages)), start=i32([0]), cached=i32(np.zeros(n)),
              new=i32([7, 1, 0, 30, 5]), off=i32(np.zeros(n + 1)), pos=i32(np.zeros(64)), slots=i32(np.zeros(64)), need=i32([0]),
              q=f(64, Hq, d), k=f(64, Hkv, d), v=f(64, Hkv, d), kp=f(n_pages, page, Hkv, d), vp=f(n_pages, page, Hkv, d))
    st["qr"], st["out"] = torch.empty_like(st["q"]), torch.zeros_like(st["q"])
    st["lse"] = torch.zeros((64, Hq), device="cuda")
    return st


def _step(ctx, s):
    ctx.fr_page_tables(s["cached"], s["new"], s["n"], s["page"], s["free"], s["n_pages"], s["start"], s["table"], 20, s["T"], s["off"], s["pos"], s["slots"], s["need"])
    ctx.fr_paged_append(s["q"], s["k"], s["v"], s["pos"], s["slots"], s["T"], s["kp"], s["vp"], s["n_pages"], s["page"], s["qr"])
    ctx.fr_paged_attn(s["qr"], s["off"], s["cached"], s["n"], s["T"], 30, s["kp"], s["vp"], s["n_pages"], s["page"], s["table"], 20, s["out"], s["lse"])
    s["cached"] += s["off"][1:] - s["off"][:-1]
    s["start"] += s["need"]


STEPS = [[7, 1, 0, 30, 5], [1, 1, 1, 1, 1], [3, 0, 30, 2, 1], [1, 8, 1, 1, 0]]


@pytest.mark.parametrize("layer", ["g4", "g2_d64", "f32_g5_d128"])
def test_steps_against_the_oracle(layer):
    """Four steps of five requests, everything followed by the oracle from the stored values on."""
    Hq, Hkv, d, dt = LAYERS[layer]
    ctx, s = make_ctx(LAYERS[layer]), _step_case(LAYERS[layer], 1)
    table, cached, start = s["table"].cpu().numpy(), np.zeros(5, dtype=np.int64), 0
    for new in STEPS:
        s["new"].copy_(i32(new))
        s["out"].fill_(7)
        table, off, pos, slots, need = orc.page_tables(cached, new, 8, s["free"].cpu().numpy(), start, table, 64)
        before = down(s["kp"]), down(s["vp"])
        _step(ctx, s)
        assert np.array_equal(s["table"].cpu().numpy(), table) and np.array_equal(s["slots"].cpu().numpy(), slots)
        wq, wk, wv = orc.paged_append(down(s["q"]), down(s["k"]), down(s["v"]), pos, slots, *before, 5e5)
        u = UBF if dt == "bf16" else U32
        for got, want in ((s["qr"], wq), (s["kp"], wk)):
            assert np.all(np.abs(down(got) - want) <= u * np.abs(want) + 1e-5)
        assert np.array_equal(down(s["vp"]), wv)
        check_attn(dict(layer=LAYERS[layer], page=8, table=table, kp=down(s["kp"]), vp=down(s["vp"]), offs=off, cached=cached, q=down(s["qr"])), s["out"], s["lse"])
        assert bool((s["out"][off[-1]:] == 7).all())
        cached, start = cached + np.diff(off), start + need
    ctx.close()


@pytest.mark.parametrize("kernel,layer", [("auto", "g4"), ("auto", "f32_d64"), ("tiled", "g4")])
def test_a_captured_step_is_replayed_for_other_lengths(kernel, layer):
    ctx, s = make_ctx(LAYERS[layer], kernel=kernel), _step_case(LAYERS[layer], 2)
    other_ctx, e = make_ctx(LAYERS[layer], kernel=kernel), _step_case(LAYERS[layer], 2)
    _step(ctx, s)                                             # once eagerly, on both
    _step(other_ctx, e)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    saved = s["cached"].clone(), s["start"].clone()
    with torch.cuda.graph(g):
        _step(ctx, s)
    s["cached"].copy_(saved[0]); s["start"].copy_(saved[1])
    for new in STEPS + STEPS[1:2]:
        for x in (s, e):
            x["new"].copy_(i32(new))
            for t in ("q", "k", "v"):
                x[t].mul_(0.5).add_(0.25)
        g.replay()
        torch.cuda.synchronize()
        _step(other_ctx, e)
        torch.cuda.synchronize()
        for name in ("table", "off", "pos", "slots", "need", "qr", "kp", "vp", "out", "lse", "cached", "start"):
            assert torch.equal(s[name], e[name]), name
    ctx.close()
    other_ctx.close()


def test_two_contexts_on_two_streams():
    """Two steps at once, each with a context of its own, on streams of their own."""
    pairs = [(make_ctx(LAYERS[n]), _step_case(LAYERS[n], 3)) for n in ("g4", "g2_d64")]
    want = []
    for c, s in pairs:
        _step(c, s)
        want.append((s["out"].clone(), s["lse"].clone()))
        s["cached"].zero_(); s["start"].zero_(); s["out"].zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in pairs]
    for (c, s), st in zip(pairs, streams):
        with torch.cuda.stream(st):
            _step(c, s)
    torch.cuda.synchronize()
    for (c, s), (o, l) in zip(pairs, want):
        assert torch.equal(s["out"], o) and torch.equal(s["lse"][: int(s["off"][-1])], l[: int(s["off"][-1])])
        c.close()


@pytest.mark.parametrize("d,half", [(128, False), (64, True)])
def test_stack_in_steps_equals_the_stack_at_once(d, half):
    """Decoder layers over a paged cache: prompts in one step, and in chunks and single rows, end in the same rows."""
    Hq, Hkv, hidden, ffn, L = 8, 2, 512, 256, 2
    gen = torch.Generator(device="cuda").manual_seed(3)
    layers = [S.random_layer(hidden, ffn, Hq, Hkv, d, gen, std=0.05) for _ in range(L)]
    ctx = make_ctx((Hq, Hkv, d, "bf16"), half, tokens=256)
    stack = S.PagedStack(ctx, layers, hidden, ffn)
    lens = [90, 41, 1]
    x = [torch.randn((n, hidden), generator=gen, device="cuda").bfloat16() for n in lens]
    whole_cache = S.PagedCache(L, 3, 40, 8, 16, Hkv, d)
    whole = stack.forward(torch.cat(x).clone(), i32(lens), 90, whole_cache)
    assert whole_cache.cached_len.tolist() == lens
    cache = S.PagedCache(L, 3, 40, 8, 16, Hkv, d)
    got, done = [[], [], []], [0, 0, 0]
    while done != lens:
        new = [min(n - k, m) for n, k, m in zip(lens, done, (37, 1, 1) if done[1] < 5 else (20, 36, 1))]
        h = torch.cat([a[k: k + m] for a, k, m in zip(x, done, new)] + [torch.ones((3, hidden), device="cuda").bfloat16()])
        out = stack.forward(h, i32(new), 40, cache)
        for b, o in enumerate(torch.split(out[: sum(new)], new)):
            got[b].append(o.clone())
        done = [k + m for k, m in zip(done, new)]
    assert cache.cached_len.tolist() == lens and int(cache.free_start) == int(whole_cache.free_start) == 12 + 6 + 1
    got = torch.cat([torch.cat(g) for g in got])
    # about ten roundings of 2^-8 a layer lie between the two orders of work, each of a value of the rows' own size
    size = float(whole.float().abs().max())
    assert float((got.float() - whole.float()).abs().max()) <= 10 * L * UBF * size
    assert torch.isfinite(got.float()).all()
    ctx.close()


def test_captured_stack_steps_beside_eager_ones():
    """Two captured steps of one stack (a decoding step, a chunk) and eager steps of other sizes between their replays: the rows of
    the same steps taken eagerly."""
    Hq, Hkv, d, hidden, ffn, L, n = 8, 2, 128, 512, 256, 2, 3
    gen = torch.Generator(device="cuda").manual_seed(5)
    layers = [S.random_layer(hidden, ffn, Hq, Hkv, d, gen, std=0.05) for _ in range(L)]
    x = torch.randn((400, hidden), generator=gen, device="cuda").bfloat16()
    results = []
    for captured in (False, True):
        ctx = make_ctx((Hq, Hkv, d, "bf16"), tokens=256)
        stack = S.PagedStack(ctx, layers, hidden, ffn)
        cache = S.PagedCache(L, n, 60, 8, 16, Hkv, d)
        graphs = {}
        if captured:
            for T in (n, 48):
                h, new = torch.zeros((T, hidden), device="cuda").bfloat16(), i32([0] * n)
                stack.forward(h, new, T, cache)      # (once outside: the library's first calls set up what a capture may not; no rows)
                torch.cuda.synchronize()
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g):
                    stack.forward(h, new, T, cache)
                graphs[T] = g, h, new
        got, at = [], 0
        for new in ([20, 0, 28], [1, 1, 1], [30, 5, 7], [1, 0, 1], [10, 20, 18], [1, 1, 1]):
            T = n if max(new) == 1 else 48 if new != [30, 5, 7] else 50      # (50 rows: always eager)
            rows = x[at: at + T].clone()
            at += sum(new)
            if T in graphs:
                g, h, dev_new = graphs[T]
                h.copy_(rows)
                dev_new.copy_(i32(new))
                g.replay()
                torch.cuda.synchronize()
                rows = h.clone()
            else:
                stack.forward(rows, i32(new), T, cache)
            got.append(rows[: sum(new)])
        assert cache.cached_len.tolist() == [63, 27, 56]
        results.append(torch.cat(got))
        ctx.close()
    assert torch.isfinite(results[0].float()).all() and torch.equal(results[0], results[1])
