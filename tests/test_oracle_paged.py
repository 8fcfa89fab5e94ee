"""Pins of the oracle's paged step: worked examples by hand, and its attention against the causal attention that is written row by row."""
import numpy as np

from oracle import fusionrag_oracle as orc


def test_tables_worked_example():
    # pages of 4: request 0 holds 5 positions (2 pages) and brings 4, request 1 is new with 5, request 2 brings nothing, request 3 ends a page
    table = np.array([[7, 8, -5, -5], [-5, -5, -5, -5], [3, -5, -5, -5], [1, -5, -5, -5]])
    t, offs, pos, slots, taken = orc.page_tables([5, 0, 2, 3], [4, 5, 0, 1], 4, [20, 21, 22, 23, 24], 1, table, 12)
    assert t.tolist() == [[7, 8, 21, -5], [22, 23, -5, -5], [3, -5, -5, -5], [1, -5, -5, -5]] and taken == 3
    assert offs.tolist() == [0, 4, 9, 9, 10]
    assert pos.tolist() == [5, 6, 7, 8, 0, 1, 2, 3, 4, 3, 0, 0]
    assert slots.tolist() == [33, 34, 35, 84, 88, 89, 90, 91, 92, 7, -1, -1]


def test_tables_short_list_narrow_table_and_few_rows():
    t, offs, pos, slots, taken = orc.page_tables([0, 0], [5, 9], 2, [9, 4], 0, np.full((2, 3), -7), 10)
    assert t.tolist() == [[9, 4, -1], [-1, -1, -1]] and taken == 6        # the list ends after two pages; three blocks are all there are
    assert offs.tolist() == [0, 5, 10]                                     # ten rows: the second request is cut
    assert slots.tolist() == [18, 19, 8, 9, -1, -1, -1, -1, -1, -1]
    assert pos.tolist() == [0, 1, 2, 3, 4, 0, 1, 2, 3, 4]


def test_paged_attention_is_the_causal_attention_of_each_request():
    rng = np.random.default_rng(3)
    P, Hq, Hkv, d, lens = 3, 4, 2, 8, [(0, 5), (4, 1), (2, 6)]
    table = np.array([[4, 9, -1], [1, 0, -1], [5, 2, 8]])
    kp, vp = rng.standard_normal((10, P, Hkv, d)), rng.standard_normal((10, P, Hkv, d))
    offs = np.concatenate([[0], np.cumsum([n for _, n in lens])])
    q = rng.standard_normal((offs[-1], Hq, d))
    got = orc.paged_attn(q, offs, [c for c, _ in lens], kp, vp, table)
    for b, (c, n) in enumerate(lens):
        k, v = (x[table[b]].reshape(-1, Hkv, d)[: c + n] for x in (kp, vp))
        full = np.concatenate([rng.standard_normal((c, Hq, d)), q[offs[b]: offs[b + 1]]])
        want = orc.full_causal_attention(full, k, v)[c:]
        assert np.allclose(np.stack([got[t][0] for t in range(offs[b], offs[b + 1])]), want, atol=1e-12)


def test_invisible_positions():
    rng = np.random.default_rng(4)
    kp, vp = rng.standard_normal((4, 2, 1, 8)), rng.standard_normal((4, 2, 1, 8))
    q = rng.standard_normal((3, 1, 8))
    got = orc.paged_attn(q, [0, 1, 2, 3], [3, -4, 3], kp, vp, np.array([[1, -1], [0, 1], [-1, 9]]))
    only = orc.paged_attn(q, [0, 1, 1, 1], [1, 0, 0], kp, vp, np.array([[1, -1], [0, 1], [0, 1]]))
    assert np.array_equal(got[0][0], only[0][0])
    assert np.all(got[1][0] == 0) and np.all(np.isneginf(got[1][1])) and np.all(got[2][0] == 0)


def test_append_places_rows():
    rng = np.random.default_rng(5)
    k, v, q = rng.standard_normal((3, 1, 8)), rng.standard_normal((3, 1, 8)), rng.standard_normal((3, 2, 8))
    kp = np.zeros((2, 2, 1, 8))
    qo, k2, v2 = orc.paged_append(q, k, v, [5, 6, 7], [2, -1, 9], kp, kp, 1e4)
    assert np.array_equal(v2[1, 0], v[0]) and np.array_equal(k2[1, 0], orc.rope_rotate(k, [5, 6, 7], 1e4)[0])
    assert np.all(k2[0] == 0) and np.all(k2[1, 1] == 0) and np.array_equal(qo, orc.rope_rotate(q, [5, 6, 7], 1e4))
    _, k3, _ = orc.paged_append(None, k, v, None, [0, 1, 2], kp, kp, 1e4)
    assert np.array_equal(k3.reshape(4, 1, 8)[:3], k)
