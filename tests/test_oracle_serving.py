"""Pins of the serving oracle (CPU): visible sets by brute force, limits that
reduce to plain attention, closed forms, and invariants of the page pool."""
import numpy as np
import pytest

import oracle
from oracle import serving as S


def test_visible_sets_small():
    assert S.visible(0, 10, 3, 2) == [0, 1, 8, 9, 10]
    assert S.visible(2, 10, 3, 0) == [10, 11, 12]
    assert S.visible(0, 0, 1, 0) == [0]
    assert S.visible(1, 1, 1, 5) == [0, 1, 2]
    assert S.visible(3, 4, 100, 0) == [0, 1, 2, 3, 4, 5, 6, 7]
    # root 0, children 1 2, grandchild 3 of 1: positions 10, 11, 11, 12
    par = [-1, 0, 0, 1]
    assert S.visible(3, 10, 3, 1, par) == [0, 10, 11, 13]
    assert S.visible(2, 10, 3, 0, par) == [9, 10, 12]
    assert S.visible(3, 10, 2, 0, par) == [11, 13]
    assert S.visible(3, 10, 1, 0, par) == [13]
    assert S.visible(3, 10, 1, 11, par) == list(range(10)) + [10, 13]


def test_wide_window_is_plain_causal_attention():
    rng = np.random.default_rng(0)
    T, H, D, L = 5, 2, 8, 7
    q, k, v = (rng.standard_normal((1, n, H, D)) for n in (T, L + T, L + T))
    sel = [(0, t, h) for t in range(T) for h in range(H)]
    out, lse, _ = oracle.attention_rows(q, k, v, [T], [L], 0.3, True, sel)
    got = S.window_rows(q[0], lambda s, g: (k[0, s, g], v[0, s, g]), L, 0.3, 10 ** 6, 0, lambda h: h,
                        sel=[(t, h) for _, t, h in sel])
    for i, (o, _, z) in enumerate(got):
        np.testing.assert_allclose(o, out[i], rtol=1e-12)
        np.testing.assert_allclose(z, lse[i], rtol=1e-12)


def test_equal_scores_average_the_window():
    v = np.arange(20.0)[:, None]
    (o, a, z), = S.window_rows(np.zeros((3, 1, 1)), lambda s, g: (np.ones((len(s), 1)), v[s]), 15, 1.0, 4, 2,
                               lambda h: h, sel=[(2, 0)])
    seen = [0, 1, 14, 15, 16, 17]
    assert o[0] == pytest.approx(np.mean(seen)) and a[0] == pytest.approx(np.mean(seen))
    assert z == pytest.approx(np.log(len(seen)))


def _holders(table, n):
    return np.bincount(table[table >= 0], minlength=n)


def test_pool_counts_stay_the_holders():
    rng = np.random.default_rng(3)
    B, P, n = 6, 8, 40
    table, ref = np.full((B, P), -1, np.int32), np.zeros(n, np.int32)
    lens = np.zeros(B, np.int32)
    pools = [rng.standard_normal((1, n, S.PAGE, 1))]
    for _ in range(60):
        kind = rng.integers(3)
        if kind == 0:
            grow = rng.integers(0, 90, B).astype(np.int32)
            new_table, ref, f = S.reserve(table, ref, lens, grow)
            for b in range(B):
                if lens[b] + grow[b] <= P * S.PAGE and all(new_table[b, : -(-(lens[b] + grow[b]) // S.PAGE)] >= 0):
                    lens[b] += grow[b]
            table = new_table
        elif kind == 1:
            parent = rng.integers(-1, B, B)
            table, ref, lens, f = S.fork(table, ref, parent, lens, pools)
        else:
            table, ref, f = S.release(table, ref, lens, np.full(B, P * S.PAGE))
        assert (_holders(table, n) == ref).all()
        # the page of the next slot belongs to one sequence
        for b in range(B):
            for e in range(lens[b] // S.PAGE, P):
                assert table[b, e] < 0 or ref[table[b, e]] == 1


def test_fork_copies_what_each_row_held():
    rng = np.random.default_rng(5)
    B, P, n = 5, 3, 20
    table = np.full((B, P), -1, np.int32)
    lens = np.array([70, 64, 5, 130, 0], np.int32)
    ref = np.zeros(n, np.int32)
    table, ref, _ = S.reserve(table, ref, np.zeros(B, np.int32), lens)
    pool = rng.standard_normal((2, n, S.PAGE, 3))
    rows = lambda b: np.concatenate([pool[:, table[b, s // 64], s % 64] for s in range(lens[b])] or [np.zeros(0)])  # noqa: E731
    before = [rows(b) for b in range(B)]
    parent = [3, 0, 0, 2, 3]
    table, ref, lens, f = S.fork(table, ref, parent, lens, [pool])
    assert f == 0
    for i, q in enumerate(parent):
        np.testing.assert_array_equal(rows(i), before[q])


def test_prune_moves_small():
    assert S.prune_moves([3, 5], 2, 4, 9) == [(2, 3), (3, 5), (4, 6), (5, 7), (6, 8)]
    assert S.prune_moves([], 0, 2, 3) == [(0, 2)]
