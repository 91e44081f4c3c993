"""Pins for the oracle of rotary positions and of chunks of new tokens: turns against complex numbers in 80 bits and against what a rotation has to keep, chunk
attention against the oracle's chains, rows against row by row decoding."""
import numpy as np
import pytest

from kvq_util import random_cache, seed, tables_for
from oracle import kvq


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("P,D,axes", [(32, 64, 1), (8, 64, 3), (64, 128, 4), (24, 128, 2)])
def test_turns_are_complex_products(P, D, axes, interleaved):
    rng = seed(600 + P + axes)
    inv = (10000.0 ** (-np.arange(P) / P)).astype(np.float32)
    axis = rng.integers(0, axes, P)
    x = rng.normal(size=(3, D))
    for top in (10, 1 << 20, (1 << 31) - 1):
        pos = [int(p) for p in rng.integers(0, top, axes)]
        got = kvq.turn(x, pos, inv, axis, interleaved, 0.75)
        one = np.arange(P) * 2 if interleaved else np.arange(P)
        two = one + 1 if interleaved else one + P
        # the angle is an fp64 product: 31 bits by 24 may round; what is checked is the turn by that angle
        t = (np.array([pos[a] for a in axis], np.float64) * inv.astype(np.float64)).astype(np.longdouble)
        c, s = np.cos(t), np.sin(t)
        a, b = x[:, one].astype(np.longdouble), x[:, two].astype(np.longdouble)
        assert np.abs(got[:, one] - 0.75 * (a * c - b * s)).max() < 1e-14 and np.abs(got[:, two] - 0.75 * (a * s + b * c)).max() < 1e-14
        assert np.array_equal(got[:, 2 * P:], x[:, 2 * P:])


def test_scores_depend_on_differences_only():
    rng, inv = seed(610), (10000.0 ** (-np.arange(32) / 32)).astype(np.float32)
    q, k = rng.normal(size=(2, 1, 64))
    axis = np.arange(32) % 3
    base = None
    for shift in (0, 17, 100000):
        a = kvq.turn(q, [5 + shift, 3 + shift, 9 + shift], inv, axis)
        b = kvq.turn(k, [2 + shift, 3 + shift, 1 + shift], inv, axis)
        score = float((a @ b.T)[0, 0])
        base = score if base is None else base
        assert abs(score - base) < 1e-9
    assert np.allclose(np.linalg.norm(a), np.linalg.norm(q))
    once = kvq.turn(kvq.turn(q, [3, 4, 5], inv, axis), [10, 20, 30], inv, axis)
    assert np.abs(once - kvq.turn(q, [13, 24, 35], inv, axis)).max() < 1e-12


def test_rows():
    assert kvq.new_rows(2, 3) == [(0, 0, 0), (1, 0, 1), (2, 0, 2), (3, 1, 0), (4, 1, 1), (5, 1, 2)]
    assert kvq.new_rows(3, 3, ctx=[4, -1, 0], n_new=[1, 3, 9]) == [(0, 0, 0), (6, 2, 0), (7, 2, 1), (8, 2, 2)]
    assert kvq.new_rows(3, 2, ctx=[0, 0, 0], row_starts=[1, 1, 4, 5]) == [(1, 1, 0), (2, 1, 1), (4, 2, 0)]


@pytest.mark.parametrize("D,R,Hq,H", [(64, 16, 4, 2), (128, 32, 3, 1)])
def test_chunk_attention_is_a_chains(D, R, Hq, H):
    rng = seed(620 + D)
    B, T, ctx = 3, 7, np.array([20, 0, -1], np.int32)
    tables, n_blocks = tables_for(rng, [27, 7, 7], R, width=2)
    cache = random_cache(rng, 1, n_blocks, H, R, D)
    tables[0, 16 // R] = n_blocks                                          # rows of a block that is not there
    q = rng.normal(size=(B, T, Hq, D))
    nodes = np.array([7, 4, 2], np.int32)
    want = kvq.attention(q, cache, R, D, 0, tables, ctx, None, nodes, S_max=25, want_sizes=True)
    got = kvq.chunk_attention(q.reshape(B * T, Hq, D), cache, R, D, 0, tables, ctx, T, n_new=nodes, S_max=25)
    for w, g in zip(want, got):
        assert np.allclose(w.reshape(g.shape), g, rtol=1e-12, atol=1e-13, equal_nan=True)
    assert np.array_equal(got[4].reshape(B, T).sum(1), [7, 4, 0])
    starts = np.array([0, 7, 11, 11], np.int32)
    rows = np.concatenate([q[0], q[1, :4]])
    packed = kvq.chunk_attention(rows, cache, R, D, 0, tables, ctx, T, row_starts=starts, S_max=25)
    assert np.allclose(packed[0], np.concatenate([want[0][0], want[0][1, :4]]), rtol=1e-12, atol=1e-13)


def test_decoded_rows_are_the_ones_decoded_alone():
    rng, R, D = seed(630), 16, 64
    tables, n_blocks = tables_for(rng, [50], R)
    cache = random_cache(rng, 2, n_blocks, 3, R, D)
    tables[0, 2] = -1
    K, V, there = kvq.all_rows(cache, R, D, 1, tables[0], 70)
    for j in range(70):
        slot = kvq.row_slot(tables[0], R, n_blocks, j)
        k, v = kvq.get(cache, R, D, 1, slot)
        assert there[j] == (slot >= 0) and np.array_equal(K[j], k) and np.array_equal(V[j], v)
