"""Sequences that radar_kvq_blocks refuses, in the oracle: a pass over them touches no block of another sequence."""
import numpy as np

from kvq_util import bf16, random_cache, seed
from oracle import kvq


def test_a_refused_sequence_does_not_follow_what_it_gave_back():
    """Sequence 0 gives a block back, sequence 1 takes it, sequence 0 asks again and there is none."""
    R, D, H, T = 16, 64, 1, 8
    tables, owned = np.array([[0, 1, -1], [2, 3, -1], [4, -1, -1]], np.int32), np.array([2, 2, 1], np.int32)
    free, n_free = np.full(5, -1, np.int32), 0
    _, granted, owned, n_free, tables, free = kvq.blocks([8, 28, 8], [8, 8, 8], tables, owned, free, n_free, R, T)
    assert granted.tolist() == [1, 1, 1] and tables[1].tolist() == [2, 3, 1] and n_free == 0
    ctx = np.array([14, 32, 8], np.int32)
    slots, granted, owned, n_free, tables, free = kvq.blocks(ctx, [8, 8, 8], tables, owned, free, n_free, R, T)
    assert granted.tolist() == [0, 1, 1] and owned.tolist() == [1, 3, 1] and (slots[0] == -1).all()
    assert tables.tolist() == [[0, -1, -1], [2, 3, 1], [4, -1, -1]]
    rng = seed(110)
    cache = random_cache(rng, 1, 5, H, R, D)
    path = np.tile(np.arange(0, 9, 2, dtype=np.int32), (3, 1))
    new, _ = kvq.commit(cache, R, D, tables, ctx, np.array([4, 0, 0], np.int32), path)
    assert np.array_equal(new[:, 1:], cache[:, 1:])
    q = bf16(rng.normal(size=(3, T, 2, D)))[0]
    out, _ = kvq.attention(q, cache, R, D, 0, tables, ctx)
    cache[:, 1:] = random_cache(rng, 1, 4, H, R, D)                  # whatever the others' blocks hold
    assert np.array_equal(out[0], kvq.attention(q, cache, R, D, 0, tables, ctx)[0][0])


def test_no_refused_sequence_knows_of_a_block_that_is_not_its_own():
    rng = seed(111)
    B, M, R, T, n = 9, 7, 16, 20, 30
    tables, owned = rng.integers(0, n, (B, M)).astype(np.int32), np.zeros(B, np.int32)              # (entries behind the owned ones hold anything)
    free, n_free, refused = rng.permutation(n).astype(np.int32), n, 0
    for _ in range(200):
        ctx = np.where(rng.random(B) < 0.2, -1, rng.integers(0, 120, B)).astype(np.int32)
        new = rng.integers(0, T + 1, B).astype(np.int32)
        before = tables.copy()
        _, granted, owned, n_free, tables, free = kvq.blocks(ctx, new, tables, owned, free, n_free, R, T)
        for b in range(B):
            if granted[b]:                                           # entries behind the owned ones are left as they were
                assert np.array_equal(tables[b, owned[b]:], before[b, owned[b]:])
            else:
                assert (tables[b, owned[b]:] == -1).all() and np.array_equal(tables[b, :owned[b]], before[b, :owned[b]])
                refused += owned[b] > 0
    assert refused > 50
