"""Pins for the oracle of the paged 4-bit cache: the format against a search over all of its numbers, the layout against
its description, block tables against what they have to keep, attention against the oracle of the dense cache."""
import numpy as np
import pytest

from kvq_util import bf16, random_cache, random_parents, seed, tables_for
from oracle import kvq
from paper_2512_14069_amd import synth


def test_every_bf16_value_becomes_the_nearest_code():
    """One value of each block sets the scale, the others are all finite bf16 patterns in turn."""
    rng = seed(0)
    bits = np.arange(1 << 16, dtype=np.uint32).astype(np.uint16)
    vals = synth.bf16_bits_to_f32(bits).astype(np.float64)
    vals = vals[np.isfinite(vals)]
    for top in (1.0, 1.7421875, 1.75, 1.7578125, 2.0 ** -120, 3.0 * 2.0 ** 100):
        pick = vals[np.abs(vals) <= top]
        pick = pick[rng.permutation(len(pick))[:31 * 32]].reshape(32, 31)
        x = np.concatenate([np.full((32, 1), top), pick], 1)
        codes, scales = kvq.encode(x)
        got = kvq.decode(codes, scales)
        step = 2.0 ** (scales.astype(np.float64) - 127)
        every = np.concatenate([kvq.MAGNITUDES, -kvq.MAGNITUDES])
        best = np.abs(x[..., None] - every * step[..., None]).min(-1)
        assert np.array_equal(np.abs(x - got), best)
        assert (np.abs(x - got) <= step).all() and (top < 7 * step).all() and (top >= 7 * step / 2).all()


def test_ties_zero_and_the_ends_of_the_range():
    x = np.zeros((8, 32))
    x[0, :10] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -5]
    x[1, 0] = 0.0
    x[2, 0] = 2.0 ** -133                                            # the smallest bf16
    x[3, 0] = 1.9921875 * 2.0 ** 127                                 # the largest
    x[4, 3] = np.inf
    x[5, 31] = np.nan
    x[6, :2] = [7 * 2.0 ** -126, 2.0 ** -126]
    x[7, :2] = [6.96875, 6.5]
    c, s = kvq.encode(x)
    assert kvq.decode(c, s)[0, :10].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 0, -4]
    assert s[:, 0].tolist() == [127, 1, 1, 252, 255, 255, 2, 127]
    got = kvq.decode(c, s)
    assert got[2, 0] == 0 and got[3, 0] == 6 * 2.0 ** 125 and np.isnan(got[4]).all() and np.isnan(got[5]).all()
    assert got[7, 0] == 6 and got[7, 1] == 6
    again = kvq.encode(np.where(np.isnan(got), 0.0, got))
    assert np.array_equal(kvq.decode(*again)[:4], got[:4])


@pytest.mark.parametrize("R,D", [(16, 64), (16, 128), (32, 128), (128, 64)])
def test_a_chunk_is_filled_without_gaps_or_overlaps(R, D):
    rng = seed(1)
    cache = np.full((1, 2, 1, kvq.chunk_bytes(R, D)), 0xAA, np.uint8)
    count = np.zeros(kvq.chunk_bytes(R, D), int)
    for row in range(R):
        places, half, sc = kvq._code_places(R, D, row)
        for at in places:
            np.add.at(count, at, 1)
        for at in sc:
            np.add.at(count, at, 2)
    assert (count == 2).all()
    rows = rng.normal(size=(R, 2, 1, D))
    for row in rng.permutation(R):
        kvq.put(cache, R, D, 0, R + row, *rows[row])
    assert (cache[0, 0] == 0xAA).all()
    for row in range(R):
        for x, y in zip(kvq.get(cache, R, D, 0, R + row), rows[row]):
            assert np.array_equal(x, kvq.decode(*kvq.encode(y)))
    assert kvq.get(cache, R, D, 0, 2 * R)[0].sum() == 0 and kvq.get(cache, R, D, 0, -1)[1].sum() == 0


def test_blocks_are_never_lost_or_held_twice():
    rng = seed(2)
    B, M, R, T, n = 9, 7, 16, 20, 30
    tables, owned = np.full((B, M), -1, np.int32), np.zeros(B, np.int32)
    free, n_free = rng.permutation(n).astype(np.int32), n
    refused = 0
    for _ in range(200):
        ctx = np.where(rng.random(B) < 0.2, -1, rng.integers(0, 120, B)).astype(np.int32)
        new = rng.integers(0, T + 1, B).astype(np.int32)
        slots, granted, owned, n_free, tables, free = kvq.blocks(ctx, new, tables, owned, free, n_free, R, T)
        held = [t for b in range(B) for t in tables[b, :owned[b]]]
        assert sorted(held + free[:n_free].tolist()) == list(range(n))
        for b in range(B):
            want = 0 if ctx[b] < 0 else -(-(ctx[b] + new[b]) // R)
            assert (owned[b] == want) if granted[b] else True
            live = slots[b][slots[b] >= 0]
            assert len(live) == (new[b] if granted[b] and ctx[b] >= 0 else 0)
            assert all(s // R in held for s in live)
        used = slots[slots >= 0]
        assert len(set(used)) == len(used)
        refused += int((granted == 0).sum())
    assert refused > 50


def test_attention_agrees_with_the_oracle_of_the_dense_cache():
    import oracle
    rng = seed(3)
    for D, H, G, R, T, ctx in ((64, 1, 4, 16, 7, [5, 40, 0]), (128, 2, 2, 32, 12, [33, 0, 64])):
        B = len(ctx)
        nodes = np.array([T, 3, 1], np.int32)
        table, n_blocks = tables_for(rng, [c + T for c in ctx], R)
        cache = random_cache(rng, 1, n_blocks, H, R, D)
        par = random_parents(rng, B, T, nodes)
        q, qbits = bf16(rng.normal(size=(B, T, H * G, D)))
        out, lse = kvq.attention(q, cache, R, D, 0, table, np.array(ctx), par, nodes)
        S = max(ctx) + T
        kc = np.zeros((B, H, S, D))
        vc = np.zeros((B, H, S, D))
        for b in range(B):
            for j in range(ctx[b] + T):
                kc[b, :, j], vc[b, :, j] = kvq.get(cache, R, D, 0, kvq.row_slot(table[b], R, n_blocks, j))
        ref, rlse = oracle.tree_attention(qbits, bf16(kc)[1], bf16(vc)[1], par, np.array(ctx, np.int32), nodes, want_lse=True)
        assert np.array_equal(bf16(kc)[0], kc) and np.array_equal(bf16(vc)[0], vc)
        assert np.abs(out - synth.bf16_bits_to_f32(ref)).max() <= np.abs(out).max() * 2.0 ** -8
        assert np.abs(lse - rlse).max() <= 1e-5


def test_commit_moves_what_was_there():
    rng = seed(4)
    R, D, H, ctx = 16, 64, 2, np.array([13, -1, 30], np.int32)
    table, n_blocks = tables_for(rng, [60, 16, 60], R)
    cache = random_cache(rng, 2, n_blocks, H, R, D)
    path = np.array([[0, 2, 1, 9, -1], [0, 1, 2, 3, 4], [0, 4, 5, 6, 63]], np.int32)
    new, ctx_out = kvq.commit(cache, R, D, table, ctx, np.array([3, 2, 9], np.int32), path)
    assert ctx_out.tolist() == [17, -1, 35]
    at = lambda c, b, j: kvq.raw(c, R, D, 1, kvq.row_slot(table[b], R, n_blocks, j))                            # noqa: E731
    assert np.array_equal(at(new, 0, 14), at(cache, 0, 15)) and np.array_equal(at(new, 0, 15), at(cache, 0, 14))
    assert np.array_equal(at(new, 0, 16), at(cache, 0, 22)) and np.array_equal(at(new, 2, 33), at(cache, 2, 36))
    assert np.array_equal(at(new, 2, 34), at(cache, 2, 34))          # row 93 is not in the table
    changed = {(b, j) for b, rows in ((0, 60), (2, 60)) for j in range(rows) if not np.array_equal(at(new, b, j), at(cache, b, j))}
    assert changed == {(0, 14), (0, 15), (0, 16), (2, 31), (2, 32), (2, 33)}
