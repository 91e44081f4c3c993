"""Rotary positions on the GPU against the oracle (numpy, 64 bits), bit for bit: rows turned, and rows on the way into the paged 4-bit cache."""
import numpy as np
import pytest
import torch

from gpu_util import bf16_bits, bf16_dev, dev, host
from kvq_util import bf16, seed
from oracle import kvq
from test_gpu_kvq import binding, gpu_cache

pytestmark = pytest.mark.gpu


def frequencies(P):
    return (10000.0 ** (-np.arange(P) / P)).astype(np.float32)


def rounded(x):
    """float64 -> bf16 patterns: to fp32, then to bf16, to the nearest even."""
    return bf16(x.astype(np.float32))[1]


def turned(bits, x, rows, positions, ctx, inv, axis, interleaved, scale):
    """bf16 patterns [N,H,D] after the turn, rows that are not there as they were in `bits`."""
    out = bits.copy()
    for n, b, i in rows:
        base = 0 if ctx is None else int(ctx[b])
        at = [base + (i if positions is None else int(positions[a, n])) for a in range(max(axis) + 1)]
        P = len(inv)
        new = rounded(kvq.turn(x[n], at, inv, axis, interleaved, scale))
        new[:, 2 * P:] = rounded(x[n])[:, 2 * P:]
        out[n] = new
    return out


CASES = [  # B, T, packed, Hq, Hkv, D, P, axes, interleaved, with ctx, with positions
    (1, 1, False, 1, 1, 64, 32, 1, False, False, False), (1, 60, False, 32, 8, 128, 64, 1, False, True, True), (3, 7, False, 4, 2, 64, 8, 2, True, True, False),
    (2, 9, False, 5, 5, 80, 40, 1, False, True, True), (2, 5, False, 3, 1, 256, 128, 4, False, True, True), (2, 5, False, 3, 1, 256, 24, 3, True, False, True),
    (4, 19, True, 8, 2, 128, 48, 3, False, True, True), (70, 3, True, 4, 1, 64, 32, 1, True, True, False), (3, 33, True, 9, 3, 96, 16, 2, False, True, True),
    (1, 37, True, 40, 8, 128, 64, 3, True, True, True), (5, 300, True, 20, 5, 128, 64, 1, False, True, False), (2, 3, False, 2, 2, 16, 8, 1, False, True, True)]


@pytest.mark.parametrize("case", CASES)
def test_rows_are_the_oracles_bit_for_bit(case):
    B, T, packed, Hq, Hkv, D, P, axes, interleaved, with_ctx, with_positions = case
    b, rng = binding(), seed(700 + B * T + D)
    new = rng.integers(0, T + 1, B).astype(np.int32)
    new[0] = T
    N = int(new.sum()) + 2 if packed else B * T                      # (two rows behind the last sequence)
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32) if packed else None
    ctx = rng.integers(0, 1 << 20, B).astype(np.int32) if with_ctx else None
    if ctx is not None and B > 2:
        ctx[1] = -1
    positions = rng.integers(0, 4000, (axes, N)).astype(np.int32) if with_positions else None
    inv, axis, scale = frequencies(P), [int(a) for a in rng.integers(0, axes, P)], 1.0 if P != 48 else 1.1386
    wide = rng.normal(size=(N, Hq + Hkv + 1, D)) * 2.0 ** rng.integers(-6, 7, (N, 1, 1))
    x, bits = bf16(wide)
    rows = kvq.new_rows(B, T, ctx, starts, None if packed else new)
    assert 0 < len(rows) <= N
    rope = b.Rope(dev(inv), axes=axes, pair_axis=axis, interleaved=interleaved, scale=scale)
    lead = (N,) if packed else (B, T)
    fused = bf16_dev(bits).view(lead + bits.shape[1:])
    q, k = fused[..., :Hq, :], fused[..., Hq:Hq + Hkv, :]
    room = torch.full(lead + (Hq + 3, D), 3.0, dtype=torch.bfloat16, device="cuda")
    kw = dict(positions=None if positions is None else dev(positions), ctx_lens=None if ctx is None else dev(ctx), row_starts=None if starts is None else dev(starts),
              n_new=None if packed else dev(new), T_max=T)
    q_out, k_out = b.radar_rope(q, k, rope, q_out=room[..., 1:1 + Hq, :], k_out=torch.full(k.shape, 3.0, dtype=torch.bfloat16, device="cuda"), **kw)
    scale32 = float(np.float32(scale))
    want = turned(np.full_like(bits, 0x4040), x, rows, positions, ctx, inv, axis, interleaved, scale32)
    assert np.array_equal(bf16_bits(q_out).reshape(N, Hq, D), want[:, :Hq]) and np.array_equal(bf16_bits(k_out).reshape(N, Hkv, D), want[:, Hq:Hq + Hkv])
    assert (room[..., 0, :] == 3).all() and (room[..., 1 + Hq:, :] == 3).all()
    # in place, and one of the two alone
    b.radar_rope(q, None, rope, q_out=q, **kw)
    b.radar_rope(None, k, rope, k_out=k, **kw)
    want = turned(bits, x, rows, positions, ctx, inv, axis, interleaved, scale32)
    want[:, Hq + Hkv:] = bits[:, Hq + Hkv:]
    assert np.array_equal(bf16_bits(fused).reshape(bits.shape), want)


def test_far_positions_and_values_that_are_not_finite():
    b, rng, P, D = binding(), seed(720), 64, 128
    pos = np.array([[0, 1, (1 << 20) + 7, (1 << 24) + 1, (1 << 30) - 1, (1 << 31) - 1, 12345678, 3]], np.int32)
    x, bits = bf16(rng.normal(size=(8, 3, D)))
    bits[7, 0, 5], bits[7, 1, 70], bits[7, 2, 1] = 0x7f80, 0x7fc0, 0xff80
    rope = b.Rope(dev(frequencies(P)))
    got, _ = b.radar_rope(bf16_dev(bits)[None], None, rope, positions=dev(pos))
    got = bf16_bits(got)[0]
    want = np.stack([rounded(kvq.turn(x[n], [int(pos[0, n])], frequencies(P), [0] * P)) for n in range(7)])
    assert np.array_equal(got[:7], want)
    bad = ~np.isfinite(torch.from_numpy(got[7].view(np.int16)).view(torch.bfloat16).float().numpy())
    assert bad.sum() == 6 and bad[0, [5, 69]].all() and bad[1, [6, 70]].all() and bad[2, [1, 65]].all()      # both values of a pair, and no others


def test_many_sequences_without_rows():
    """More sequences than a wavefront looks at at once, long stretches of them without a row."""
    b, rng, B, P, D = binding(), seed(721), 9000, 32, 64
    new = np.zeros(B, np.int64)
    new[[0, 5, 70, 71, 200, 4096, 4097, 8999]] = [1, 2, 1, 9, 3, 1, 5, 4]
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    N, ctx = int(starts[-1]), rng.integers(0, 5000, B).astype(np.int32)
    x, bits = bf16(rng.normal(size=(N, 2, D)))
    rope = b.Rope(dev(frequencies(P)), interleaved=True)
    got, _ = b.radar_rope(bf16_dev(bits), None, rope, ctx_lens=dev(ctx), row_starts=dev(starts), T_max=8)
    rows = kvq.new_rows(B, 8, ctx, starts)
    assert len(rows) == N - 1                                        # (the ninth row of a sequence is not there)
    want = turned(bf16_bits(got), x, rows, None, ctx, frequencies(P), [0] * P, True, 1.0)
    assert np.array_equal(bf16_bits(got), want)


@pytest.mark.parametrize("B,T,packed,Hq,H,D,R,P,axes,interleaved", [(1, 1, True, 1, 1, 64, 16, 32, 1, False), (16, 60, False, 32, 8, 128, 16, 64, 1, False),
                                                                   (3, 25, True, 4, 2, 64, 32, 8, 3, True), (2, 300, True, 10, 5, 128, 128, 24, 2, False),
                                                                   (70, 2, True, 8, 8, 128, 64, 64, 4, True), (5, 90, False, 7, 7, 64, 64, 32, 1, False)])
def test_append_is_a_turn_and_an_append(B, T, packed, Hq, H, D, R, P, axes, interleaved):
    """The bytes of the oracle, and of the two calls made one after the other; rows without a slot, and other layers, as they were."""
    b, rng = binding(), seed(740 + B + T + D)
    new = rng.integers(0, T + 1, B).astype(np.int32)
    new[B // 2] = T
    N = int(new.sum()) + 1 if packed else B * T
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32) if packed else None
    ctx = rng.integers(0, 5000, B).astype(np.int32)
    if B > 2:
        ctx[0] = -1
    positions, inv, axis = rng.integers(0, 300, (axes, N)).astype(np.int32), frequencies(P), [j % axes for j in range(P)]
    n_blocks = -(-B * T // R) + 2
    slots = rng.permutation(n_blocks * R)[:B * T].astype(np.int32).reshape(B, T)
    slots.reshape(-1)[rng.random(B * T) < 0.1] = -1
    slots[B // 2, 0] = n_blocks * R
    x, bits = bf16(rng.normal(size=(N, Hq + 2 * H, D)) * 2.0 ** rng.integers(-3, 4, (N, 1, 1)))
    lead = (N,) if packed else (B, T)
    fused = bf16_dev(bits).view(lead + bits.shape[1:])
    q, k, v = fused[..., :Hq, :], fused[..., Hq:Hq + H, :], fused[..., Hq + H:, :]
    cache = np.full((2, n_blocks, H, kvq.chunk_bytes(R, D)), 0xAA, np.uint8)
    c = gpu_cache(cache, R, D)
    rope = b.Rope(dev(inv), axes=axes, pair_axis=axis, interleaved=interleaved)
    kw = dict(positions=dev(positions), ctx_lens=dev(ctx), row_starts=None if starts is None else dev(starts), n_new=None if packed else dev(new))
    q_out = torch.full(q.shape, 3.0, dtype=torch.bfloat16, device="cuda")
    assert b.radar_kvq_append_rope(c, q, k, v, dev(slots), rope, layer=1, q_out=q_out, **kw) is q_out
    rows = kvq.new_rows(B, T, ctx, starts, None if packed else new)
    want = turned(np.full_like(bits, 0x4040), x, rows, positions, ctx, inv, axis, interleaved, 1.0)
    assert np.array_equal(bf16_bits(q_out).reshape(N, Hq, D), want[:, :Hq])
    for n, bb, i in rows:
        kk = torch.from_numpy(want[n, Hq:Hq + H].view(np.int16)).view(torch.bfloat16).double().numpy()
        kvq.put(cache, R, D, 1, int(slots[bb, i]), kk, x[n, Hq + H:])
    assert np.array_equal(host(c.data), cache)
    two = gpu_cache(np.full_like(cache, 0xAA), R, D)
    flat = np.full(N, -1, np.int32)
    for n, bb, i in rows:
        flat[n] = slots[bb, i]
    k_out = b.radar_rope(None, k, rope, T_max=T, **kw)[1]
    b.radar_kvq_append(two, k_out, v.contiguous(), dev(flat), layer=1)
    assert torch.equal(two.data, c.data)
    again = gpu_cache(np.full_like(cache, 0xAA), R, D)              # keys and values only
    assert b.radar_kvq_append_rope(again, None, k, v, dev(slots), rope, layer=1, **kw) is None
    assert torch.equal(again.data, c.data)


@pytest.mark.parametrize("D,P,interleaved", [(128, 64, False), (64, 32, True), (96, 40, False)])
def test_more_rows_than_the_caches_hold(D, P, interleaved):
    """Rows of more than 64 MB are read and stored past the caches: the same bits as in small calls, some of which are the oracle's, at once, in place and into the 4-bit cache."""
    b, rng, Hq, H, R = binding(), seed(760 + D), 16, 4, 64
    N = (64 << 20) // (D * 4 * (Hq + H)) + 77
    inv, n_some = frequencies(P), 40
    rope, ctx = b.Rope(dev(inv), interleaved=interleaved), dev(np.array([5], np.int32))
    fused = torch.randn((N, Hq + 2 * H, D), device="cuda").bfloat16()
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + H], fused[:, Hq + H:]
    starts = dev(np.array([0, N - 3], np.int32))                     # (three rows behind the last sequence)
    fresh = lambda n, h: torch.full((n, h, D), 3.0, dtype=torch.bfloat16, device="cuda")            # noqa: E731
    q_out, k_out = b.radar_rope(q, k, rope, ctx_lens=ctx, row_starts=starts, T_max=N, q_out=fresh(N, Hq), k_out=fresh(N, H))
    assert (q_out[N - 3:] == 3).all() and (k_out[N - 3:] == 3).all()
    step = 1500
    for at in range(0, N - 3, step):
        n = min(step, N - 3 - at)
        few_q, few_k = b.radar_rope(q[at:at + n][None], k[at:at + n][None], rope, ctx_lens=ctx + at)
        assert torch.equal(few_q[0], q_out[at:at + n]) and torch.equal(few_k[0], k_out[at:at + n])
    some = np.concatenate([np.arange(n_some), np.arange(N - 3 - n_some, N - 3)])
    bits = bf16_bits(fused[dev(some.astype(np.int64))])
    x = host(fused[dev(some.astype(np.int64))].double())
    want = np.stack([rounded(kvq.turn(x[j], [5 + int(n)], inv, [0] * P, interleaved)) for j, n in enumerate(some)])
    want[:, :, 2 * P:] = bits[:, :, 2 * P:]
    assert np.array_equal(bf16_bits(q_out)[some], want[:, :Hq]) and np.array_equal(bf16_bits(k_out)[some], want[:, Hq:Hq + H])
    if D in (64, 128):
        n_blocks = -(-N // R)
        slots = torch.randperm(n_blocks * R, device="cuda")[:N].int()[None]
        one, two = b.KvqCache(n_blocks, R, H, D), b.KvqCache(n_blocks, R, H, D)
        one.data.fill_(0xAA), two.data.fill_(0xAA)
        turned_q = b.radar_kvq_append_rope(one, q, k, v, slots, rope, ctx_lens=ctx, row_starts=starts, q_out=fresh(N, Hq))
        assert torch.equal(turned_q, q_out)
        b.radar_kvq_append(two, k_out[:N - 3], v[:N - 3].contiguous(), slots[0, :N - 3].contiguous())
        assert torch.equal(one.data, two.data)
    before = fused.clone()
    b.radar_rope(q, k, rope, ctx_lens=ctx, row_starts=starts, T_max=N, q_out=q, k_out=k)
    assert torch.equal(q[:N - 3], q_out[:N - 3]) and torch.equal(k[:N - 3], k_out[:N - 3])
    assert torch.equal(v, before[:, Hq + H:]) and torch.equal(fused[N - 3:], before[N - 3:])


def test_keys_that_are_not_finite_make_blocks_of_nan():
    b, rng, D, R = binding(), seed(760), 128, 16
    x, bits = bf16(rng.normal(size=(5, 6, D)))
    bits[1, 4, 3], bits[2, 5, 100], bits[3, 4, 64 + 40] = 0x7fc0, 0x7f80, 0xff80
    fused, c = bf16_dev(bits), b.KvqCache(2, R, 1, D)
    slots = torch.arange(5, dtype=torch.int32, device="cuda")[None]
    b.radar_kvq_append_rope(c, fused[None, :, :4], fused[None, :, 4:5], fused[None, :, 5:], slots, b.Rope(dev(frequencies(64))))
    k, v = (host(t.float())[0, :, 0] for t in b.radar_kvq_read(c, slots))
    nan = lambda a, n: [bool(np.isnan(a[n, 32 * z:32 * z + 32]).all()) for z in range(4)]           # noqa: E731
    assert [nan(k, n) for n in range(5)] == [[False] * 4, [True, False, True, False], [False] * 4, [False, True, False, True], [False] * 4]
    assert [nan(v, n) for n in range(5)] == [[False] * 4, [False] * 4, [False, False, False, True], [False] * 4, [False] * 4]
    assert np.isnan(k).sum() == 128 and np.isnan(v).sum() == 32


def test_no_rows():
    b = binding()
    rope, starts = b.Rope(dev(frequencies(64))), torch.zeros(3, dtype=torch.int32, device="cuda")
    x = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16, device="cuda")                      # noqa: E731
    c = b.KvqCache(2, 16, 2, 128)
    assert b.radar_rope(x(0, 4, 128), x(0, 2, 128), rope, row_starts=starts)[0].shape == (0, 4, 128)
    assert b.radar_kvq_append_rope(c, None, x(0, 2, 128), x(0, 2, 128), torch.zeros((2, 3), dtype=torch.int32, device="cuda"), rope, row_starts=starts) is None
    # rows, none of which is anybody's
    q = x(3, 4, 128) + 2
    out = b.radar_rope(q, None, rope, row_starts=starts, q_out=x(3, 4, 128) + 5)[0]
    assert (out == 5).all()


def test_a_captured_turn_with_other_lengths():
    b, rng, B, T, D, P = binding(), seed(770), 5, 40, 64, 32
    N, inv = 60, frequencies(32)
    z = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")                         # noqa: E731
    starts, ctx, slots, positions = z(B + 1), z(B), z(B, T), z(2, N)
    axis = [j % 2 for j in range(P)]
    rope = b.Rope(dev(inv), axes=2, pair_axis=axis)
    x = torch.zeros((N, 4, D), dtype=torch.bfloat16, device="cuda")
    out, c = torch.zeros((N, 2, D), dtype=torch.bfloat16, device="cuda"), b.KvqCache(16, 16, 1, D)
    call = lambda: b.radar_kvq_append_rope(c, x[:, :2], x[:, 2:3], x[:, 3:], slots, rope, positions=positions, ctx_lens=ctx, row_starts=starts, q_out=out)      # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for trial in range(4):
        new = rng.multinomial(30 + 10 * trial, np.ones(B) / B)
        hs, hc = np.concatenate([[0], np.cumsum(new)]).astype(np.int32), rng.integers(0, 100, B).astype(np.int32)
        hc[trial] = -1
        hp, hx = rng.integers(0, 50, (2, N)).astype(np.int32), bf16(rng.normal(size=(N, 4, D)))
        for t, y in ((starts, dev(hs)), (ctx, dev(hc)), (positions, dev(hp)), (slots, dev(rng.permutation(256)[:B * T].reshape(B, T).astype(np.int32))), (x, bf16_dev(hx[1]))):
            t.copy_(y)
        out.fill_(3.0)
        c.data.fill_(0xAA)
        g.replay()
        torch.cuda.synchronize()
        want = turned(np.full_like(hx[1], 0x4040), hx[0], kvq.new_rows(B, T, hc, hs), hp, hc, inv, axis, False, 1.0)
        assert np.array_equal(bf16_bits(out), want[:, :2])
        kept = c.data.clone()
        c.data.fill_(0xAA)
        call()
        assert torch.equal(c.data, kept)
