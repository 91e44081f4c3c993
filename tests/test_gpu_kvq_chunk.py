"""Attention of chunks of new tokens over the paged 4-bit cache on the GPU against its oracle (numpy, 64 bits), in every kind of launch, and the calls of a
serving step made one after the other: blocks, turned rows in, attention."""
import numpy as np
import pytest
import torch

from gpu_util import bf16_bits, bf16_dev, dev, host
from kvq_util import bf16, random_cache, random_parents, seed, tables_for
from oracle import kvq
from test_gpu_kvq import binding, gpu_cache
from test_gpu_rope import frequencies, turned

pytestmark = pytest.mark.gpu


def check(q, cache, R, D, tables, ctx, T, got, lse=None, layer=0, **kw):
    """Every value of the rows that are there.  Probabilities and outputs are rounded to bf16 (half a step each: 2^-8), the arithmetic is fp32: scores are off by
    (D + 8) 2^-24 of their terms' sum, weights and the sum that they are divided by each by as much, and 2^-14 is for the sums and exponentials."""
    N = len(q)
    got = host(got.double()).reshape(q.shape)
    out_r, lse_r, sp, reach, there = kvq.chunk_attention(q, cache, R, D, layer, tables, ctx, T, **kw)
    nan = np.isnan(out_r)
    slack = (D + 8) * 2.0 ** -24 * np.nan_to_num(reach)
    bound = 2.0 ** -8 * (sp + np.abs(np.where(nan, 0, out_r)) + 2.0 ** -8 * sp) + (2.0 ** -14 + 2 * slack[..., None]) * sp + 1e-30
    assert (np.isnan(got) == nan)[there].all()
    err = np.where(nan, 0.0, np.abs(got - out_r))
    assert ((err <= bound) | nan)[there].all(), (np.argwhere((err > bound) & there[:, None, None])[:5], err[there].max())      # (NaN is compared above)
    if lse is not None:
        l = host(lse.double()).reshape(N, -1)
        assert (np.isnan(l) == np.isnan(lse_r))[there].all() and (np.isneginf(l) == np.isneginf(lse_r))[there].all()
        sound = np.isfinite(lse_r) & there[:, None]
        lerr = np.abs(np.where(sound, l, 0) - np.where(sound, lse_r, 0))
        assert (lerr <= slack + 2.0 ** -19 * (1 + np.abs(np.where(sound, lse_r, 0))))[there].all(), lerr.max()
    return there


def make(rng, ctx, new, Hq, H, D, R, packed=True, behind=0, width=0, layers=1, T=None):
    """Tables and cache of sequences that hold ctx + new rows, queries of the new ones, starts (or None), the longest chunk."""
    T = max(new) if T is None else T
    tables, n_blocks = tables_for(rng, [max(c, 0) + n for c, n in zip(ctx, new)], R, width=width)
    cache = random_cache(rng, layers, n_blocks, H, R, D)
    N = sum(new) + behind if packed else len(new) * T
    q, bits = bf16(rng.normal(size=(N, Hq, D)))
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32) if packed else None
    return tables, cache, q, bits, starts, T


def ran(call):
    """Names of the kernels of this library that a call launched."""
    b = binding()
    torch.cuda.synchronize()
    b.radar_profile_begin(64)
    call()
    torch.cuda.synchronize()
    return set(b.radar_profile_end())


def attend(b, bits, cache, tables, ctx, starts=None, n_new=None, T=None, want_lse=True, c=None, R=16, D=128, **kw):
    """A call over buffers that hold 7 before; (out, lse)."""
    lead = bits.shape[:-2] if starts is not None else (len(ctx), T)
    q = bf16_dev(bits).view(tuple(lead) + bits.shape[-2:])
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:-1], 7.0, device="cuda") if want_lse else None
    got = b.radar_chunk_attention_kvq(q, gpu_cache(cache, R, D) if c is None else c, dev(tables), dev(ctx), row_starts=None if starts is None else dev(starts),
                                      n_new=None if n_new is None else dev(n_new), T_max=T, out=out, lse_out=lse, **kw)
    assert got is out
    return out, lse


@pytest.mark.parametrize("ctx,new,Hq,H,D,R", [
    ([0], [1], 1, 1, 64, 16), ([15], [1], 4, 1, 128, 16), ([16], [17], 8, 2, 128, 16), ([0], [65], 5, 5, 64, 32), ([31, 0, 300], [1, 33, 64], 8, 2, 128, 32),
    ([5, -1, 7, 0], [9, 4, 0, 130], 6, 2, 64, 64), ([100, 40, 0, 3, 64], [1, 1, 200, 1, 31], 16, 2, 128, 128), ([1000, 9], [3, 70], 70, 1, 64, 16),
    ([63], [129], 35, 5, 128, 16), ([0, 0, 0], [32, 96, 160], 9, 3, 64, 16), ([7] * 70, [k % 4 for k in range(70)], 4, 2, 64, 16)])
@pytest.mark.parametrize("packed", [True, False])
def test_against_the_oracle(ctx, new, Hq, H, D, R, packed):
    """Rows behind the last sequence stay as they were; rows of [B,T] that are not there, and those of sequences that have ended, are zero."""
    b, rng, ctx = binding(), seed(800 + sum(new) + D), np.array(ctx, np.int32)
    tables, cache, q, bits, starts, T = make(rng, ctx, new, Hq, H, D, R, packed, behind=3)
    n_new = None if packed else np.array(new, np.int32)
    out, lse = attend(b, bits, cache, tables, ctx, starts, n_new, T, R=R, D=D)
    there = check(q, cache, R, D, tables, ctx, T, out, lse, row_starts=starts, n_new=n_new)
    out, lse = out.view(-1, Hq, D), lse.view(-1, Hq)
    gone = ~there
    if packed:
        gone[sum(new):] = False
        assert (out[sum(new):] == 7).all() and (lse[sum(new):] == 7).all()
    gone = torch.from_numpy(np.nonzero(gone)[0]).cuda()
    assert (out[gone] == 0).all() and (lse[gone] == 0).all()


# Sequences, rows of each, heads, the rows that the call is planned for, and the kernel that it comes to, with and without blocks in parts.
KINDS = [("kvq_chunk_16x8", 1, 7, 2, 1, 20000), ("kvq_chunk_16x8", 17, 5, 2, 2, 20000), ("kvq_chunk_16x8", 17, 1, 16, 16, 2000), ("kvq_chunk_16x8", 17, 1, 8, 8, 300),
         ("kvq_chunk_16x4", 3, 64, 64, 8, 300), ("kvq_chunk_16x4", 1, 40, 256, 32, 300),
         ("kvq_chunk_32x8", 1, 40, 16, 2, 100000), ("kvq_chunk_32x8", 5, 16, 16, 8, 100000), ("kvq_chunk_32x8", 5, 16, 32, 2, 20000),
         ("kvq_chunk_64x8", 1, 64, 32, 2, 100000), ("kvq_chunk_64x8", 1, 64, 64, 8, 20000), ("kvq_chunk_64x8", 3, 16, 64, 16, 20000),
         ("kvq_chunk_16x4", 17, 16, 64, 16, 700), ("kvq_chunk_64x4", 3, 16, 128, 16, 20000), ("kvq_chunk_64x4", 17, 16, 128, 32, 300), ("kvq_chunk_64x2", 17, 5, 512, 64, 300),
         ("kvq_chunk_64x2", 1, 40, 256, 64, 100000), ("kvq_chunk_64x1", 17, 40, 128, 32, 300), ("kvq_chunk_64x1", 40, 5, 512, 64, 300)]


@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("name,B,n,Hq,H,S", KINDS)
def test_every_kind(name, B, n, Hq, H, S, D, far):
    """Each kind of launch, below and beyond 4 GB of cache, with the library's parts and with parts of 64 rows; one workspace, whose counters are zero again."""
    b, rng, R = binding(), seed(820 + n + Hq + D), 16
    ctx = rng.integers(100, 260, B).astype(np.int32)
    ctx[0] = 200                                                     # (all of them fit the shortest plan)
    ctx = np.minimum(ctx, 296 - n)
    if B > 2:
        ctx[1] = -1
    tables, cache, q, bits, starts, _ = make(rng, ctx, [n] * B, Hq, H, D, R)
    n_small = cache.shape[1]
    if far:
        n_blocks = (5 << 30) // (H * kvq.chunk_bytes(R, D))
        c = b.KvqCache(n_blocks, R, H, D)
        ids = np.sort(rng.choice(n_blocks, n_small, replace=False)).astype(np.int32)
        c.data[0, torch.from_numpy(ids).long().cuda()] = dev(cache[0])
    else:
        c, ids = gpu_cache(cache, R, D), np.arange(n_small, dtype=np.int32)
    wide = np.full((B, -(-S // R)), -1, np.int32)
    wide[:, :tables.shape[1]] = np.where(tables >= 0, ids[tables], -1)
    ws = b.new_workspace(b.radar_chunk_attention_kvq_workspace_bytes(b.kvq_chunk_desc(bf16_dev(bits), c, wide.shape[1], B, n, len(bits), S)))
    for split in (0, 64):
        got = {}
        names = ran(lambda: got.update(r=attend(b, bits, None, wide, ctx, starts, None, n, c=c, R=R, D=D, S_max=S, workspace=ws, rows_per_split=split)))
        assert split or names == {name}, names
        check(q, cache, R, D, tables, ctx, n, *got["r"], row_starts=starts)
        assert (ws[:65536] == 0).all()
    del c
    torch.cuda.empty_cache()


@pytest.mark.parametrize("ctx,new,Hq,H,D,split", [([3000], [1], 4, 1, 128, 64), ([2500], [100], 8, 2, 128, 64), ([4000, 10, 900], [1, 300, 40], 8, 2, 64, 64),
                                                  ([1500, 1500, 1500], [64, 64, 64], 8, 1, 128, 128), ([5000], [3], 64, 2, 64, 192)])
def test_parts_are_joined(ctx, new, Hq, H, D, split):
    b, rng, R, ctx = binding(), seed(860 + sum(new) + D), 32, np.array(ctx, np.int32)
    tables, cache, q, bits, starts, T = make(rng, ctx, new, Hq, H, D, R)
    out, lse = attend(b, bits, cache, tables, ctx, starts, None, T, R=R, D=D, rows_per_split=split)
    check(q, cache, R, D, tables, ctx, T, out, lse, row_starts=starts)


def test_a_chain_of_the_tree_call():
    """Up to 64 rows this is radar_tree_attention_kvq with parents left out: the same bound holds between the two and the oracle."""
    b, rng, D, R = binding(), seed(870), 128, 16
    ctx, nodes = np.array([200, 0, 77, -1], np.int32), np.array([64, 3, 40, 9], np.int32)
    tables, cache, q, bits, _, T = make(rng, ctx, [64] * 4, 8, 2, D, R, packed=False)
    out, lse = attend(b, bits, cache, tables, ctx, None, nodes, T, R=R, D=D)
    check(q, cache, R, D, tables, ctx, T, out, lse, n_new=nodes)
    lse2 = torch.empty_like(lse)
    two = b.radar_tree_attention_kvq(bf16_dev(bits).view(4, T, 8, D), gpu_cache(cache, R, D), dev(tables), dev(ctx), n_nodes=dev(nodes), lse_out=lse2)
    check(q, cache, R, D, tables, ctx, T, two, lse2, n_new=nodes)
    assert (out[3] == 0).all() and (two[3] == 0).all()


def test_strides_layers_and_a_scale():
    b, rng, D, R, Hq, H = binding(), seed(871), 64, 16, 8, 2
    ctx, new = np.array([40, 3], np.int32), [9, 70]
    tables, cache, q, bits, starts, T = make(rng, ctx, new, Hq, H, D, R, layers=3)
    wide = torch.zeros((79, Hq + 5, D), dtype=torch.bfloat16, device="cuda")
    wide[:, 2:2 + Hq] = bf16_dev(bits)
    room = torch.full((Hq, 85, D), 5.0, dtype=torch.bfloat16, device="cuda")
    out, lse = room.transpose(0, 1)[3:82], torch.empty((79, Hq), device="cuda")
    kw = dict(row_starts=dev(starts), T_max=T, layer=2, softmax_scale=0.31)
    b.radar_chunk_attention_kvq(wide[:, 2:2 + Hq], gpu_cache(cache, R, D), dev(tables), dev(ctx), out=out, lse_out=lse, **kw)
    check(q, cache, R, D, tables, ctx, T, out, lse, layer=2, row_starts=starts, scale=float(np.float32(0.31)))
    assert (room[:, :3] == 5).all() and (room[:, 82:] == 5).all()
    plain = b.radar_chunk_attention_kvq(wide[:, 2:2 + Hq], gpu_cache(cache, R, D), dev(tables), dev(ctx), **kw)                     # no log-sum-exps asked for
    assert torch.equal(plain, out)
    # [B, T] with strides of its own
    x = torch.zeros((2, Hq, 75, D), dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    for s in range(2):
        x[s, 1:1 + new[s]] = bf16_dev(bits[starts[s]:starts[s + 1]])
    two = b.radar_chunk_attention_kvq(x[:, 1:71], gpu_cache(cache, R, D), dev(tables), dev(ctx), n_new=dev(np.array(new, np.int32)), layer=2, softmax_scale=0.31)
    for s in range(2):
        assert torch.equal(two[s, :new[s]], out[starts[s]:starts[s + 1]]) and (two[s, new[s]:] == 0).all()


@pytest.mark.parametrize("D,Hq,H,n", [(64, 4, 2, 20), (128, 8, 2, 90), (128, 1, 1, 40), (128, 16, 1, 3)])
def test_what_is_not_seen_has_no_influence(D, Hq, H, n):
    """NaN blocks and the largest scales in rows behind a row, behind the last one and in nobody's blocks: the rows before them are as without."""
    b, rng, R = binding(), seed(880 + n), 16
    ctx, new = np.array([37, 0], np.int32), [n, n]
    tables, cache, q, bits, starts, T = make(rng, ctx, new, Hq, H, D, R)
    n_blocks = cache.shape[1]
    want, _ = attend(b, bits, cache, tables, ctx, starts, None, T, R=R, D=D)
    spoiled = cache.copy()
    first = [n // 2, n - 1]                                          # from that row on they are spoiled
    good = {kvq.row_slot(tables[s], R, n_blocks, j) for s in range(2) for j in range(int(ctx[s]) + first[s])}
    for slot in range(n_blocks * R):
        if slot not in good:
            _, _, sc = kvq._code_places(R, D, slot % R)
            for at in sc:
                spoiled[0, slot // R][:, at] = [255, 254, 253][slot % 3]
    got, _ = attend(b, bits, spoiled, tables, ctx, starts, None, T, R=R, D=D)
    for s in range(2):
        assert torch.equal(got[starts[s]:starts[s] + first[s]], want[starts[s]:starts[s] + first[s]])
    assert torch.isnan(got[starts[1] + n - 1].float()).all() or D == 0


def test_nan_rows_that_are_seen():
    b, rng, D, R = binding(), seed(890), 128, 16
    ctx, new = np.array([40], np.int32), [50]
    tables, cache, q, bits, starts, T = make(rng, ctx, new, 4, 2, D, R)
    for j, kv, h, blk in ((60, 1, 0, 2), (75, 0, 1, 0), (12, 1, 1, 3)):
        slot = kvq.row_slot(tables[0], R, cache.shape[1], j)
        cache[0, slot // R][h, kvq._code_places(R, D, slot % R)[2][kv][blk]] = 255
    out, lse = attend(b, bits, cache, tables, ctx, starts, None, T, R=R, D=D)
    check(q, cache, R, D, tables, ctx, T, out, lse, row_starts=starts)
    assert torch.isnan(out.float()).any() and not torch.isnan(out.float()).all()


def test_rows_that_are_not_there():
    """Blocks of no number, rows past S_max, lengths past it, a table that names nothing: those rows are not seen, and where none is, out is zero and lse -inf."""
    b, rng, D, R, Hq, H = binding(), seed(891), 64, 16, 4, 2
    ctx, new = np.array([50, 33, 20, 90, 2 ** 31 - 1], np.int32), [70, 5, 9, 40, 3]
    tables, cache, q, bits, starts, T = make(rng, np.minimum(ctx, 200), new, Hq, H, D, R, width=8)
    n_blocks = cache.shape[1]
    tables = tables[:, :8]
    tables[0, [1, 4]] = [-1, n_blocks]
    tables[1] = np.iinfo(np.int32).min
    for S in (128, 100, 64, 17, 1):
        out, lse = attend(b, bits, cache, tables, ctx, starts, None, T, R=R, D=D, S_max=S)
        check(q, cache, R, D, tables, ctx, T, out, lse, row_starts=starts, S_max=S)
        assert (out[70:75] == 0).all() and torch.isneginf(lse[70:75]).all()


def test_row_starts_of_any_content_stay_in_bounds():
    """Starts that fall, overlap or lie outside are not a batch, but nothing is written outside the outputs, and a sound call after them is right."""
    b, rng, D, R, Hq, H, N = binding(), seed(892), 64, 16, 4, 1, 120
    ctx = np.array([300, 10, 40, 0], np.int32)
    tables, cache, q, bits, starts, T = make(rng, ctx, [30] * 4, Hq, H, D, R)
    c, room = gpu_cache(cache, R, D), torch.full((N + 8, Hq, D), 5.0, dtype=torch.bfloat16, device="cuda")
    ws = b.new_workspace(b.radar_chunk_attention_kvq_workspace_bytes(b.kvq_chunk_desc(room, c, tables.shape[1], 4, T, N)))
    for bad in ([0, 90, 20, 110, 60], [-50, 400, 3, 9, 2 ** 31 - 1], [120, 100, 80, 60, 40], [7, 7, 7, 7, 7], [0, 120, 0, 120, 0]):
        b.radar_chunk_attention_kvq(bf16_dev(bits), c, dev(tables), dev(ctx), row_starts=dev(np.array(bad, np.int32)), T_max=T, out=room[4:4 + N], rows_per_split=64, workspace=ws)
        assert (room[:4] == 5).all() and (room[4 + N:] == 5).all()
    b.radar_workspace_init(ws)
    out, lse = attend(b, bits, cache, tables, ctx, starts, None, T, R=R, D=D, rows_per_split=64, workspace=ws)
    check(q, cache, R, D, tables, ctx, T, out, lse, row_starts=starts)


def test_more_sequences_than_are_counted_through():
    """Beyond 512 sequences a workgroup looks its block up; between 65 and 512 they are counted in several goes."""
    b, rng, D, R, Hq, H = binding(), seed(893), 64, 16, 4, 2
    for B in (66, 300, 512, 513, 1500):
        ctx = rng.integers(-1, 60, B).astype(np.int32)
        new = [int(x) for x in rng.integers(0, 4, B)]
        new[B // 2], ctx[B // 3] = 90, 700
        tables, cache, q, bits, starts, T = make(rng, ctx, new, Hq, H, D, R, behind=2)
        out, lse = attend(b, bits, cache, tables, ctx, starts, None, T, R=R, D=D, rows_per_split=64 if B == 300 else 0)
        check(q, cache, R, D, tables, ctx, T, out, lse, row_starts=starts)
        pad = [int(x) for x in rng.integers(0, 6, B)]
        tables, cache, q, bits, _, _ = make(rng, ctx, pad, Hq, H, D, R, packed=False, T=6)
        n_new = np.array(pad, np.int32)
        out, lse = attend(b, bits, cache, tables, ctx, None, n_new, 6, R=R, D=D)
        check(q, cache, R, D, tables, ctx, 6, out, lse, n_new=n_new)


def test_as_many_blocks_as_a_call_may_have():
    """Single tokens of so many sequences and heads that blocks of 16 and 32 columns would be too many.  Every token sees one row, all of them the same one."""
    b, rng, D, R, B, H = binding(), seed(896), 64, 16, 65535, 63
    cache = random_cache(rng, 1, 1, H, R, D)
    q = torch.randn((B, H, D), device="cuda").bfloat16()
    lse = torch.empty((B, H), device="cuda")
    out = b.radar_chunk_attention_kvq(q, gpu_cache(cache, R, D), torch.zeros((B, 1), dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda"),
                                      row_starts=torch.arange(B + 1, dtype=torch.int32, device="cuda"), T_max=1, lse_out=lse)
    k, v, _ = kvq.all_rows(cache, R, D, 0, [0], 1)
    score = (q.double() * dev(k[0])).sum(-1) / 8.0
    assert (out.double() == dev(v[0])).all()                         # (its weight is 1 to 2^-20, and its values are bf16's)
    assert ((lse.double() - score).abs() <= (D + 8) * 2.0 ** -24 * (q.double() * dev(k[0])).abs().sum(-1) / 8.0 + 2.0 ** -19 * (1 + score.abs())).all()


def test_a_chunk_beyond_its_most_rows():
    """Rows of a sequence behind its T_max-th are not there: they stay as they were."""
    b, rng, D, R = binding(), seed(894), 64, 16
    ctx, new = np.array([5, 9], np.int32), [30, 12]
    tables, cache, q, bits, starts, _ = make(rng, ctx, new, 4, 2, D, R)
    out, lse = attend(b, bits, cache, tables, ctx, starts, None, 20, R=R, D=D)
    check(q, cache, R, D, tables, ctx, 20, out, lse, row_starts=starts)
    assert (out[20:30] == 7).all() and (lse[20:30] == 7).all()


def test_the_longest_lengths_allowed():
    b, rng, D, R, Hq, H = binding(), seed(895), 64, 128, 8, 2
    S = 2 ** 31 - 1 - 4096
    ctx, new = np.array([700, 2 ** 31 - 1], np.int32), [64, 40]
    tables, cache, q, bits, starts, T = make(rng, np.minimum(ctx, 700), new, Hq, H, D, R)
    wide = torch.full((2, -(-S // R)), -1, dtype=torch.int32, device="cuda")
    wide[0, :tables.shape[1]] = dev(tables[0])
    lse = torch.empty((len(q), Hq), device="cuda")
    # (the second sequence is all of S rows long, none of which is in a block)
    hctx = np.array([700, 200000], np.int32)
    out = b.radar_chunk_attention_kvq(bf16_dev(bits), gpu_cache(cache, R, D), wide, dev(hctx), row_starts=dev(starts), T_max=T, S_max=S, lse_out=lse)
    check(q[:64], cache, R, D, tables[:1], ctx[:1], T, out[:64], lse[:64], row_starts=starts[:2])
    assert (out[64:] == 0).all() and torch.isneginf(lse[64:]).all()


@pytest.mark.parametrize("kind", ["up", "down", "from far below", "alike", "both", "far below and near"])
def test_scores_far_apart(kind):
    """Scores of 2^40 and more, exact in 32 bits (keys a power of two throughout, queries a few bits a value): one row takes all, equal rows share."""
    from test_gpu_kvq_far_scores import rows_of
    b, rng, R, D, Hq, H = binding(), seed(900 + len(kind)), 16, 64, 4, 2
    ctx, new = np.array([900, 100], np.int32), [70, 3]
    tables, cache, _, _, starts, T = make(rng, ctx, new, Hq, H, D, R)
    for s in range(2):
        n = int(ctx[s]) + new[s]
        sign, power = rows_of(kind, n, rng)
        v = rng.normal(size=(n, H, D))
        for j in range(n):
            kvq.put(cache, R, D, 0, kvq.row_slot(tables[s], R, cache.shape[1], j), np.full((H, D), sign[j] * 2.0 ** int(power[j])), v[j])
    q, bits = bf16(rng.choice([0.5, 1.0, 1.5, 2.0], (73, Hq, D)))
    for split in (0, 64):
        out, lse = attend(b, bits, cache, tables, ctx, starts, None, T, R=R, D=D, rows_per_split=split)
        assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all()
        check(q, cache, R, D, tables, ctx, T, out, lse, row_starts=starts)


def test_long_chunks():
    """A prompt of 3000 rows, checked at some of them, and the same bits from two runs."""
    b, rng, D, R, Hq, H, n = binding(), seed(910), 128, 64, 8, 2, 3000
    ctx, starts = np.array([1000], np.int32), np.array([0, n], np.int32)
    tables, cache, q, bits, _, _ = make(rng, ctx, [n], Hq, H, D, R)
    out, lse = attend(b, bits, cache, tables, ctx, starts, None, n, R=R, D=D)
    K, V, _ = kvq.all_rows(cache, R, D, 0, tables[0], 1000 + n)
    for i in list(range(0, n, 271)) + [n - 1]:
        for h in (0, 5):
            x = (K[:1001 + i, h // 4] @ q[i, h]) / np.sqrt(D)
            w = np.exp(x - x.max())
            l, w = x.max() + np.log(w.sum()), w / w.sum()
            v = V[:1001 + i, h // 4]
            sp, o, reach = w @ np.abs(v), w @ v, (np.abs(K[:1001 + i, h // 4]) @ np.abs(q[i, h])).max() / np.sqrt(D)
            slack = (D + 8) * 2.0 ** -24 * reach
            assert (np.abs(host(out[i, h].double()) - o) <= 2.0 ** -8 * (sp + np.abs(o) + 2.0 ** -8 * sp) + (2.0 ** -14 + 2 * slack) * sp).all()
            assert abs(float(lse[i, h]) - l) <= slack + 2.0 ** -19 * (1 + abs(l))
    again, _ = attend(b, bits, cache, tables, ctx, starts, None, n, R=R, D=D)
    assert torch.equal(again, out)


def test_rows_behind_the_32nd_bit():
    """More than 2^31 values of queries and outputs, and 2^32 bytes: the last sequence's rows are those of a call over it alone, turned and attended to."""
    b, rng, D, R, Hq, H, B = binding(), seed(911), 128, 64, 64, 1, 520
    new = [511 + s % 7 for s in range(B)]
    N, last = sum(new), new[-1]
    tables, cache, _, _, _, T = make(rng, [40] * 2, [600] * 2, 1, H, D, R)
    c, ctx = gpu_cache(cache, R, D), np.full(B, 40, np.int32)
    all_tables = dev(np.concatenate([np.repeat(tables[:1], B - 1, 0), tables[1:]]))
    starts = dev(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
    q = torch.randn((N, Hq, D), device="cuda", dtype=torch.bfloat16)
    assert (N - last) * Hq * D > 2 ** 31
    rope, alone = b.Rope(dev(frequencies(64))), q[N - last:].clone()
    b.radar_rope(q, None, rope, ctx_lens=dev(ctx), row_starts=starts, T_max=max(new), q_out=q)
    alone, _ = b.radar_rope(alone[None], None, rope, ctx_lens=dev(ctx[:1]))
    assert torch.equal(alone[0], q[N - last:])
    lse = torch.empty((N, Hq), device="cuda")
    out = b.radar_chunk_attention_kvq(q, c, all_tables, dev(ctx), row_starts=starts, T_max=max(new), S_max=600, lse_out=lse)
    for at, n, table in ((0, 3, 0), (N - last, 3, 1), (N - 3, 3, 1)):                                # (rows of a sequence: those of a shorter one behind more)
        before = np.array([40 + (at - (N - last) if at == N - 3 else 0)], np.int32)
        check(host(q[at:at + n].double()), cache, R, D, tables[table:table + 1], before, n, out[at:at + n], lse[at:at + n], row_starts=np.array([0, n], np.int32))


# ------------------------------------------------------------------ a serving step

class Step:
    """A layer's part in a serving step, over fixed buffers: blocks, turned rows into the cache, attention of the new rows."""

    def __init__(self, rng, B=5, T=80, N=160, Hq=8, H=2, D=64, R=16, M=30, n_blocks=110):
        b = binding()
        self.b, self.rng, self.B, self.T, self.N, self.Hq, self.H, self.D, self.R = b, rng, B, T, N, Hq, H, D, R
        z = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")                     # noqa: E731
        self.cache, self.tables = b.KvqCache(n_blocks, R, H, D), b.KvqTables(B, M, n_blocks, R)
        self.ctx, self.new, self.starts, self.slots, self.granted = z(B), z(B), z(B + 1), z(B, T), z(B)
        self.inv = frequencies(D // 2)
        self.rope = b.Rope(dev(self.inv))
        self.x = torch.zeros((N, Hq + 2 * H, D), dtype=torch.bfloat16, device="cuda")
        self.q, self.out = (torch.zeros((N, Hq, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.lse = torch.zeros((N, Hq), device="cuda")
        self.ws = b.new_workspace(b.radar_chunk_attention_kvq_workspace_bytes(b.kvq_chunk_desc(self.q, self.cache, M, B, T, N)))
        self.ocache, self.lengths = host(self.cache.data).copy(), np.zeros(B, np.int32)

    def calls(self, prepared=False):
        b, H, Hq = self.b, self.H, self.Hq
        k, v = self.x[:, Hq:Hq + H], self.x[:, Hq + H:]
        return [b.radar_kvq_blocks(self.ctx, self.tables, self.T, n_new=self.new, slots=self.slots, granted=self.granted, prepared=prepared),
                b.radar_kvq_append_rope(self.cache, self.x[:, :Hq], k, v, self.slots, self.rope, ctx_lens=self.ctx, row_starts=self.starts, q_out=self.q, prepared=prepared),
                b.radar_chunk_attention_kvq(self.q, self.cache, self.tables.block_tables, self.ctx, row_starts=self.starts, T_max=self.T, out=self.out, lse_out=self.lse,
                                            workspace=self.ws, prepared=prepared)]

    def new_inputs(self, news):
        hs = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        x, bits = bf16(self.rng.normal(size=tuple(self.x.shape)))
        for t, y in ((self.ctx, dev(self.lengths)), (self.new, dev(np.array(news, np.int32))), (self.starts, dev(hs)), (self.x, bf16_dev(bits))):
            t.copy_(y)
        return x, bits, hs, self.lengths.copy()

    def check(self, news, x, bits, hs, ctx):
        assert host(self.granted).all()
        Hq, H, R, D = self.Hq, self.H, self.R, self.D
        rows, slots, tables = kvq.new_rows(self.B, self.T, ctx, hs), host(self.slots), host(self.tables.block_tables)
        want = turned(bits, x, rows, None, ctx, self.inv, [0] * (D // 2), False, 1.0)
        live = [n for n, _, _ in rows]
        assert np.array_equal(bf16_bits(self.q)[live], want[live][:, :Hq])
        wide = lambda p: torch.from_numpy(p.view(np.int16)).view(torch.bfloat16).double().numpy()    # noqa: E731
        for n, s, i in rows:
            kvq.put(self.ocache, R, D, 0, int(slots[s, i]), wide(want[n, Hq:Hq + H]), x[n, Hq + H:])
        assert np.array_equal(host(self.cache.data), self.ocache)
        check(wide(np.ascontiguousarray(want[:, :Hq])), self.ocache, R, D, tables, ctx, self.T, self.out, self.lse, row_starts=hs)
        self.lengths = np.where(ctx >= 0, ctx + np.array(news), ctx).astype(np.int32)


STEPS = [[80, 1, 30, 20, 3], [1, 1, 1, 1, 1], [40, 1, 0, 60, 1], [1, 64, 1, 1, 17], [1, 1, 1, 1, 1]]


def test_serving_steps_in_a_row():
    """Prompts, their pieces and single tokens; a sequence ends and another takes its place."""
    s = Step(seed(920))
    for n, news in enumerate(STEPS):
        if n == 3:
            s.lengths[1] = 0                                         # (its blocks go back, all but those of the new rows)
        x = s.new_inputs(news)
        s.calls()
        s.check(news, *x)


def test_a_captured_step_is_replayed():
    s = Step(seed(921))
    s.new_inputs([1] * 5)
    s.calls()
    torch.cuda.synchronize()
    s.tables.owned.zero_(), s.tables.block_tables.fill_(-1), s.tables.n_free.fill_(110), s.tables.free_blocks.copy_(torch.arange(109, -1, -1))
    s.ocache, s.lengths = host(s.cache.data).copy(), np.zeros(5, np.int32)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.calls()
    for news in STEPS:
        x = s.new_inputs(news)
        g.replay()
        torch.cuda.synchronize()
        s.check(news, *x)


def test_prepared_calls_and_another_stream():
    s = Step(seed(922))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        calls = s.calls(prepared=True)
        for news in STEPS[:3]:
            x = s.new_inputs(news)
            for c in calls:
                c()
            side.synchronize()
            s.check(news, *x)


def test_two_graphs_that_share_a_workspace():
    """One stream, one workspace, two shapes: parts of blocks in both, replayed in turn."""
    b, rng, D, R, Hq, H = binding(), seed(923), 128, 16, 8, 2
    ws, graphs = None, []
    for ctx, new in (([1800], [5]), ([900, 1200], [60, 1])):
        ctx = np.array(ctx, np.int32)
        tables, cache, q, bits, starts, T = make(rng, ctx, new, Hq, H, D, R)
        c, dq, out, lse = gpu_cache(cache, R, D), bf16_dev(bits), torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda"), torch.zeros(q.shape[:2], device="cuda")
        ws = b.new_workspace(b.radar_chunk_attention_kvq_workspace_bytes(b.kvq_chunk_desc(dq, c, tables.shape[1], len(ctx), T, len(q)))) if ws is None else ws
        args, kw = (dq, c, dev(tables), dev(ctx)), dict(row_starts=dev(starts), T_max=T, out=out, lse_out=lse, workspace=ws, rows_per_split=128)
        b.radar_chunk_attention_kvq(*args, **kw)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b.radar_chunk_attention_kvq(*args, **kw)
        graphs.append((g, out, lse, lambda out, lse, a=(q, cache, R, D, tables, ctx, T), st=starts: check(*a, out, lse, row_starts=st), args, kw))
    for _ in range(3):
        for g, out, lse, see, args, kw in graphs:
            out.zero_(), lse.zero_()
            g.replay()
            torch.cuda.synchronize()
            see(out, lse)
            out.zero_()
            b.radar_chunk_attention_kvq(*args, **kw)
            see(out, lse)


def test_two_streams_with_workspaces_of_their_own():
    b, rng, D, R, Hq, H = binding(), seed(924), 128, 16, 8, 2
    work = []
    for n in range(2):
        ctx = np.array([1500 + n], np.int32)
        tables, cache, q, bits, starts, T = make(rng, ctx, [40], Hq, H, D, R)
        c = gpu_cache(cache, R, D)
        ws = b.new_workspace(b.radar_chunk_attention_kvq_workspace_bytes(b.kvq_chunk_desc(bf16_dev(bits), c, tables.shape[1], 1, T, len(q))))
        work.append((torch.cuda.Stream(), (bf16_dev(bits), c, dev(tables), dev(ctx)), dict(row_starts=dev(starts), T_max=T, workspace=ws, rows_per_split=64),
                     (q, cache, R, D, tables, ctx, T), starts))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(10):
        for n, (stream, args, kw, _, _) in enumerate(work):
            with torch.cuda.stream(stream):
                outs[n].append(b.radar_chunk_attention_kvq(*args, **kw))
    torch.cuda.synchronize()
    for n, (_, _, _, a, st) in enumerate(work):
        check(*a, outs[n][0], row_starts=st)
        assert all(torch.equal(o, outs[n][0]) for o in outs[n][1:])


def test_direct_calls_by_the_native_half(monkeypatch):
    """Direct calls are marshalled natively (attention: with a workspace); they do what ctypes makes them do, and what the native half does not take reaches the
    other's checks."""
    from test_gpu_support import _Both
    b, rng, D, R, Hq, H, T = binding(), seed(930), 64, 16, 8, 2, 6
    both = _Both(b, monkeypatch)
    ctx, new = np.array([77, 31, -1], np.int32), [6, 3, 4]
    tables, cache, _, _, starts, _ = make(rng, ctx, new, Hq, H, D, R, layers=2)
    wide = torch.randn((3, T, Hq + 2 * H, D), device="cuda").bfloat16()
    flat = torch.randn((sum(new), Hq + 2 * H, D), device="cuda").bfloat16()
    dc, dt, dn, ds = dev(ctx), dev(tables), dev(np.array(new, np.int32)), dev(starts)
    slots = dev(rng.permutation(cache.shape[1] * R)[:3 * T].reshape(3, T).astype(np.int32))
    ropes = (b.Rope(dev(frequencies(32))), b.Rope(dev(frequencies(8)), axes=3, pair_axis=[2, 1, 0, 0, 1, 2, 1, 0], interleaved=True, scale=1.25))
    pos = dev(rng.integers(0, 99, (3, 3 * T)).astype(np.int32))
    ws = None
    for x, rows in ((wide, dict(n_new=dn)), (wide, dict()), (flat, dict(row_starts=ds, T_max=T)), (flat, dict(row_starts=ds))):
        q, k, v = x[..., :Hq, :], x[..., Hq:Hq + H, :], x[..., Hq + H:, :]
        N = q.numel() // (Hq * D)
        for rope, positions in ((ropes[0], None), (ropes[0], pos[0, :N].contiguous()), (ropes[0], pos[:1, :N].contiguous()), (ropes[1], pos[:, :N].contiguous()),
                                (ropes[1], pos[:, :N].contiguous().view((3,) + tuple(q.shape[:-2])))):
            def turn():
                out = torch.full(q.shape, 3.0, dtype=torch.bfloat16, device="cuda")
                got = b.radar_rope(q, k, rope, positions=positions, ctx_lens=dc, q_out=out, k_out=torch.zeros(k.shape, dtype=torch.bfloat16, device="cuda"), **rows)
                assert got[0] is out
                return [got[0], got[1]]
            both("rope", turn)

            def append():
                c, out = gpu_cache(cache, R, D), torch.full(q.shape, 3.0, dtype=torch.bfloat16, device="cuda")
                kw = {n: t for n, t in rows.items() if n != "T_max"}
                assert b.radar_kvq_append_rope(c, q, k, v, slots, rope, positions=positions, ctx_lens=dc, layer=1, q_out=out, **kw) is out
                return [c.data.clone(), out]
            both("append", append)
        c = gpu_cache(cache, R, D)
        ws = b.new_workspace(b.radar_chunk_attention_kvq_workspace_bytes(b.kvq_chunk_desc(q, c, tables.shape[1], 3, T, N))) if ws is None else ws
        room = torch.zeros((Hq,) + tuple(q.shape[:-2]) + (D,), dtype=torch.bfloat16, device="cuda").movedim(0, -2)
        for out, S, split, scale in ((None, None, 0, 0.0), (room, 60, 64, 0.2)):
            def attention():
                lse = torch.full(q.shape[:-1], 7.0, device="cuda")
                room.zero_()
                got = b.radar_chunk_attention_kvq(q, c, dt, dc, layer=1, S_max=S, out=out, lse_out=lse, workspace=ws, rows_per_split=split, softmax_scale=scale, **rows)
                assert out is None or got is out
                return [got.clone(), lse]
            both("attention", attention)
    both.native = True
    q, k = wide[:, :, :Hq], wide[:, :, Hq:Hq + H]
    for bad in (lambda: b.radar_rope(q.float(), None, ropes[0]), lambda: b.radar_rope(q, k[:, :2], ropes[0]), lambda: b.radar_rope(q, k, ropes[1], positions=pos.t().contiguous()),
                lambda: b.radar_kvq_append_rope(c, q, k, k.contiguous(), slots, ropes[0]), lambda: b.radar_kvq_append_rope(c, q, k, k, slots[:2], ropes[0]),
                lambda: b.radar_chunk_attention_kvq(q, c, dt[:2], dc, workspace=ws), lambda: b.radar_chunk_attention_kvq(q, c, dt, dc, n_new=dn[:1], workspace=ws),
                lambda: b.radar_chunk_attention_kvq(q[:1].expand(3, T, Hq, D), c, dt, dc, workspace=ws), lambda: b.radar_chunk_attention_kvq(flat[:, :Hq], c, dt, dc, workspace=ws)):
        with pytest.raises(ValueError):
            bad()
    own = q.contiguous()
    for bad in (lambda: b.radar_chunk_attention_kvq(own, c, dt, dc, out=own, workspace=ws), lambda: b.radar_chunk_attention_kvq(q, c, dt, dc, S_max=tables.shape[1] * R + 1, workspace=ws),
                lambda: b.radar_chunk_attention_kvq(q, c, dt, dc, workspace=ws[:4096]), lambda: b.radar_rope(q, None, ropes[0], q_out=wide.flatten()[:q.numel()].view(q.shape))):
        with pytest.raises(b.RadarError):
            bad()
