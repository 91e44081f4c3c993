"""Attention of chunks whose blocks of columns are dealt to several workgroups: in every kind of launch, by the library's plan and by parts of so many rows, against the
oracle, and the parts as they lie in the workspace."""
import numpy as np
import pytest
import torch

from gpu_util import bf16_dev, dev
from kvq_util import seed
from oracle import kvq
from test_gpu_kvq import binding, gpu_cache
from test_gpu_kvq_chunk import attend, check, make, ran

pytestmark = pytest.mark.gpu
COUNTERS, MOST, UNTOUCHED = 65536, 1024, -0x5A5A5A5B             # bytes of the workspace before the parts; parts at most; a word of 0xA5 bytes


def beside(n, ctx, new):
    """One long sequence among n short ones."""
    return [ctx] + [20 + 7 * k % 41 for k in range(n)], [new] + [1 + 5 * k % 17 for k in range(n)]


def workspace(b, q, cache, M, B, T, N, S):
    ws = b.new_workspace(b.radar_chunk_attention_kvq_workspace_bytes(b.kvq_chunk_desc(q, cache, M, B, T, N, S)))
    ws[COUNTERS:] = 0xA5
    return ws


def parts_of(ws, D, columns):
    """What a call over blocks of so many columns left in the workspace: (columns of the part, its sums of weights), in the order of their places.  A part is its
    outputs, then a maximum and a sum a column; a block whose columns fit 16 or 32 is handed over as one of those."""
    words = ws[COUNTERS:].view(torch.int32)[:MOST * columns * (D + 2)].view(MOST, -1)
    got = []
    for part in words[(words != UNTOUCHED).any(1)]:
        last = int((part != UNTOUCHED).nonzero().max())
        cols = min(c for c in (16, 32, 64) if last < c * (D + 2))
        got.append((cols, part[cols * D:cols * (D + 2)].view(torch.float32)[1::2].cpu().numpy()))
    return got


# The kernel, contexts, new rows, heads, the rows of a part (0: the library's), and the widths of blocks that come in parts.
CASES = [("16x8", [2061], [3], 1, 1, 0, {16}), ("16x8", [512], [3], 1, 1, 128, {16}), ("16x4", [1885], [3], 1, 1, 0, {16}), ("16x4", [365], [3], 1, 1, 64, {16}),
         ("32x8", [1636, 2247], [130, 118], 16, 8, 0, {16, 32}), ("32x8", [1699, 1752, 2873, 1554], [180, 74, 4, 64], 16, 4, 0, {16}),
         ("32x8", [558, 408, 397, 386, 653], [17, 1, 17, 13, 4], 64, 8, 128, {16, 32}),
         ("64x8", [8733, 9871, 6333, 7205, 6479], [180, 90, 122, 120, 158], 6, 2, 0, {16, 32, 64}),
         ("64x8", [6526, 7309, 8093, 11515], [130, 96, 84, 24], 12, 4, 128, {16, 32, 64}),
         ("64x4", [7323, 11982, 6015, 10804, 9892], [70, 4, 58, 21, 1], 32, 4, 0, {16, 32, 64}), ("64x4", [783, 1393, 1236], [180, 8, 90], 64, 8, 0, {16, 64}),
         ("64x4", [530, 584], [300, 206], 32, 4, 128, {32, 64}), ("64x4", [1277, 1043, 922, 1196, 1000], [130, 121, 96, 96, 75], 32, 8, 64, {16, 64}),
         ("64x2", *beside(39, 1500, 17), 80, 16, 0, {32, 64}), ("64x2", *beside(39, 1500, 17), 80, 16, 64, {32, 64}),
         ("64x1", *beside(39, 1500, 17), 128, 32, 0, {16, 64}), ("64x1", *beside(39, 1500, 17), 160, 32, 0, {32, 64}),
         ("64x1", *beside(39, 1500, 17), 128, 32, 64, {16, 64}), ("64x1", *beside(39, 1500, 17), 160, 32, 64, {32, 64})]


@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("name,ctx,new,Hq,H,split,widths", CASES)
def test_parts_in_every_kind(name, ctx, new, Hq, H, split, widths, D, far):
    """The kernel that is named ran, parts were handed over of blocks of those widths, the joined rows are the oracle's, the counters zero, and a second call leaves the same bits."""
    b, rng, R, B, T, N = binding(), seed(940 + sum(new) + Hq + D), 64, len(ctx), max(new), sum(new)
    ctx = np.array(ctx, np.int32)
    S = int((ctx + np.array(new)).max())
    tables, cache, q, bits, starts, _ = make(rng, ctx, new, Hq, H, D, R)
    if far:                                                          # more than 4 GB of cache, the blocks all over it
        n_blocks = (5 << 30) // (H * kvq.chunk_bytes(R, D))
        c = b.KvqCache(n_blocks, R, H, D)
        ids = np.sort(rng.choice(n_blocks, cache.shape[1], replace=False)).astype(np.int32)
        c.data[0, torch.from_numpy(ids).long().cuda()] = dev(cache[0])
        on_card = np.where(tables >= 0, ids[tables], -1).astype(np.int32)
    else:
        c, on_card = gpu_cache(cache, R, D), tables
    ws = workspace(b, bf16_dev(bits), c, tables.shape[1], B, T, N, S)
    got = []
    call = lambda: got.append(attend(b, bits, None, on_card, ctx, starts, None, T, c=c, R=R, D=D, S_max=S, workspace=ws, rows_per_split=split))      # noqa: E731
    assert ran(call) == {"kvq_chunk_" + name}
    assert {cols for cols, _ in parts_of(ws, D, int(name[:2]))} == widths
    assert (ws[:COUNTERS] == 0).all()
    check(q, cache, R, D, tables, ctx, T, *got[0], row_starts=starts)
    call()
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    del c
    torch.cuda.empty_cache()


@pytest.mark.parametrize("ctx,new,Hq,H,D,split", [([512], [3], 1, 1, 128, 128), ([365], [3], 1, 1, 64, 64), ([11815], [402], 1, 1, 64, 512), ([11815], [402], 1, 1, 128, 448),
                                                  ([2500], [100], 8, 2, 128, 192), ([4000, 10, 900], [1, 300, 40], 8, 2, 64, 320), ([6000, 5000], [200, 31], 8, 2, 128, 1024),
                                                  ([5003], [3], 64, 2, 64, 192), ([1300, 1290, 3101], [64, 64, 90], 8, 1, 128, 256)])
def test_no_part_has_fewer_rows_than_asked_for(ctx, new, Hq, H, D, split):
    """Queries of zeros weigh every key alike: a part's sum, of the block's last column, is the number of its keys.  Between them the parts have all the keys of their columns."""
    b, rng, R, ctx = binding(), seed(960 + sum(new) + D), 32, np.array(ctx, np.int32)
    S = int((ctx + np.array(new)).max())
    tables, cache, q, bits, starts, T = make(rng, ctx, new, Hq, H, D, R)
    c = gpu_cache(cache, R, D)
    ws = workspace(b, bf16_dev(bits), c, tables.shape[1], len(ctx), T, len(q), S)
    got = {}
    name, = ran(lambda: got.update(r=attend(b, np.zeros_like(bits), None, tables, ctx, starts, None, T, c=c, R=R, D=D, S_max=S, workspace=ws, rows_per_split=split)))
    out, lse = got["r"]
    check(np.zeros_like(q), cache, R, D, tables, ctx, T, out, lse, row_starts=starts)
    parts = parts_of(ws, D, int(name[len("kvq_chunk_"):].split("x")[0]))
    assert len(parts) > 1
    # (a column that is not there has no word: what the bytes before it make is less than zero)
    keys = np.array([sums[sums >= 0].max() for _, sums in parts])
    assert (keys == np.round(keys)).all() and keys.min() >= split, (name, np.sort(keys)[:8])
