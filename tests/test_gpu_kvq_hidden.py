"""Attention over the paged 4-bit cache: rows that a node may not see have no influence on it, whatever bytes they hold."""
import numpy as np
import pytest
import torch

from gpu_util import bf16_dev, dev, host
from kvq_util import seed
from oracle import kvq
from test_gpu_kvq import binding, gpu_cache, make_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [253, 254, 255, None])
@pytest.mark.parametrize("D,T,Hq,H", [(64, 6, 4, 2), (128, 12, 8, 2), (64, 40, 2, 2), (128, 64, 8, 1)])
def test_any_bytes_in_hidden_rows(D, T, Hq, H, scale):
    """Every row of the tree but one path, the rows behind it and blocks of nobody hold bytes at random, with scales that no row is written with
    (253 and 254 reach infinity) or any.  Nodes that see none of it get the very bits that they get over zeros."""
    b, rng = binding(), seed(600 + T + (scale or 0))
    R, ctx, nodes = 16, np.array([37, 0, 64], np.int32), np.array([T, T, 3], np.int32)
    tables, cache, q, qb, par = make_attention(rng, ctx, T, nodes, Hq, H, D, R)
    n_blocks = cache.shape[1]
    good, sound = set(), np.zeros((3, T), bool)
    for bb in range(3):
        good |= {kvq.row_slot(tables[bb], R, n_blocks, j) for j in range(int(ctx[bb]))}
        a, way = nodes[bb] - 1, set()
        while a >= 0:
            way.add(a)
            a = par[bb, a]
        good |= {kvq.row_slot(tables[bb], R, n_blocks, int(ctx[bb]) + int(a)) for a in way}
        for i in range(nodes[bb]):                                   # nodes all of whose path is sound
            a = i
            while a >= 0 and a in way:
                a = par[bb, a]
            sound[bb, i] = a < 0
    bad = cache.copy()
    for slot in range(n_blocks * R):
        if slot in good:
            continue
        for data, fill in ((cache, False), (bad, True)):
            row = kvq.raw(data, R, D, 0, slot)
            kvq.put_raw(data, R, D, 0, slot, rng.integers(0, 256, row.shape, dtype=np.uint8) if fill else np.zeros_like(row))
        if scale is not None:
            for at in kvq._code_places(R, D, slot % R)[2]:
                bad[0, slot // R][:, at] = scale
    assert sound.sum() > 3
    got = []
    for data in (cache, bad):
        for split in (0, 64):
            lse = torch.empty(q.shape[:3], dtype=torch.float32, device="cuda")
            out = b.radar_tree_attention_kvq(bf16_dev(qb), gpu_cache(data, R, D), dev(tables), dev(ctx), dev(par), dev(nodes), lse_out=lse, rows_per_split=split)
            got.append((host(out.float())[sound], host(lse)[sound]))
    for one, other in ((0, 2), (1, 3)):
        assert np.isfinite(got[other][0]).all() and np.isfinite(got[other][1]).all()
        assert np.array_equal(got[one][0], got[other][0]) and np.array_equal(got[one][1], got[other][1])
