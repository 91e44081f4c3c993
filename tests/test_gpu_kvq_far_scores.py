"""Attention over the paged 4-bit cache where scores reach far beyond what an exponent can be told apart in 32 bits (2^40 and more): one row takes
all, equal rows share, and a reference that moves between such scores and ordinary ones keeps what was added up before."""
import numpy as np
import pytest
import torch

from gpu_util import bf16_dev, dev
from kvq_util import bf16, random_cache, random_parents, seed, tables_for
from oracle import kvq
from test_gpu_kvq import binding, check_attention, gpu_cache

pytestmark = pytest.mark.gpu


def rows_of(kind, n, rng):
    """Sign and exponent of every row's keys, in the order of the rows."""
    up = np.arange(n) * 46 // n - 4
    mixed = np.where(rng.random(n) < 0.3, up[::-1], rng.integers(-4, 4, n))
    return {"up": (np.ones(n), up), "down": (np.ones(n), up[::-1]), "from far below": (-np.ones(n), up[::-1]), "to far below": (-np.ones(n), up),
            "all far below": (-np.ones(n), 38 + np.arange(n) % 3), "alike": (np.ones(n), np.full(n, 36)), "alike below": (-np.ones(n), np.full(n, 36)),
            "both": (rng.choice([-1.0, 1.0], n), rng.permutation(up)), "far below and near": (np.where(mixed > 5, -1.0, 1.0), mixed),
            "small": (rng.choice([-1.0, 1.0], n), rng.integers(-5, -2, n))}[kind]


@pytest.mark.parametrize("kind", ["up", "down", "from far below", "to far below", "all far below", "alike", "alike below", "both", "far below and near", "small"])
@pytest.mark.parametrize("D,T,Hq,H,L", [(64, 1, 2, 1, 1500), (128, 3, 8, 1, 1100), (128, 40, 2, 2, 900), (64, 60, 1, 1, 1400)])
def test_scores_far_apart(D, T, Hq, H, L, kind):
    """A key is a power of two throughout and a query a few bits a value, so that every score is exact in 32 bits: the bounds of ordinary
    scores hold.  Rows in one launch, in a line of divided units, and joined by several workgroups."""
    b, rng, R = binding(), seed(500 + T + len(kind)), 16
    ctx, nodes = np.array([L, L // 9], np.int32), np.array([T, T], np.int32)
    tables, n_blocks = tables_for(rng, [int(c) + T for c in ctx], R, width=(1 << 15) // R)
    cache = random_cache(rng, 1, n_blocks, H, R, D)
    for bb in range(2):
        n = int(ctx[bb]) + T
        sign, power = rows_of(kind, n, rng)
        v = rng.normal(size=(n, H, D))
        for j in range(n):
            kvq.put(cache, R, D, 0, kvq.row_slot(tables[bb], R, n_blocks, j), np.full((H, D), sign[j] * 2.0 ** int(power[j])), v[j])
    q, qb = bf16(rng.choice([0.5, 1.0, 1.5, 2.0], (2, T, Hq, D)))
    par, c = random_parents(rng, 2, T, nodes), gpu_cache(cache, R, D)
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device="cuda")
    for kw in (dict(S_max=L + T), dict(S_max=1 << 15), dict(rows_per_split=64)):
        out = b.radar_tree_attention_kvq(bf16_dev(qb), c, dev(tables), dev(ctx), dev(par), dev(nodes), lse_out=lse, **kw)
        assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all()
        check_attention(q, cache, R, D, 0, tables, ctx, par, nodes, out, lse)


def test_the_largest_query_decides():
    """Scores of ordinary rows under queries of 2^20 and 2^40: the row with the largest score is the output."""
    b, rng, R, D, T, Hq, H = binding(), seed(520), 16, 128, 2, 4, 2
    ctx, nodes = np.array([700], np.int32), np.array([T], np.int32)
    tables, n_blocks = tables_for(rng, [700 + T], R)
    cache = random_cache(rng, 1, n_blocks, H, R, D)
    q, qb = bf16(rng.normal(size=(1, T, Hq, D)) * np.array([2.0 ** 20, 2.0 ** 40, 2.0 ** 30, 2.0 ** 60])[:, None])
    par = np.array([[-1, 0]], np.int32)
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device="cuda")
    got = b.radar_tree_attention_kvq(bf16_dev(qb), gpu_cache(cache, R, D), dev(tables), dev(ctx), dev(par), dev(nodes), lse_out=lse)
    kv = [kvq.get(cache, R, D, 0, kvq.row_slot(tables[0], R, n_blocks, j)) for j in range(700 + T)]
    for i in range(T):
        for h in range(Hq):
            K, V = (np.array([x[s][h // 2] for x in kv[:701 + i]]) for s in (0, 1))
            x, reach = K @ q[0, i, h] / np.sqrt(D), (np.abs(K) @ np.abs(q[0, i, h])).max() / np.sqrt(D)
            first, second = np.sort(x)[-1], np.sort(x)[-2]
            slack = (D + 8) * 2.0 ** -24 * reach
            assert first - second > 2 * slack + 200                  # whatever 32 bits make of the scores
            assert np.array_equal(got[0, i, h].double().cpu().numpy(), V[x.argmax()])
            assert abs(float(lse[0, i, h]) - first) <= slack + 2.0 ** -19 * abs(first)
