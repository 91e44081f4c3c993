"""Verification passes over the paged 4-bit cache in which sequences are refused blocks: nobody's rows but their own are touched."""
import numpy as np
import pytest
import torch

from gpu_util import dev, host
from kvq_util import seed
from oracle import kvq
from test_gpu_kvq import Serving, binding, check_attention

pytestmark = pytest.mark.gpu


class Tight(Serving):
    """A pool that does not hold what the batch asks for.  The caller keeps a refused sequence's length."""
    taken_back = 0

    def calls(self):
        b, (B, T, Hq, H, D, R, M, n_blocks, layers) = self.b, self.shape
        b.radar_kvq_blocks(self.ctx, self.tables, T, n_new=self.nodes, slots=self.slots, granted=self.granted)
        for layer in range(layers):
            b.radar_kvq_append(self.cache, self.k[layer], self.v[layer], self.slots, layer=layer)
            b.radar_tree_attention_kvq(self.q[layer], self.cache, self.tables.block_tables, self.ctx, self.parents, self.nodes, layer=layer,
                                       out=self.out[layer], lse_out=self.lse[layer], workspace=self.ws)
        b.radar_kvq_commit(self.cache, self.tables.block_tables, self.ctx, self.len, self.path, new_ctx_lens=self.new_ctx)
        self.ctx.copy_(torch.where(self.granted > 0, self.new_ctx, self.ctx))

    def check(self, x):
        B, T, Hq, H, D, R, M, n_blocks, layers = self.shape
        old = self.h_tables[0]
        slots, granted, owned, n_free, tables, free = kvq.blocks(x["ctx"], x["nodes"], *self.h_tables, R, T)
        self.h_tables = (tables, owned, free, n_free)
        for got, want in ((self.slots, slots), (self.granted, granted), (self.tables.block_tables, tables), (self.tables.owned, owned),
                          (self.tables.free_blocks, free), (self.tables.n_free, [n_free])):
            assert np.array_equal(host(got), want)
        held = [t for bb in range(B) for t in tables[bb, :owned[bb]]]
        for bb in np.nonzero(granted == 0)[0]:                       # what its stale entries would have reached
            self.taken_back += any(t in held for t in old[bb, owned[bb]:-(-(x["ctx"][bb] + x["nodes"][bb]) // R)] if t >= 0)
        for layer in range(layers):
            for bb in range(B):
                for i in range(T):
                    kvq.put(self.h_cache, R, D, layer, int(slots[bb, i]), x["k"][layer, bb, i], x["v"][layer, bb, i])
            check_attention(x["q"][layer], self.h_cache, R, D, layer, tables, x["ctx"], x["parents"], x["nodes"], self.out[layer], self.lse[layer])
        self.h_cache, new = kvq.commit(self.h_cache, R, D, tables, x["ctx"], x["len"], x["path"])
        assert np.array_equal(host(self.new_ctx), new) and np.array_equal(host(self.ctx), np.where(granted, new, x["ctx"]))
        assert np.array_equal(host(self.cache.data), self.h_cache)
        return int((granted == 0).sum())

    def long_trees(self, x):
        """Trees that are chains, accepted whole: as many rows asked for and moved as there can be."""
        B, T = self.shape[:2]
        x["nodes"], x["parents"] = np.full(B, T, np.int32), np.tile(np.arange(-1, T - 1, dtype=np.int32), (B, 1))
        x["len"], x["path"] = np.full(B, T // 2, np.int32), np.tile(np.arange(0, 2 * T, 2, dtype=np.int32) % T, (B, 1))
        for n in ("nodes", "parents", "len", "path"):
            getattr(self, n).copy_(dev(x[n]))
        return x

    def step(self, n, run):
        """A pass; every third hands a block back to whoever asks first (a sequence goes back to a shorter prefix), some end and start again."""
        B = self.shape[0]
        if n % 3 == 2:
            self.ctx[n % B] = self.ctx[n % B].clamp(max=3)
        self.ctx.clamp_(min=0)
        if n % 7 == 6:
            self.ctx[(n + 1) % B] = -1
        x = self.new_inputs()
        if n % 2:
            x = self.long_trees(x)
        run()
        torch.cuda.synchronize()
        return self.check(x)


def test_passes_with_refused_sequences():
    s = Tight(seed(112), B=4, n_blocks=8)
    refused = [s.step(n, s.calls) for n in range(40)]
    assert sum(refused) > 8 and s.taken_back > 0


def test_a_captured_pass_with_refused_sequences():
    s = Tight(seed(113), B=4, D=128, n_blocks=8, layers=1)
    s.step(0, s.calls)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.calls()
    refused = [s.step(n, s.calls if n % 5 == 4 else g.replay) for n in range(1, 40)]
    assert sum(refused) > 8 and s.taken_back > 0


@pytest.mark.parametrize("B,M", [(3, 200), (1500, 70)])
def test_refused_sequences_of_wide_tables(B, M):
    """More entries than a wavefront has lanes, more sequences than a workgroup; the call repeated with the same result."""
    b, rng = binding(), seed(124 + B)
    R, T, n = 16, 9, B * 2
    tables, owned = rng.integers(0, n, (B, M)).astype(np.int32), np.zeros(B, np.int32)
    free = rng.permutation(n).astype(np.int32)
    owned[:] = rng.integers(0, 2, B)
    n_free = n - int(owned.sum())
    tables[owned == 1, 0] = free[n_free:]
    t = b.KvqTables(block_tables=dev(tables), owned=dev(owned), free_blocks=dev(free), n_free=dev(np.array([n_free], np.int32)), block_rows=R)
    ctx = rng.choice([0, 10, 40, M * R - 2, M * R + 5, -1], B).astype(np.int32)
    want = kvq.blocks(ctx, None, tables, owned, free, n_free, R, T)
    assert (want[1] == 0).any()
    out = dict(owned_out=torch.empty_like(t.owned), n_free_out=torch.empty_like(t.n_free))
    for _ in range(2):
        slots, granted = b.radar_kvq_blocks(dev(ctx), t, T, **out)
        for got, w in zip((slots, granted, out["owned_out"], out["n_free_out"], t.block_tables, t.free_blocks), want):
            assert np.array_equal(host(got).reshape(-1), np.asarray(w).reshape(-1))
