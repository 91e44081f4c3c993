"""The paged 4-bit cache on the GPU against its oracle (numpy, 64 bits): block tables, rows in and out, the accepted path's
rows, attention, and a run of all of them as a verification pass makes the calls."""
import numpy as np
import pytest
import torch

from gpu_util import bf16_dev, dev, host
from kvq_util import bf16, random_cache, random_parents, seed, tables_for
from oracle import kvq
from paper_2512_14069_amd import synth

pytestmark = pytest.mark.gpu


def binding():
    from paper_2512_14069_amd import binding as b
    return b


def gpu_cache(data, R, D):
    return binding().KvqCache(data=dev(data), block_rows=R, D=D)


# ------------------------------------------------------------------ rows in and out

@pytest.mark.parametrize("N,H,D,R", [(1, 1, 64, 16), (1, 8, 128, 16), (7, 3, 64, 32), (8, 1, 128, 64), (60, 8, 128, 16), (65, 5, 64, 128), (203, 2, 128, 32)])
def test_append_writes_the_oracles_bytes_and_no_others(N, H, D, R):
    b, rng = binding(), seed(10 + N)
    n_blocks = -(-N // R) + 3
    cache = np.full((2, n_blocks, H, kvq.chunk_bytes(R, D)), 0xAA, np.uint8)
    slots = rng.permutation(n_blocks * R)[:N].astype(np.int32)
    if N > 4:
        slots[rng.choice(N, 3, replace=False)] = [-1, n_blocks * R, np.iinfo(np.int32).min]
    x = rng.normal(size=(2, N, H, D)) * 2.0 ** rng.integers(-3, 4, (2, N, H, 1))
    x[:, :, :, ::37] *= 20
    (k, v), (kb, vb) = bf16(x)
    c = gpu_cache(cache, R, D)
    wide = torch.randn((N, 2 * H + 3, D), device="cuda").bfloat16()  # a projection's output, of which the rows are slices
    wide[:, 1:1 + H], wide[:, 2 + H:2 + 2 * H] = bf16_dev(kb), bf16_dev(vb)
    assert b.radar_kvq_append(c, wide[:, 1:1 + H], wide[:, 2 + H:2 + 2 * H], dev(slots), layer=1) is c
    for n in range(N):
        kvq.put(cache, R, D, 1, int(slots[n]), k[n], v[n])
    assert np.array_equal(host(c.data), cache)


def test_append_of_every_bf16_value():
    """All 65536 patterns, in blocks whose scale each of a few values sets; infinities and NaN make NaN blocks."""
    b, D, R = binding(), 128, 128
    bits = np.arange(1 << 16, dtype=np.uint32).astype(np.uint16)
    with np.errstate(invalid="ignore"):
        vals = synth.bf16_bits_to_f32(bits)
    for top in (None, 0x3f80, 0x3fdf, 0x3fe0, 0x7f7f, 0x0080):       # none, 1, 1.742, 1.75, the largest, the smallest normal number
        a = bits.copy()
        if top is not None:                                          # what is larger is left out, and each block of 32 starts with the top
            a[(a & 0x7fff) > top] = 0
            a[::32] = top
        rows = a.reshape(-1, 1, D)
        N = len(rows)
        with np.errstate(invalid="ignore"):
            x = synth.bf16_bits_to_f32(rows).astype(np.float64)
        cache = np.zeros((1, N // R, 1, kvq.chunk_bytes(R, D)), np.uint8)
        c = gpu_cache(cache, R, D)
        b.radar_kvq_append(c, bf16_dev(rows), bf16_dev(rows[::-1].copy()), dev(np.arange(N, dtype=np.int32)))
        for n in range(N):
            kvq.put(cache, R, D, 0, n, x[n], x[N - 1 - n])
        assert np.array_equal(host(c.data), cache), top
    assert np.isnan(vals).any()


@pytest.mark.parametrize("H,D,R,layers", [(1, 64, 16, 1), (3, 128, 32, 2), (8, 64, 128, 3)])
def test_read_gives_what_the_codes_stand_for(H, D, R, layers):
    b, rng = binding(), seed(20 + H)
    n_blocks = 5
    cache = random_cache(rng, layers, n_blocks, H, R, D)
    cache[..., R * D:] = rng.integers(0, 256, cache[..., R * D:].shape, dtype=np.uint8)             # every scale, 255 among them
    store = torch.zeros((layers, cache[0].nbytes + 48), dtype=torch.uint8, device="cuda")           # layers with a gap between them
    data = store[:, :cache[0].nbytes].view((layers,) + cache.shape[1:])
    data.copy_(dev(cache))
    c = b.KvqCache(data=data, block_rows=R, D=D)
    slots = np.concatenate([rng.integers(0, n_blocks * R, 20), [0, n_blocks * R - 1, n_blocks * R, -1, np.iinfo(np.int32).max]]).astype(np.int32)
    k, v = b.radar_kvq_read(c, dev(slots))
    k1, v1 = b.radar_kvq_read(c, dev(slots), layer=layers - 1)
    want = [[kvq.get(cache, R, D, layer, int(s)) for s in slots] for layer in range(layers)]
    for got, i in ((k, 0), (v, 1)):
        w = np.array([[x[i] for x in one] for one in want])
        # exact in bf16 down to the smallest scale (2^-128 is a bf16); bytes 253 and 254, which append never writes, reach past the largest: infinity
        with np.errstate(over="ignore", invalid="ignore"):
            r = bf16(w)[0]
        assert np.array_equal(r[np.abs(w) < 2.0 ** 128], w[np.abs(w) < 2.0 ** 128])
        assert np.array_equal(host(got.double()), r, equal_nan=True)
    assert torch.equal(k1[0].view(torch.int16), k[-1].view(torch.int16)) and torch.equal(v1[0].view(torch.int16), v[-1].view(torch.int16))


def test_no_rows():
    b = binding()
    c = b.KvqCache(2, 16, 2, 64)
    none = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    b.radar_kvq_append(c, none, none, torch.zeros(0, dtype=torch.int32, device="cuda"))
    k, v = b.radar_kvq_read(c, torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert tuple(k.shape) == tuple(v.shape) == (1, 0, 2, 64)


# ------------------------------------------------------------------ block tables

def run_blocks(b, rng, B, M, R, T, n, rounds, in_place, use_new):
    tables, owned = np.full((B, M), -1, np.int32), np.zeros(B, np.int32)
    free, n_free = rng.permutation(n).astype(np.int32), n
    t = b.KvqTables(block_tables=dev(tables), owned=dev(owned), free_blocks=dev(free), n_free=dev(np.array([n_free], np.int32)), block_rows=R)
    denied = 0
    for _ in range(rounds):
        ctx = np.where(rng.random(B) < 0.15, -rng.integers(1, 9, B), rng.integers(0, max(1, M * R * 9 // 8 - T), B)).astype(np.int32)
        new = rng.integers(-1, T + 3, B).astype(np.int32) if use_new else None
        want = kvq.blocks(ctx, new, tables, owned, free, n_free, R, T)
        kw = {} if in_place else dict(owned_out=torch.empty_like(t.owned), n_free_out=torch.empty_like(t.n_free))
        for _ in range(1 if in_place else 2):                        # with outputs of their own the call may be repeated
            slots, granted = b.radar_kvq_blocks(dev(ctx), t, T, n_new=None if new is None else dev(new), **kw)
            got = [host(x) for x in (slots, granted, kw.get("owned_out", t.owned), kw.get("n_free_out", t.n_free), t.block_tables, t.free_blocks)]
            for name, x, y in zip(("slots", "granted", "owned", "n_free", "tables", "free"), got, want):
                assert np.array_equal(x.reshape(-1), np.asarray(y).reshape(-1)), name
        if not in_place:
            t.owned, t.n_free = kw["owned_out"], kw["n_free_out"]
        denied += int((want[1] == 0).sum())
        owned, n_free, tables, free = want[2:]
    return denied


@pytest.mark.parametrize("B,M,R,T,n,in_place,use_new", [
    (1, 1, 16, 1, 1, True, True), (1, 300, 16, 64, 301, False, True), (16, 20, 16, 60, 200, True, True), (16, 20, 32, 60, 200, False, False),
    (700, 9, 64, 3, 3000, True, True), (1500, 6, 16, 7, 4000, False, True), (2100, 3, 128, 30, 3500, True, True), (64, 40, 16, 400, 2000, False, True)])
def test_blocks_against_the_oracle(B, M, R, T, n, in_place, use_new):
    """Batches of one and of several rounds of lanes, tables that run out, slots mapped in the same launch and in one of their own."""
    denied = run_blocks(binding(), seed(30 + B + T), B, M, R, T, n, 6, in_place, use_new)
    assert denied > 0 or B == 1


def test_blocks_stay_in_bounds_for_any_content():
    """Counts, heights and block numbers that no earlier call wrote: every output is written, inside its array."""
    b, rng = binding(), seed(40)
    B, M, R, T, n = 37, 5, 16, 9, 64
    big = np.iinfo(np.int32).max
    for height in (-5, 0, 63, 64, 65, big):
        pad = lambda x: dev(np.concatenate([np.full(64, 77, np.int32), np.asarray(x, np.int32).reshape(-1), np.full(64, 77, np.int32)]))     # noqa: E731
        tab, fre, own = pad(rng.integers(-9, 99, B * M)), pad(rng.integers(-9, 99, n)), pad(rng.integers(-3, M + 4, B))
        cut = lambda t, *shape: t[64:-64].view(*shape)                                                                                      # noqa: E731
        t = b.KvqTables(block_tables=cut(tab, B, M), owned=cut(own, B), free_blocks=cut(fre, n), n_free=dev(np.array([height], np.int32)), block_rows=R)
        ctx = rng.choice([-1, 0, 3, 40, 80, big, big - 5, -big], B).astype(np.int32)
        slots, granted = b.radar_kvq_blocks(dev(ctx), t, T, n_new=dev(rng.choice([0, 4, 9, big, -big], B).astype(np.int32)))
        s = host(slots)
        assert ((s >= -1) & (s < n * R)).all() and set(host(granted)) <= {0, 1}
        assert (s[ctx > M * R] == -1).all() and (s[ctx < 0] == -1).all()
        assert 0 <= int(host(t.n_free)[0]) <= n and ((host(t.owned) >= 0) & (host(t.owned) <= M)).all()
        for x in (tab, fre, own):
            assert (host(x[:64]) == 77).all() and (host(x[-64:]) == 77).all()


# ------------------------------------------------------------------ the accepted path

@pytest.mark.parametrize("B,H,D,R,layers,P", [(1, 1, 64, 16, 1, 9), (3, 8, 128, 16, 2, 64), (5, 3, 64, 32, 3, 64), (2, 5, 128, 128, 4, 2), (4, 2, 128, 64, 1, 1)])
def test_commit_against_the_oracle(B, H, D, R, layers, P):
    b, rng = binding(), seed(50 + B)
    ctx = rng.integers(0, 100, B).astype(np.int32)
    if B > 2:
        ctx[1] = -4
    tables, n_blocks = tables_for(rng, [max(0, c) + 64 for c in ctx], R)
    cache = random_cache(rng, layers, n_blocks, H, R, D)
    for trial in range(6):
        if trial < 3:                                                # a way down a tree: ever larger row numbers
            path = np.array([np.concatenate([[0], np.sort(rng.permutation(np.arange(1, 64))[:P - 1])]) for _ in range(B)]).astype(np.int32)
            n = rng.integers(0, P, B).astype(np.int32)
        else:                                                        # any content
            path = rng.integers(-3, 70, (B, P)).astype(np.int32)
            n = rng.choice([-7, 0, P // 2, P - 1, P + 9], B).astype(np.int32)
        if trial == 5:
            tables = tables.copy()
            tables[0, ctx[0] // R] = rng.choice([-1, n_blocks, 1 << 30])
        c = gpu_cache(cache, R, D)
        new = b.radar_kvq_commit(c, dev(tables), dev(ctx), dev(n), dev(path))
        cache, want = kvq.commit(cache, R, D, tables, ctx, n, path)
        assert np.array_equal(host(new), want), trial
        assert np.array_equal(host(c.data), cache), trial


@pytest.mark.parametrize("D,n_hi", [(64, 9), (128, 9), (128, 12)])
def test_commit_of_many_layers(D, n_hi):
    """So many pairs of layer and head that a wavefront has several of them, their number no multiple of it; short paths and long ones."""
    b, rng = binding(), seed(55 + n_hi)
    B, H, R, layers, P = 37, 8, 16, 83, 20
    ctx = rng.integers(0, 40, B).astype(np.int32)
    tables, n_blocks = tables_for(rng, [c + 30 for c in ctx], R)
    cache = random_cache(rng, layers, n_blocks, H, R, D)
    path = np.array([np.concatenate([[0], np.sort(rng.permutation(np.arange(1, 30))[:P - 1])]) for _ in range(B)]).astype(np.int32)
    n = rng.integers(0, n_hi, B).astype(np.int32)
    c = gpu_cache(cache, R, D)
    new = b.radar_kvq_commit(c, dev(tables), dev(ctx), dev(n), dev(path))
    cache, want = kvq.commit(cache, R, D, tables, ctx, n, path)
    assert np.array_equal(host(new), want) and np.array_equal(host(c.data), cache)


@pytest.mark.parametrize("N,H,D,layers", [(1001, 3, 128, 22), (2050, 5, 64, 13), (1700, 8, 128, 5)])
def test_read_of_many_layers(N, H, D, layers):
    """Layers read four at a time, and the rest; what a call for a layer alone gives is what the oracle gives (test_read_gives_what_the_codes_stand_for)."""
    b, rng, R = binding(), seed(25 + H), 16
    n_blocks = N // R + 3
    cache = random_cache(rng, layers, n_blocks, H, R, D)
    slots = rng.permutation(n_blocks * R)[:N].astype(np.int32)
    slots[rng.choice(N, 5, replace=False)] = [-1, n_blocks * R, 2 ** 31 - 1, -2 ** 31, -7]
    k, v = b.radar_kvq_read(gpu_cache(cache, R, D), dev(slots))
    for layer in range(layers):
        k1, v1 = b.radar_kvq_read(gpu_cache(cache[layer:layer + 1], R, D), dev(slots))
        for many, one in ((k[layer], k1[0]), (v[layer], v1[0])):
            assert torch.equal(many.view(torch.int16), one.view(torch.int16))
    for n in rng.choice(N, 20, replace=False):
        if 0 <= slots[n] < n_blocks * R:
            want = kvq.get(cache, R, D, layers - 1, int(slots[n]))
            assert np.array_equal(host(k[-1, n].double()), want[0], equal_nan=True) and np.array_equal(host(v[-1, n].double()), want[1], equal_nan=True)


# ------------------------------------------------------------------ attention

def check_attention(q, cache, R, D, layer, tables, ctx, par, nodes, got, lse, S_max=None, scale=0.0):
    """Every output within its own bound.  out: the probabilities are rounded to bf16 (half a step, 2^-8 of each, so of sum p |v|) and so is
    the output (2^-8 of it); fp32 arithmetic (scores, exponentials, sums) is within 2^-14 of sum p |v| as long as a score's error is below it, which the bound on lse checks.  lse: a score is D products added in fp32
    (2^-24 of the magnitudes a step) and scaled; exponentials, their sum and the logarithm 2^-19 together."""
    out_r, lse_r, spread, reach = kvq.attention(q, cache, R, D, layer, tables, ctx, par, nodes, S_max, scale, want_sizes=True)
    out, lse = host(got.double()), host(lse.double())
    nan = np.isnan(out_r)
    assert np.array_equal(np.isnan(out), nan)
    err = np.abs(np.where(nan, 0, out) - np.where(nan, 0, out_r))
    sp = np.where(nan, 0, spread)
    bound = 2.0 ** -8 * (sp + np.abs(np.where(nan, 0, out_r)) + 2.0 ** -8 * sp) + 2.0 ** -14 * sp + 1e-30
    assert (err <= bound).all(), (err / bound).max()
    same = (lse == lse_r) | (np.isnan(lse) & np.isnan(lse_r))
    lerr = np.where(same, 0, np.abs(np.where(same, 0, lse) - np.where(same, 0, lse_r)))
    lbound = (D + 8) * 2.0 ** -24 * np.where(np.isnan(reach), 0, reach) + 2.0 ** -19 * (1 + np.abs(np.where(np.isfinite(lse_r), lse_r, 0)))
    assert (lerr <= lbound).all(), (lerr / lbound).max()


def make_attention(rng, ctx, T, nodes, Hq, H, D, R, layers=1, extra=2):
    B = len(ctx)
    tables, n_blocks = tables_for(rng, [max(0, c) + T for c in ctx], R, spare=extra)
    cache = random_cache(rng, layers, n_blocks, H, R, D)
    q, qb = bf16(rng.normal(size=(B, T, Hq, D)))
    par = random_parents(rng, B, T, nodes)
    return tables, cache, q, qb, par


SHAPES = [  # ctx, T, nodes, Hq, Hkv, D, R
    ([0], 1, [1], 1, 1, 64, 16), ([1], 1, [1], 4, 1, 64, 16), ([31, 32, 33, 0], 1, [1, 1, 1, 1], 8, 2, 128, 16), ([300], 1, [1], 8, 1, 128, 128),
    ([7, 200], 2, [2, 1], 12, 3, 64, 32), ([64], 5, [5], 16, 8, 128, 64), ([127, 5, 63], 4, [4, 1, 3], 16, 2, 128, 16),
    ([96], 33, [33], 2, 2, 64, 16), ([40, 0], 17, [17, 9], 10, 2, 128, 32), ([500], 60, [60], 4, 1, 64, 16), ([130, 4], 64, [64, 31], 8, 1, 128, 16),
    ([70], 64, [64], 8, 8, 128, 128), ([15, 16, 17], 20, [20, 1, 13], 20, 4, 64, 64), ([1000, 3], 7, [7, 7], 40, 5, 128, 16),
]


@pytest.mark.parametrize("ctx,T,nodes,Hq,H,D,R", SHAPES)
def test_attention_against_the_oracle(ctx, T, nodes, Hq, H, D, R):
    b, rng = binding(), seed(60 + sum(ctx) + T)
    ctx, nodes = np.array(ctx, np.int32), np.array(nodes, np.int32)
    tables, cache, q, qb, par = make_attention(rng, ctx, T, nodes, Hq, H, D, R, layers=2)
    c = gpu_cache(cache, R, D)
    lse = torch.full(q.shape[:3], 7.0, dtype=torch.float32, device="cuda")
    S = int(ctx.max()) + T
    for kw in (dict(S_max=S), dict(), dict(S_max=S, rows_per_split=64), dict(rows_per_split=192)):
        out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        got = b.radar_tree_attention_kvq(bf16_dev(qb), c, dev(tables), dev(ctx), parents=dev(par), n_nodes=dev(nodes), layer=1, out=out, lse_out=lse, **kw)
        assert got is out
        check_attention(q, cache, R, D, 1, tables, ctx, par, nodes, got, lse)


@pytest.mark.parametrize("ctx,T,Hq,H,D,R,split", [
    ([2048], 60, 32, 8, 128, 32, 0), ([700, 2900, 1], 1, 32, 8, 128, 16, 0), ([4099], 3, 16, 2, 64, 16, 0), ([1500, 9], 40, 64, 8, 128, 64, 0),
    ([9001], 1, 4, 1, 128, 16, 64), ([9001], 20, 4, 1, 64, 16, 64), ([6000, 300], 40, 2, 1, 128, 32, 64)])
def test_attention_over_long_contexts(ctx, T, Hq, H, D, R, split):
    """Rows split over workgroups and joined, up to 140 parts.  The trees are chains (parents left out), all nodes used (n_nodes left out)."""
    b, rng = binding(), seed(70 + T)
    ctx = np.array(ctx, np.int32)
    tables, cache, q, qb, _ = make_attention(rng, ctx, T, np.full(len(ctx), T), Hq, H, D, R)
    c = gpu_cache(cache, R, D)
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device="cuda")
    got = b.radar_tree_attention_kvq(bf16_dev(qb), c, dev(tables), dev(ctx), lse_out=lse, S_max=int(ctx.max()) + T, rows_per_split=split)
    pick = sorted({0, T // 2, T - 1})                                # of the rows; the oracle is slow
    par = np.tile(np.arange(-1, T - 1, dtype=np.int32), (len(ctx), 1))
    some = q.copy()
    heads = sorted({0, Hq // 2, Hq - 1})
    ref = one_rows(some, cache, R, D, tables, ctx, par, pick, heads)
    for (bb, i, h), (o, l, sp, re) in ref.items():
        err = np.abs(host(got[bb, i, h].double()) - o)
        assert (err <= 2.0 ** -8 * (sp + np.abs(o) + 2.0 ** -8 * sp) + 2.0 ** -14 * sp).all()
        assert abs(float(lse[bb, i, h]) - l) <= (D + 8) * 2.0 ** -24 * re + 2.0 ** -19 * (1 + abs(l))


def one_rows(q, cache, R, D, tables, ctx, par, rows, heads):
    """The oracle's formula for some rows and heads only (bounds as in check_attention)."""
    H, n_blocks, Hq = cache.shape[2], cache.shape[1], q.shape[2]
    found = {}
    for b in range(len(ctx)):
        kv = [kvq.get(cache, R, D, 0, kvq.row_slot(tables[b], R, n_blocks, j)) for j in range(int(ctx[b]) + q.shape[1])]
        K, V = np.array([x[0] for x in kv]), np.array([x[1] for x in kv])
        for i in rows:
            mine, a = list(range(int(ctx[b]))), i
            while a >= 0:
                mine.append(int(ctx[b]) + a)
                a = int(par[b, a])
            for h in heads:
                g = h // (Hq // H)
                x = K[mine, g] @ q[b, i, h] / np.sqrt(D)
                w = np.exp(x - x.max())
                found[b, i, h] = ((w / w.sum()) @ V[mine, g], x.max() + np.log(w.sum()), (w / w.sum()) @ np.abs(V[mine, g]),
                                  (np.abs(K[mine, g]) @ np.abs(q[b, i, h])).max() / np.sqrt(D))
    return found


@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,S", [(16, 2048), (16, 1 << 18), (32, 2048), (32, 1 << 18), (64, 2048), (64, 1 << 18)])
def test_attention_of_a_batch_in_every_shape(T, S, D, far):
    """16, 32 and 64 columns a workgroup, whole units (S_max of 2048) and divided ones, caches below and beyond 4 GB; more sequences than a wavefront
    has lanes, of all lengths, some of them ended."""
    b, rng = binding(), seed(200 + T + D)
    B, H, R = 70, 2, 16
    ctx = rng.integers(0, 90, B).astype(np.int32)
    ctx[[3, 64, 69]], ctx[[7, 66]] = -1, [900, 333]
    nodes = rng.integers(1, T + 1, B).astype(np.int32)
    nodes[[7, 8]] = T, T
    tables, cache, q, qb, par = make_attention(rng, ctx, T, nodes, H, H, D, R)
    n_small = cache.shape[1]
    if far:
        n_blocks = (5 << 30) // (H * kvq.chunk_bytes(R, D))
        c = b.KvqCache(n_blocks, R, H, D)
        assert c.data[0].numel() > 1 << 32
        ids = np.sort(rng.choice(n_blocks, n_small, replace=False)).astype(np.int32)
        c.data[0, torch.from_numpy(ids).long().cuda()] = dev(cache[0])
    else:
        c, ids = gpu_cache(cache, R, D), np.arange(n_small, dtype=np.int32)
    wide = np.full((B, S // R), -1, np.int32)
    wide[:, :tables.shape[1]] = np.where((tables >= 0) & (tables < n_small), ids[np.clip(tables, 0, n_small - 1)], -1)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:3], 7.0, dtype=torch.float32, device="cuda")
    b.radar_tree_attention_kvq(bf16_dev(qb), c, dev(wide), dev(ctx), dev(par), dev(nodes), out=out, lse_out=lse, S_max=S)
    check_attention(q, cache, R, D, 0, tables, ctx, par, nodes, out, lse)
    del c
    torch.cuda.empty_cache()


@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,T,Hq,H,S", [(3, 4, 8, 2, 4096), (2, 1, 4, 1, 60000), (1, 60, 32, 8, 7000), (4, 60, 32, 8, 9000)])
def test_units_that_several_workgroups_join(B, T, Hq, H, S, D, far):
    """Few units and room for long sequences: parts of a unit in several workgroups, 16, 32 and 64 columns each.  One workspace for calls whose lengths
    leave parts without a step, units with one part, and none; its counters are zero again after every call."""
    b, rng, R = binding(), seed(300 + T + D + B), 16
    tables, cache, _, _, _ = make_attention(rng, np.full(B, 900), T, np.full(B, T), Hq, H, D, R)
    n_small = cache.shape[1]
    if far:
        n_blocks = (5 << 30) // (H * kvq.chunk_bytes(R, D))
        c = b.KvqCache(n_blocks, R, H, D)
        ids = np.sort(rng.choice(n_blocks, n_small, replace=False)).astype(np.int32)
        c.data[0, torch.from_numpy(ids).long().cuda()] = dev(cache[0])
    else:
        c, ids = gpu_cache(cache, R, D), np.arange(n_small, dtype=np.int32)
    wide = np.full((B, -(-S // R)), -1, np.int32)
    wide[:, :tables.shape[1]] = ids[tables]
    dt, ws = dev(wide), None
    for ctx in ([900, 700, 37, 500], [0, -1, 300, 31], [65, 900, -1, 600]):
        ctx, nodes = np.array(ctx[:B], np.int32), rng.integers(1, T + 1, B).astype(np.int32)
        q, qb = bf16(rng.normal(size=(B, T, Hq, D)))
        par = random_parents(rng, B, T, nodes)
        ws = b.new_workspace(b.radar_tree_attention_kvq_workspace_bytes(b.kvq_attn_desc(bf16_dev(qb), c, wide.shape[1], S))) if ws is None else ws
        out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full(q.shape[:3], 7.0, dtype=torch.float32, device="cuda")
        b.radar_tree_attention_kvq(bf16_dev(qb), c, dt, dev(ctx), dev(par), dev(nodes), out=out, lse_out=lse, S_max=S, workspace=ws)
        check_attention(q, cache, R, D, 0, tables, ctx, par, nodes, out, lse)
        assert (ws[:16384] == 0).all()
    del c
    torch.cuda.empty_cache()


def test_one_workspace_for_calls_of_any_shape():
    """Units joined by different numbers of workgroups and units in a line, one call after the other in a workspace initialised once."""
    b, rng = binding(), seed(97)
    T, Hq, H, D, R, S = 16, 8, 2, 128, 16, 1 << 18
    ctx, nodes = rng.integers(200, 700, 12).astype(np.int32), rng.integers(1, T + 1, 12).astype(np.int32)
    tables, cache, q, qb, par = make_attention(rng, ctx, T, nodes, Hq, H, D, R)
    wide = np.full((12, S // R), -1, np.int32)
    wide[:, :tables.shape[1]] = tables
    c, dq, dt, dc, dp, dn = gpu_cache(cache, R, D), bf16_dev(qb), dev(wide), dev(ctx), dev(par), dev(nodes)
    shapes = [(12, S), (1, 8192), (12, 800), (1, S), (3, 4096), (12, 8192)]
    ws = b.new_workspace(max(b.radar_tree_attention_kvq_workspace_bytes(b.kvq_attn_desc(dq[:B], c, S // R, S_max=n)) for B, n in shapes))
    for B, n in 2 * shapes:
        lse = torch.full((B, T, Hq), 7.0, device="cuda")
        got = b.radar_tree_attention_kvq(dq[:B], c, dt[:B], dc[:B], dp[:B], dn[:B], lse_out=lse, S_max=n, workspace=ws)
        check_attention(q[:B], cache, R, D, 0, tables[:B], ctx[:B], par[:B], nodes[:B], got, lse)


def test_attention_at_the_longest_lengths_allowed():
    """S_max up to the limit, where the work is counted in more than one step: short sequences under it, and a long one."""
    b, rng = binding(), seed(99)
    T, Hq, H, D, R = 64, 64, 8, 64, 128
    S = 2 ** 31 - 1 - 4096
    ctx, nodes = np.array([700], np.int32), np.array([64], np.int32)
    tables, cache, q, qb, par = make_attention(rng, ctx, T, nodes, Hq, H, D, R)
    wide = torch.full((1, -(-S // R)), -1, dtype=torch.int32, device="cuda")
    wide[:, :tables.shape[1]] = dev(tables)
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device="cuda")
    got = b.radar_tree_attention_kvq(bf16_dev(qb), gpu_cache(cache, R, D), wide, dev(ctx), dev(par), dev(nodes), lse_out=lse, S_max=S)
    check_attention(q, cache, R, D, 0, tables, ctx, par, nodes, got, lse)


def test_a_captured_divided_batch_with_other_lengths():
    """Divided units, one workspace: a graph replayed while lengths, trees and which sequences there are change, between eager calls of another shape
    in the same workspace."""
    b, rng = binding(), seed(98)
    B, T, Hq, H, D, R, S = 6, 20, 8, 2, 128, 16, 1 << 16
    tables, cache, _, _, _ = make_attention(rng, np.full(B, 1200), T, np.full(B, T), Hq, H, D, R)
    c = gpu_cache(cache, R, D)
    wide = np.full((B, S // R), -1, np.int32)
    wide[:, :tables.shape[1]] = tables
    z = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")                                                                 # noqa: E731
    q, out = (torch.zeros((B, T, Hq, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lse = torch.zeros((B, T, Hq), device="cuda")
    t, ctx, par, nodes = dev(wide), z(B), z(B, T), z(B)
    ws = b.new_workspace(max(b.radar_tree_attention_kvq_workspace_bytes(b.kvq_attn_desc(x, c, S // R, S_max=S)) for x in (q, q[:2])))
    call = lambda n=B: b.radar_tree_attention_kvq(q[:n], c, t[:n], ctx[:n], par[:n], nodes[:n], out=out[:n], lse_out=lse[:n], S_max=S, workspace=ws)   # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for trial in range(6):
        hc = rng.integers(0, 1200 if trial % 2 else 100, B).astype(np.int32)
        hc[trial] = -1 if trial % 2 else 1100
        hn = rng.integers(1, T + 1, B).astype(np.int32)
        hp = random_parents(rng, B, T, hn)
        hq, bits = bf16(rng.normal(size=(B, T, Hq, D)))
        for x, y in ((ctx, dev(hc)), (nodes, dev(hn)), (par, dev(hp)), (q, bf16_dev(bits))):
            x.copy_(y)
        g.replay()
        torch.cuda.synchronize()
        check_attention(hq, cache, R, D, 0, tables, hc, hp, hn, out, lse)
        call(2)
        torch.cuda.synchronize()
        check_attention(hq[:2], cache, R, D, 0, tables[:2], hc[:2], hp[:2], hn[:2], out[:2], lse[:2])


def test_attention_with_strides_and_a_scale():
    b, rng = binding(), seed(80)
    ctx, T, nodes, Hq, H, D, R = np.array([50, 11], np.int32), 9, np.array([9, 4], np.int32), 8, 2, 128, 16
    tables, cache, q, qb, par = make_attention(rng, ctx, T, nodes, Hq, H, D, R)
    wide = torch.zeros((2, T, Hq + 5, D), dtype=torch.bfloat16, device="cuda")
    wide[:, :, 2:2 + Hq] = bf16_dev(qb)
    room = torch.full((2, Hq, T + 3, D), 5.0, dtype=torch.bfloat16, device="cuda")
    out = room.transpose(1, 2)[:, 1:1 + T]
    lse = torch.empty((2, T, Hq), dtype=torch.float32, device="cuda")
    b.radar_tree_attention_kvq(wide[:, :, 2:2 + Hq], gpu_cache(cache, R, D), dev(tables), dev(ctx), dev(par), dev(nodes), out=out, lse_out=lse, softmax_scale=0.31)
    check_attention(q, cache, R, D, 0, tables, ctx, par, nodes, out, lse, scale=0.31)
    assert (room[:, :, 0] == 5).all() and (room[:, :, 1 + T:] == 5).all()


@pytest.mark.parametrize("D,T,Hq,H", [(64, 6, 4, 2), (128, 12, 8, 2), (128, 64, 8, 1)])
def test_what_is_hidden_has_no_influence(D, T, Hq, H):
    """NaN blocks, of K and of V, in every row of the tree but some, in the rows behind it and in blocks of nobody."""
    b, rng = binding(), seed(81 + T)
    R, ctx, nodes = 16, np.array([37, 0, 64], np.int32), np.array([T, T, 3], np.int32)
    tables, cache, q, qb, par = make_attention(rng, ctx, T, nodes, Hq, H, D, R)
    n_blocks = cache.shape[1]
    good = set()
    for bb in range(3):
        good |= {kvq.row_slot(tables[bb], R, n_blocks, j) for j in range(int(ctx[bb]))}
        a = nodes[bb] - 1                                            # the last node's path stays sound
        while a >= 0:
            good.add(kvq.row_slot(tables[bb], R, n_blocks, int(ctx[bb]) + a))
            a = par[bb, a]
    for slot in range(n_blocks * R):
        if slot not in good:
            _, _, sc = kvq._code_places(R, D, slot % R)
            for at in sc:                                            # one block of the row, or all
                cache[0, slot // R][:, at[rng.integers(0, len(at))] if rng.random() < 0.5 else at] = 255
    c = gpu_cache(cache, R, D)
    for split in (0, 64):
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device="cuda")
        got = b.radar_tree_attention_kvq(bf16_dev(qb), c, dev(tables), dev(ctx), dev(par), dev(nodes), lse_out=lse, rows_per_split=split)
        with np.errstate(invalid="ignore"):
            check_attention(q, cache, R, D, 0, tables, ctx, par, nodes, got, lse)
        for bb in range(3):
            assert torch.isfinite(got[bb, nodes[bb] - 1].float()).all()
        assert torch.isnan(got.float()).any()


def test_queries_and_prefix_rows_that_are_not_finite():
    """NaN goes where the formula takes it and nowhere else."""
    b, rng = binding(), seed(83)
    ctx, T, nodes, Hq, H, D, R = np.array([45, 45], np.int32), 5, np.array([5, 5], np.int32), 4, 2, 64, 16
    tables, cache, q, qb, par = make_attention(rng, ctx, T, nodes, Hq, H, D, R)
    q[0, 2, 1, 7] = np.nan
    qb[0, 2, 1, 7] = 0x7fc0
    _, _, sc = kvq._code_places(R, D, kvq.row_slot(tables[1], R, cache.shape[1], 20) % R)
    cache[0, kvq.row_slot(tables[1], R, cache.shape[1], 20) // R, 1, sc[1][0]] = 255                # V of head 1, the first 32 values
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device="cuda")
    got = b.radar_tree_attention_kvq(bf16_dev(qb), gpu_cache(cache, R, D), dev(tables), dev(ctx), dev(par), dev(nodes), lse_out=lse)
    with np.errstate(invalid="ignore"):
        check_attention(q, cache, R, D, 0, tables, ctx, par, nodes, got, lse)
    assert torch.isnan(got[1, :, 2:, :32].float()).all() and not torch.isnan(got[1, :, :, 32:].float()).any()


def test_rows_that_are_not_there():
    """Sequences that have ended, prefixes longer than S_max, blocks out of range, rows that may see nothing."""
    b, rng = binding(), seed(84)
    ctx, T, nodes, Hq, H, D, R = np.array([-1, 90, 60, 2 ** 31 - 1, 30, 40], np.int32), 6, np.array([6, 6, 0, 6, 99, 6], np.int32), 4, 2, 128, 16
    tables, cache, q, qb, par = make_attention(rng, np.minimum(ctx, 90), T, np.full(6, T), Hq, H, D, R)
    tables[2, 1], tables[2, 3] = -1, cache.shape[1]
    tables[5] = rng.choice([-1, 1 << 30, cache.shape[1]], tables.shape[1])
    c = gpu_cache(cache, R, D)
    for S in (96, 40, 1):
        lse = torch.full(q.shape[:3], 7.0, dtype=torch.float32, device="cuda")
        out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        b.radar_tree_attention_kvq(bf16_dev(qb), c, dev(tables), dev(ctx), dev(par), dev(nodes), out=out, lse_out=lse, S_max=S)
        check_attention(q, cache, R, D, 0, tables, ctx, par, nodes, out, lse, S_max=S)
        assert (out[0] == 0).all() and (lse[0] == 0).all()
        assert (out[5] == 0).all() and torch.isneginf(lse[5]).all()
    bad = par.copy()
    bad[1] = [5, 0, 7, -9, 3, 5]                                     # parents that are not earlier rows end the chain
    out = b.radar_tree_attention_kvq(bf16_dev(qb), c, dev(tables), dev(ctx), dev(bad), dev(nodes), lse_out=lse, S_max=96)
    check_attention(q, cache, R, D, 0, tables, ctx, bad, nodes, out, lse, S_max=96)


def test_far_scores_and_equal_rows():
    """Scores thousands apart, and a row repeated: the probabilities are exact ones and equal shares."""
    b, rng = binding(), seed(85)
    ctx, T, nodes, Hq, H, D, R = np.array([140], np.int32), 2, np.array([2], np.int32), 2, 1, 128, 16
    tables, cache, q, qb, par = make_attention(rng, ctx, T, nodes, Hq, H, D, R)
    q, qb = bf16(q * 300)
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device="cuda")
    for _ in range(2):
        got = b.radar_tree_attention_kvq(bf16_dev(qb), gpu_cache(cache, R, D), dev(tables), dev(ctx), dev(par), dev(nodes), lse_out=lse)
        out_r, lse_r, spread, reach = kvq.attention(q, cache, R, D, 0, tables, ctx, par, nodes, want_sizes=True)
        # a score of thousands is off by (D + 8) 2^-24 of its terms, and a probability by as much, relative to itself
        slack = (D + 8) * 2.0 ** -24 * reach
        assert (np.abs(host(got.double()) - out_r) <= 2.0 ** -8 * (spread + np.abs(out_r) + 2.0 ** -8 * spread) + 2 * (slack[..., None] + 2.0 ** -14) * spread.max() * 2).all()
        assert (np.abs(host(lse.double()) - lse_r) <= slack + 2.0 ** -19 * (1 + np.abs(lse_r))).all()
        for j in range(142):                                         # second time: all rows alike
            at = kvq.row_slot(tables[0], R, cache.shape[1], j)
            kvq.put_raw(cache, R, D, 0, at, kvq.raw(cache, R, D, 0, kvq.row_slot(tables[0], R, cache.shape[1], 0)))


# ------------------------------------------------------------------ large caches, streams, graphs, a run of all

def test_blocks_beyond_four_gigabytes():
    """Rows at the far end of a cache of 4.6 GB: offsets of more than 32 bits in every call."""
    b, rng = binding(), seed(90)
    H, D, R, T = 8, 128, 16, 4
    n_blocks = 264_000
    c = b.KvqCache(n_blocks, R, H, D)
    assert c.data.numel() > 1 << 32
    ids = np.array([n_blocks - 1, n_blocks - 7, 250_001, 3], np.int32)
    table = ids[None].copy()
    ctx = np.array([40], np.int32)
    x = bf16(rng.normal(size=(2, 44, H, D)))
    slots = np.array([ids[j // R] * R + j % R for j in range(44)], np.int32)
    b.radar_kvq_append(c, bf16_dev(x[1][0]), bf16_dev(x[1][1]), dev(slots))
    small = np.zeros((1, 4, H, kvq.chunk_bytes(R, D)), np.uint8)
    order = np.arange(4, dtype=np.int32)[None]
    for j in range(44):
        kvq.put(small, R, D, 0, j, x[0][0][j], x[0][1][j])
    assert np.array_equal(host(c.data[0, torch.from_numpy(ids).long()]), small[0])
    k, v = b.radar_kvq_read(c, dev(slots))
    for n in range(44):
        assert np.array_equal(host(k[0, n].double()), kvq.get(small, R, D, 0, n)[0]) and np.array_equal(host(v[0, n].double()), kvq.get(small, R, D, 0, n)[1])
    q, qb = bf16(rng.normal(size=(1, T, 16, D)))
    par, nodes = random_parents(rng, 1, T, [T]), np.array([T], np.int32)
    lse = torch.empty((1, T, 16), dtype=torch.float32, device="cuda")
    got = b.radar_tree_attention_kvq(bf16_dev(qb), c, dev(table), dev(ctx), dev(par), dev(nodes), lse_out=lse)
    check_attention(q, small, R, D, 0, order, ctx, par, nodes, got, lse)
    path, n = np.array([[0, 2, 3]], np.int32), np.array([2], np.int32)
    b.radar_kvq_commit(c, dev(table), dev(ctx), dev(n), dev(path))
    small, _ = kvq.commit(small, R, D, order, ctx, n, path)
    assert np.array_equal(host(c.data[0, torch.from_numpy(ids).long()]), small[0])
    del c
    torch.cuda.empty_cache()


class Serving:
    """A batch's verification passes over two layers as a serving loop makes them, and the same by the oracle."""

    def __init__(self, rng, B=3, T=12, Hq=8, H=2, D=64, R=16, M=9, n_blocks=40, layers=2):
        self.b, self.rng, self.shape = binding(), rng, (B, T, Hq, H, D, R, M, n_blocks, layers)
        b = self.b
        self.cache = b.KvqCache(n_blocks, R, H, D, layers=layers)
        self.tables = b.KvqTables(B, M, n_blocks, R)
        z = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")                                                             # noqa: E731
        h = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16, device="cuda")                                                          # noqa: E731
        self.ctx, self.nodes, self.parents, self.len, self.path = z(B), z(B), z(B, T), z(B), z(B, T)
        self.slots, self.granted, self.new_ctx = z(B, T), z(B), z(B)
        self.q, self.out = h(layers, B, T, Hq, D), h(layers, B, T, Hq, D)
        self.lse = torch.zeros((layers, B, T, Hq), device="cuda")
        self.k, self.v = h(layers, B, T, H, D), h(layers, B, T, H, D)
        self.ws = b.new_workspace(b.radar_tree_attention_kvq_workspace_bytes(b.kvq_attn_desc(self.q[0], self.cache, M)))
        self.h_cache = np.zeros(tuple(self.cache.data.shape), np.uint8)
        self.h_tables = (host(self.tables.block_tables), host(self.tables.owned), host(self.tables.free_blocks), n_blocks)

    def calls(self):
        b, (B, T, Hq, H, D, R, M, n_blocks, layers) = self.b, self.shape
        b.radar_kvq_blocks(self.ctx, self.tables, T, n_new=self.nodes, slots=self.slots, granted=self.granted)
        for layer in range(layers):
            b.radar_kvq_append(self.cache, self.k[layer], self.v[layer], self.slots, layer=layer)
            b.radar_tree_attention_kvq(self.q[layer], self.cache, self.tables.block_tables, self.ctx, self.parents, self.nodes, layer=layer,
                                       out=self.out[layer], lse_out=self.lse[layer], workspace=self.ws)
        b.radar_kvq_commit(self.cache, self.tables.block_tables, self.ctx, self.len, self.path, new_ctx_lens=self.new_ctx)
        self.ctx.copy_(self.new_ctx)

    def new_inputs(self, ended=()):
        rng, (B, T, Hq, H, D, R, M, n_blocks, layers) = self.rng, self.shape
        x = {}
        x["nodes"] = rng.integers(1, T + 1, B).astype(np.int32)
        x["parents"] = random_parents(rng, B, T, x["nodes"])
        x["len"], x["path"] = np.zeros(B, np.int32), np.full((B, T), -1, np.int32)
        for bb in range(B):
            way, i = [], int(rng.integers(0, x["nodes"][bb]))
            while i > 0:
                way.append(i)
                i = int(x["parents"][bb, i])
            x["len"][bb], x["path"][bb, :len(way) + 1] = len(way), [0] + way[::-1]
        for n, shape in (("q", (layers, B, T, Hq, D)), ("k", (layers, B, T, H, D)), ("v", (layers, B, T, H, D))):
            x[n], bits = bf16(rng.normal(size=shape))
            getattr(self, n).copy_(bf16_dev(bits))
        for n in ("nodes", "parents", "len", "path"):
            getattr(self, n).copy_(dev(x[n]))
        for bb in ended:
            self.ctx[bb] = -1
        x["ctx"] = host(self.ctx).copy()
        return x

    def check(self, x):
        B, T, Hq, H, D, R, M, n_blocks, layers = self.shape
        tables, owned, free, n_free = self.h_tables
        slots, granted, owned, n_free, tables, free = kvq.blocks(x["ctx"], x["nodes"], tables, owned, free, n_free, R, T)
        self.h_tables = (tables, owned, free, n_free)
        assert np.array_equal(host(self.slots), slots) and np.array_equal(host(self.granted), granted) and np.array_equal(host(self.tables.block_tables), tables)
        assert granted.all()
        for layer in range(layers):
            for bb in range(B):
                for i in range(T):
                    kvq.put(self.h_cache, R, D, layer, int(slots[bb, i]), x["k"][layer, bb, i], x["v"][layer, bb, i])
            check_attention(x["q"][layer], self.h_cache, R, D, layer, tables, x["ctx"], x["parents"], x["nodes"], self.out[layer], self.lse[layer])
        self.h_cache, new = kvq.commit(self.h_cache, R, D, tables, x["ctx"], x["len"], x["path"])
        assert np.array_equal(host(self.new_ctx), new) and np.array_equal(host(self.ctx), new)
        assert np.array_equal(host(self.cache.data), self.h_cache)


def test_verification_passes_in_a_row():
    s = Serving(seed(91))
    for n in range(9):
        x = s.new_inputs(ended=(n % 3,) if n % 4 == 3 else ())
        s.calls()
        s.check(x)
        if n % 4 == 3:                                               # a new request takes the ended one's place
            s.ctx[n % 3] = 0


def test_a_captured_pass_is_replayed():
    """The pass as a graph, replayed with other inputs between eager passes over the same buffers."""
    s = Serving(seed(92))
    x = s.new_inputs()
    s.calls()                                                        # the first call of each entry point is made outside a capture
    torch.cuda.synchronize()
    s.check(x)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.calls()
    for n in range(6):
        x = s.new_inputs()
        g.replay() if n != 2 else s.calls()
        torch.cuda.synchronize()
        s.check(x)


def test_two_streams_with_workspaces_of_their_own():
    a, c = Serving(seed(93)), Serving(seed(94), B=2, T=5, D=128, R=32)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        xs = [s.new_inputs() for s in (a, c)]
        torch.cuda.synchronize()
        for s, st in zip((a, c), streams):
            with torch.cuda.stream(st):
                s.calls()
        torch.cuda.synchronize()
        for s, x in zip((a, c), xs):
            s.check(x)


def test_prepared_calls_are_the_same_calls():
    b, rng = binding(), seed(95)
    ctx, T, nodes, Hq, H, D, R = np.array([77], np.int32), 8, np.array([8], np.int32), 8, 2, 128, 16
    tables, cache, q, qb, par = make_attention(rng, ctx, T, nodes, Hq, H, D, R)
    args = (bf16_dev(qb), gpu_cache(cache, R, D), dev(tables), dev(ctx), dev(par), dev(nodes))
    call = b.radar_tree_attention_kvq(*args, prepared=True)
    want = b.radar_tree_attention_kvq(*args)
    for _ in range(3):
        call.out.zero_()
        assert call() is call.out and torch.equal(call.out, want)


def test_direct_calls_by_the_native_half(monkeypatch):
    """Direct calls whose buffers are all given are marshalled natively; they do what ctypes makes them do.  What the native half does not take
    reaches the other's checks."""
    from test_gpu_support import _Both
    b, rng = binding(), seed(96)
    both = _Both(b, monkeypatch)
    ctx, T, nodes, Hq, H, D, R = np.array([77, 31], np.int32), 8, np.array([8, 5], np.int32), 8, 2, 128, 16
    tables, cache, q, qb, par = make_attention(rng, ctx, T, nodes, Hq, H, D, R, layers=3)
    M, n_blocks = tables.shape[1], cache.shape[1]
    fused = torch.randn((2, T, Hq + 2 * H, D), device="cuda").bfloat16()
    fused[:, :, :Hq] = bf16_dev(qb)
    dq, dk, dv, dt, dc, dp, dn = fused[:, :, :Hq], fused[:, :, Hq:Hq + H], fused[:, :, Hq + H:], dev(tables), dev(ctx), dev(par), dev(nodes)
    slots = dev(np.stack([[kvq.row_slot(tables[bb], R, n_blocks, int(ctx[bb]) + i) for i in range(T)] for bb in range(2)]).astype(np.int32))
    wide = torch.zeros((3, cache[0].size + 64), dtype=torch.uint8, device="cuda")

    def fresh(spread=False):
        if not spread:
            return gpu_cache(cache, R, D)
        wide[:, :cache[0].size] = dev(cache.reshape(3, -1))
        return b.KvqCache(data=wide[:, :cache[0].size].view(cache.shape), block_rows=R, D=D)

    for spread in (False, True):
        for k, v in ((dk, dv), (dk.contiguous(), dv.contiguous()), (dk[:1, 3:4], dv[:1, 3:4])):
            def append():
                c = fresh(spread)
                assert b.radar_kvq_append(c, k, v, slots.view(-1)[:k.shape[0] * k.shape[1]], layer=1) is c
                return [c.data.clone()]
            both("append", append)

        def commit():
            c, new = fresh(spread), torch.full((2,), 9, dtype=torch.int32, device="cuda")
            path = dev(np.array([[0, 2, 5], [0, 3, 4]], np.int32))
            assert b.radar_kvq_commit(c, dt, dc, dev(np.array([2, 1], np.int32)), path, new_ctx_lens=new) is new
            return [c.data.clone(), new]
        both("commit", commit)
        c = fresh(spread)
        ws = b.new_workspace(b.radar_tree_attention_kvq_workspace_bytes(b.kvq_attn_desc(dq, c, M, rows_per_split=64)))
        room = torch.zeros((2, Hq, T, D), dtype=torch.bfloat16, device="cuda")
        for parents, n, S, out, split, scale in ((dp, dn, None, None, 0, 0.0), (dp, dn, 90, "own", 64, 0.2), (None, None, 90, None, 64, 0.0)):
            def attend():
                lse = torch.full((2, T, Hq), 7.0, device="cuda")
                o = room.zero_().transpose(1, 2) if out else None
                got = b.radar_tree_attention_kvq(dq, c, dt, dc, parents, n, layer=2, S_max=S, out=o, lse_out=lse, workspace=ws, rows_per_split=split,
                                                 softmax_scale=scale)
                assert o is None or got is o
                return [got.clone(), lse]
            both("attention", attend)

    def blocks():
        t = b.KvqTables(2, M, n_blocks, R)
        s, g = torch.full((2, T), 5, dtype=torch.int32, device="cuda"), torch.full((2,), 5, dtype=torch.int32, device="cuda")
        got = b.radar_kvq_blocks(dc, t, T, n_new=dn, slots=s, granted=g)
        assert got[0] is s and got[1] is g
        return [s, g, t.block_tables, t.owned, t.free_blocks, t.n_free]
    both("blocks", blocks)
    both.native = True
    c = fresh()
    for bad in (lambda: b.radar_kvq_append(c, dk.float(), dv.float(), slots), lambda: b.radar_kvq_append(c, dk, dv, slots[:1]),
                lambda: b.radar_kvq_append(c, dk, dv, slots, layer=3), lambda: b.radar_kvq_append(c, dk[:1].expand(2, T, H, D), dv[:1].expand(2, T, H, D), slots),
                lambda: b.radar_kvq_commit(c, dt, dc[:1], dc, slots, new_ctx_lens=dn), lambda: b.radar_tree_attention_kvq(dq, c, dt, dc, dp[:, :3], dn, workspace=ws),
                lambda: b.radar_tree_attention_kvq(dq[:1].expand(2, T, Hq, D), c, dt, dc, dp, dn, workspace=ws),
                lambda: b.radar_kvq_blocks(dc, b.KvqTables(3, M, n_blocks, R), T, slots=slots, granted=dn)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(b.RadarError):
        b.radar_tree_attention_kvq(dq, c, dt, dc, dp, dn, S_max=M * R + 1, workspace=ws)
