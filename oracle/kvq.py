"""The paged 4-bit key/value cache from its definition (include/radar.h), in numpy and 64 bits.

Keys and values travel as float64 rows [n, Hkv, D]; a cache is uint8 [layers, n_blocks, Hkv, chunk].  Slow and plain: every
position is computed on its own, nothing is shared with the HIP package.
"""
import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def chunk_bytes(R, D):
    return R * (D + D // 16)


def encode(x):
    """x float64 [..., D] -> codes uint8 [..., D] (one a byte), scale bytes uint8 [..., D/32]."""
    blk = np.asarray(x, np.float64).reshape(x.shape[:-1] + (-1, 32))
    bad = ~np.isfinite(blk).all(-1)
    amax = np.where(bad, 0.0, np.abs(np.where(np.isfinite(blk), blk, 0.0)).max(-1))
    e = np.full(amax.shape, -126)
    for cand in range(-126, 125):                                    # the smallest with amax < 7 * 2^e
        e = np.where(amax >= 7.0 * 2.0 ** cand, cand + 1, e)
    y = np.where(bad[..., None], 0.0, np.where(np.isfinite(blk), blk, 0.0)) / (2.0 ** e.astype(np.float64))[..., None]
    dist = np.abs(np.abs(y)[..., None] - MAGNITUDES)
    near = dist.min(-1, keepdims=True)
    even = np.where(dist == near, np.arange(8) % 2, 2)               # ties: the even code
    code = even.argmin(-1).astype(np.uint8) | (np.signbit(y).astype(np.uint8) << 3)
    return code.reshape(x.shape), np.where(bad, 255, e + 127).astype(np.uint8)


def decode(codes, scales):
    v = MAGNITUDES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    f = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127.0))
    return (v.reshape(v.shape[:-1] + (-1, 32)) * f[..., None]).reshape(v.shape)


def _code_places(R, D, row):
    """Byte and half of every d of a row, of K and of V; bytes of its scales."""
    d = np.arange(D)
    k = row * (D // 2) + d // 2
    v = R * D // 2 + ((row // 8 * (D // 8) + d // 8) * 8 + row % 8) * 4 + d % 8 // 2
    b = np.arange(D // 32)
    s = (row // 8 * (D // 32) + b) * 8 + row % 8
    return (k, v), d % 2, (R * D + s, R * D + R * D // 32 + s)


def put(cache, R, D, layer, slot, k, v):
    """One row k, v float64 [Hkv, D] at a slot; out of range: nothing."""
    if not 0 <= slot < cache.shape[1] * R:
        return
    places, half, sc = _code_places(R, D, slot % R)
    for x, at, s_at in zip((k, v), places, sc):
        codes, scales = encode(x)
        for h in range(cache.shape[2]):
            chunk = cache[layer, slot // R, h]
            byte = chunk[at]
            for side in (0, 1):
                pick = half == side
                byte = chunk[at]
                byte[pick] = (byte[pick] & (0xf0 if side == 0 else 0x0f)) | (codes[h][pick] << (4 * side))
                chunk[at[pick]] = byte[pick]
            chunk[s_at] = scales[h]


def get(cache, R, D, layer, slot):
    """(k, v) float64 [Hkv, D] at a slot; zeros if it is out of range."""
    H = cache.shape[2]
    if not 0 <= slot < cache.shape[1] * R:
        return np.zeros((H, D)), np.zeros((H, D))
    places, half, sc = _code_places(R, D, slot % R)
    chunk = cache[layer, slot // R]
    return tuple(decode((chunk[:, at] >> (4 * half).astype(np.uint8)) & 15, chunk[:, s_at]) for at, s_at in zip(places, sc))


def raw(cache, R, D, layer, slot):
    """A row's bytes in all heads, as a list that `put_raw` takes."""
    places, _, sc = _code_places(R, D, slot % R)
    at = np.unique(np.concatenate(places + sc))
    return cache[layer, slot // R][:, at].copy()


def put_raw(cache, R, D, layer, slot, data):
    places, _, sc = _code_places(R, D, slot % R)
    cache[layer, slot // R][:, np.unique(np.concatenate(places + sc))] = data


def blocks(ctx, new, tables, owned, free, n_free, R, T):
    """(slots, granted, owned, n_free, tables, free) after the call; inputs are left alone."""
    tables, owned, free = tables.copy(), owned.copy(), free.copy()
    B, M = tables.shape
    new = [min(max(int(n), 0), T) for n in (np.full(B, T) if new is None else new)]
    want = [0 if c < 0 else -(-(int(c) + n) // R) for c, n in zip(ctx, new)]
    for b in range(B):
        if want[b] <= M:
            for i in range(want[b], owned[b]):
                free[n_free] = tables[b, i]
                n_free += 1
            owned[b] = min(owned[b], want[b])
    granted, short, asked = np.zeros(B, np.int32), False, 0
    there = n_free
    for b in range(B):
        if want[b] > M:
            continue
        need = want[b] - owned[b]
        asked += need
        if need and asked > there:
            continue
        granted[b] = 1
        for i in range(owned[b], want[b]):
            n_free -= 1
            tables[b, i] = free[n_free]
        owned[b] = want[b]
    tables[(granted == 0)[:, None] & (np.arange(M) >= np.minimum(owned, M)[:, None])] = -1
    slots = np.full((B, T), -1, np.int32)
    for b in range(B):
        if granted[b] and ctx[b] >= 0:
            for i in range(new[b]):
                j = int(ctx[b]) + i
                slots[b, i] = tables[b, j // R] * R + j % R if 0 <= tables[b, j // R] < len(free) else -1
    return slots, granted, owned, n_free, tables, free


def row_slot(table, R, n_blocks, j):
    """Slot of row j of a sequence, -1 if it is not there."""
    if not 0 <= j // R < len(table) or not 0 <= table[j // R] < n_blocks:
        return -1
    return int(table[j // R]) * R + j % R


def commit(cache, R, D, tables, ctx, accept_len, path):
    """(cache, new_ctx) after the call."""
    new, P = cache.copy(), path.shape[1]
    ctx_out = ctx.copy()
    for b in range(len(ctx)):
        if ctx[b] < 0:
            continue
        n = min(max(int(accept_len[b]), 0), P - 1)
        ctx_out[b] = ctx[b] + n + 1
        for layer in range(cache.shape[0]):
            for s in range(1, n + 1):
                p = int(path[b, s])
                src, dst = (row_slot(tables[b], R, cache.shape[1], int(ctx[b]) + x) for x in (p, s))
                if 0 <= p < 64 and src >= 0 and dst >= 0:
                    put_raw(new, R, D, layer, dst, raw(cache, R, D, layer, src))
    return new, ctx_out


def attention(q, cache, R, D, layer, tables, ctx, parents=None, n_nodes=None, S_max=None, scale=0.0, want_sizes=False):
    """q float64 [B,T,Hq,D] -> out float64 [B,T,Hq,D], lse [B,T,Hq].  A hidden row has no influence; a row of NaN that is seen has.
    want_sizes: also the sums of magnitudes that rounding errors are relative to: sum_j p_j |v_j| [B,T,Hq,D], max_j scale sum_d |q k| [B,T,Hq]."""
    B, T, Hq, _ = q.shape
    H, n_blocks = cache.shape[2], cache.shape[1]
    S_max = tables.shape[1] * R if S_max is None else S_max
    scale = scale or 1.0 / np.sqrt(D)
    out, lse = np.zeros(q.shape), np.zeros((B, T, Hq))
    spread, reach = np.zeros(q.shape), np.zeros((B, T, Hq))
    for b in range(B):
        if ctx[b] < 0:
            continue
        L = min(int(ctx[b]), S_max)
        nn = T if n_nodes is None else max(1, min(int(n_nodes[b]), T))
        rows = [j for j in range(min(L + nn, S_max)) if row_slot(tables[b], R, n_blocks, j) >= 0]
        kv = [get(cache, R, D, layer, row_slot(tables[b], R, n_blocks, j)) for j in rows]
        where = {j: n for n, j in enumerate(rows)}
        K = np.array([x[0] for x in kv]).reshape(len(rows), H, D)
        V = np.array([x[1] for x in kv]).reshape(len(rows), H, D)
        prefix = [where[j] for j in rows if j < L]
        for i in range(nn):
            mine, a = list(prefix), i
            while a >= 0:
                if L + a in where:
                    mine.append(where[L + a])
                p = a - 1 if parents is None else int(parents[b, a])
                a = p if 0 <= p < a else -1
            for h in range(Hq):
                g = h // (Hq // H)
                if not mine:
                    lse[b, i, h] = -np.inf
                    continue
                x = scale * (K[mine, g] @ q[b, i, h])
                top = x.max()
                w = np.exp(x - top)
                out[b, i, h] = (w / w.sum()) @ V[mine, g]
                lse[b, i, h] = top + np.log(w.sum())
                if want_sizes:
                    spread[b, i, h] = (w / w.sum()) @ np.abs(V[mine, g])
                    reach[b, i, h] = scale * (np.abs(K[mine, g]) @ np.abs(q[b, i, h])).max()
    return (out, lse, spread, reach) if want_sizes else (out, lse)


# ------------------------------------------------------------------ rotary positions, chunks of new tokens

def new_rows(B, T, ctx=None, row_starts=None, n_new=None, N=None):
    """(row of the tensors, sequence, row of it) of every new row that there is: [B,T], or one sequence's behind the other's from row_starts[b] on."""
    got = []
    for b in range(B):
        if ctx is not None and ctx[b] < 0:
            continue
        if row_starts is None:
            got += [(b * T + i, b, i) for i in range(T if n_new is None else min(max(int(n_new[b]), 0), T))]
        else:
            got += [(int(row_starts[b]) + i, b, i) for i in range(min(int(row_starts[b + 1]) - int(row_starts[b]), T))]
    return got


def turn(x, position, inv_freq, pair_axis, interleaved=False, scale=1.0):
    """One row x float64 [H, D] turned by its positions (whole numbers, one an axis), before any rounding; inv_freq float32 [P]."""
    P = len(inv_freq)
    t = np.array([float(position[a]) for a in pair_axis]) * inv_freq.astype(np.float64)
    c, s = np.cos(t) * scale, np.sin(t) * scale
    out = np.array(x, np.float64)
    one, two = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if interleaved else (slice(0, P), slice(P, 2 * P))
    out[:, one], out[:, two] = x[:, one] * c - x[:, two] * s, x[:, one] * s + x[:, two] * c
    return out


def all_rows(cache, R, D, layer, table, n):
    """Rows 0 ... n-1 of a sequence as float64 K, V [n, H, D], and which of them are there (the others: zeros)."""
    j = np.arange(n)
    blk = np.asarray(table)[np.minimum(j // R, len(table) - 1)]
    there = (j // R < len(table)) & (blk >= 0) & (blk < cache.shape[1])
    chunk = cache[layer, np.where(there, blk, 0)]                    # [n, H, bytes]
    got = [np.zeros((n, cache.shape[2], D)) for _ in range(2)]
    for row in range(R):
        mine = np.nonzero(j % R == row)[0]
        if len(mine) == 0:
            continue
        places, half, sc = _code_places(R, D, row)
        for x, at, s_at in zip(got, places, sc):
            x[mine] = decode((chunk[mine][:, :, at] >> (4 * half).astype(np.uint8)) & 15, chunk[mine][:, :, s_at])
    for x in got:
        x[~there] = 0.0
    return got[0], got[1], there


def chunk_attention(q, cache, R, D, layer, tables, ctx, T, row_starts=None, n_new=None, S_max=None, scale=0.0):
    """q float64 [N,Hq,D] -> out float64 [N,Hq,D], lse [N,Hq], sum_j p_j |v_j| [N,Hq,D], max_j scale sum_d |q k| [N,Hq], and which rows are there.  Row i of
    sequence b sees rows up to ctx[b] + i of its own."""
    N, Hq, _ = q.shape
    H = cache.shape[2]
    scale = scale or 1.0 / np.sqrt(D)
    S_max = tables.shape[1] * R if S_max is None else S_max
    out, lse, spread, reach, there = np.zeros(q.shape), np.zeros((N, Hq)), np.zeros(q.shape), np.zeros((N, Hq)), np.zeros(N, bool)
    rows = new_rows(len(ctx), T, ctx, row_starts, n_new)
    for b in range(len(ctx)):
        mine = np.array([(n, i) for n, bb, i in rows if bb == b], np.int64).reshape(-1, 2)
        if len(mine) == 0:
            continue
        n_at, i_of = mine.T
        there[n_at] = True
        S = min(int(ctx[b]) + int(i_of.max()) + 1, S_max)
        K, V, have = all_rows(cache, R, D, layer, tables[b], S)
        sees = (np.arange(S)[None] <= int(ctx[b]) + i_of[:, None]) & have
        for h in range(Hq):
            k, v = K[:, h // (Hq // H)], V[:, h // (Hq // H)]
            with np.errstate(invalid="ignore", divide="ignore"):
                x = np.where(sees, scale * (q[n_at, h] @ k.T), -np.inf)
                top = np.where(sees.any(1), x.max(1), 0.0)
                w = np.where(sees, np.exp(x - top[:, None]), 0.0)
                total = w.sum(1)
                lse[n_at, h] = top + np.log(total)
                w = w / np.where(total == 0, 1.0, total)[:, None]
                bad = np.isnan(v)
                o = w @ np.where(bad, 0.0, v)
                out[n_at, h] = np.where((sees.astype(float) @ bad) > 0, np.nan, o)
                spread[n_at, h] = w @ np.abs(np.where(bad, 0.0, v))
                reach[n_at, h] = np.where(sees, scale * (np.abs(q[n_at, h]) @ np.abs(k).T), 0.0).max(1)
    return out, lse, spread, reach, there
