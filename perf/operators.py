"""The paged key/value cache in 4 bits, as measurable cases: its operators in plain form and by the library's calls.

Five kinds of pass:

  attend   one layer of attention over the cache: draft trees to verify, or single tokens
  blocks   block tables and slot maps of a batch from its requests' lengths
  append   rows of keys and values into the cache, and back out of it as the values they stand for
  commit   the accepted paths' rows moved into place in every layer, and the kept rows read back
  step     one layer's whole use of the cache in a verification pass: blocks, append, attend, commit, read

Format.  32 consecutive values of a row share a power of two 2^e and are e2m1 codes (0 .5 1 1.5 2 3 4 6 and a sign); e is the smallest
whole number with amax < 7 * 2^e, within [-126, 125]; codes round to nearest, ties to the even code; byte e + 127 is kept, or 255 for a block
with an infinity or NaN, which stands for 32 NaNs.  A block of R rows of one KV head is R * (D + D / 16) bytes:
K codes [R][D/2], V codes [R/8][D/8][8][4], K scales [R/8][D/32][8], V scales [R/8][D/32][8]; an even element is a byte's low half.

Lengths and tree sizes of a case come from its `shape_seed`, values from prepare()'s seed.
"""
import math
import random

import numpy as np
import torch

own = False

LUT = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def listed():
    return [
        # one new token of a single short conversation on the smallest layer that the repository configures: bound by the call itself
        dict(name="attend_token_small", kind="attend", B=1, T=1, nodes_lo=1, Hq=4, Hkv=1, D=64, R=16, ctx_lo=256, ctx_hi=256, depth=1,
             lse=True, shape_seed=1),
        # plain decoding of a served batch of 64 conversations, a token each: bound by reading the cache
        dict(name="attend_tokens_batch64", kind="attend", B=64, T=1, nodes_lo=1, Hq=32, Hkv=8, D=128, R=16, ctx_lo=512, ctx_hi=8192, depth=1,
             lse=False, shape_seed=2),
        # one layer of an 8B-class target verifying a 60-node tree
        dict(name="attend_tree_8b", kind="attend", B=1, T=60, nodes_lo=60, Hq=32, Hkv=8, D=128, R=32, ctx_lo=2048, ctx_hi=2048, depth=8,
             lse=False, shape_seed=3),
        # a served batch: 16 conversations of different lengths whose drafting stopped at different depths
        dict(name="attend_tree_ragged16", kind="attend", B=16, T=60, nodes_lo=2, Hq=32, Hkv=8, D=128, R=16, ctx_lo=512, ctx_hi=8192, depth=8,
             lse=False, shape_seed=4),
        # long contexts on a 70B-class target, the largest layer configured: bound by the matrix products
        dict(name="attend_tree_70b", kind="attend", B=4, T=60, nodes_lo=60, Hq=64, Hkv=8, D=128, R=64, ctx_lo=16384, ctx_hi=16384, depth=8,
             lse=False, shape_seed=5),
        # a served batch of 16 that grows by a tree each, the pass before every verification
        dict(name="blocks_batch16", kind="blocks", B=16, T=60, nodes_lo=2, R=16, ctx_lo=512, ctx_hi=8192, ended=1, shape_seed=6),
        # a large batch, part of whose requests have ended and give their blocks back
        dict(name="blocks_batch1024", kind="blocks", B=1024, T=8, nodes_lo=1, R=16, ctx_lo=64, ctx_hi=2048, ended=64, shape_seed=7),
        # the rows of one 60-node tree, written by every layer of every verification pass
        dict(name="append_tree", kind="append", N=60, Hq=32, Hkv=8, D=128, R=16, unused=0, shape_seed=8),
        # a long prompt's rows, with an odd number of them, out of a projection's fused output; some rows are padding
        dict(name="append_prompt", kind="append", N=8191, Hq=32, Hkv=8, D=128, R=32, unused=7, shape_seed=9),
        # the accepted path of one sequence in the 32 layers of an 8B-class target
        dict(name="commit_8b", kind="commit", B=1, T=60, layers=32, Hkv=8, D=128, R=16, ctx_lo=500, ctx_hi=500, depth=8, shape_seed=10),
        # the accepted paths of 64 sequences in 80 layers
        dict(name="commit_batch64", kind="commit", B=64, T=60, layers=80, Hkv=8, D=128, R=32, ctx_lo=33, ctx_hi=200, depth=8, shape_seed=11),
        # all of it in a row, as one layer of a verification pass over a served batch makes the calls
        dict(name="step_ragged16", kind="step", B=16, T=60, nodes_lo=2, layers=1, Hq=32, Hkv=8, D=128, R=16, ctx_lo=256, ctx_hi=2048, depth=8,
             ended=0, lse=False, shape_seed=12),
    ]


# ------------------------------------------------------------------ drawn cases

def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _heads(rng):
    Hkv = rng.choice([1, 2, 4, 5, 8])
    return Hkv * rng.choice([1, 2, 4, 5, 8]), Hkv, rng.choice([64, 128, 128])


def _draw_attend(rng):
    while True:
        Hq, Hkv, D = _heads(rng)
        B, hi, T = _log(rng, 1, 64), _log(rng, 1, 16384), rng.choice([1, 1, rng.randint(2, 12), rng.randint(13, 64)])
        lo = max(0, hi if rng.random() < 0.3 else hi // rng.choice([2, 16]))
        if B * hi * Hkv * D <= 64 * 4096 * 1024 and B * hi * Hq * T * D <= 4 * 16384 * 64 * 60 * 128:
            return dict(kind="attend", B=B, T=T, nodes_lo=rng.choice([1, T]), Hq=Hq, Hkv=Hkv, D=D, R=rng.choice([16, 32, 64, 128]), ctx_lo=lo,
                        ctx_hi=hi, depth=rng.randint(1, 10), lse=rng.random() < 0.5, shape_seed=rng.randrange(1 << 20))


def _draw_blocks(rng):
    B = _log(rng, 1, 1024)
    hi = _log(rng, 1, 4096)
    return dict(kind="blocks", B=B, T=rng.randint(1, 64), nodes_lo=1, R=rng.choice([16, 32, 64, 128]), ctx_lo=hi // 4, ctx_hi=hi, ended=B // 8,
                shape_seed=rng.randrange(1 << 20))


def _draw_append(rng):
    Hq, Hkv, D = _heads(rng)
    N = _log(rng, 1, 8191)
    return dict(kind="append", N=N, Hq=Hq, Hkv=Hkv, D=D, R=rng.choice([16, 32, 64, 128]), unused=N // 9, shape_seed=rng.randrange(1 << 20))


def _draw_commit(rng):
    while True:
        _, Hkv, D = _heads(rng)
        B, layers, hi = _log(rng, 1, 64), rng.randint(1, 80), _log(rng, 1, 512)
        if B * layers * Hkv * (hi + 200) <= 64 * 80 * 8 * 300:
            return dict(kind="commit", B=B, T=rng.randint(9, 64), layers=layers, Hkv=Hkv, D=D, R=rng.choice([16, 32, 64, 128]), ctx_lo=hi // 2,
                        ctx_hi=hi, depth=rng.randint(1, 8), shape_seed=rng.randrange(1 << 20))


def _draw_step(rng):
    while True:
        Hq, Hkv, D = _heads(rng)
        B, hi = _log(rng, 1, 32), _log(rng, 1, 4096)
        if B * hi <= 32 * 1024:
            return dict(kind="step", B=B, T=rng.randint(9, 64), nodes_lo=2, layers=1, Hq=Hq, Hkv=Hkv, D=D, R=rng.choice([16, 32, 64, 128]),
                        ctx_lo=hi // 4, ctx_hi=hi, depth=rng.randint(1, 8), ended=0, lse=False, shape_seed=rng.randrange(1 << 20))


def draw(rng):
    return rng.choice([_draw_attend] * 4 + [_draw_blocks, _draw_append, _draw_commit, _draw_step])(rng)


# ------------------------------------------------------------------ shapes of a case

def _lens(c, lo, hi, what):
    """One whole number per sequence, spread over [lo, hi]; the largest is hi."""
    r = random.Random(c["shape_seed"] * 8 + what)
    v = [r.randint(lo, hi) for _ in range(c["B"])]
    v[r.randrange(c["B"])] = hi
    return v


def _ctx(c):
    return _lens(c, c["ctx_lo"], c["ctx_hi"], 0)


def _nodes(c):
    return _lens(c, min(c.get("nodes_lo", c["T"]), c["T"]), c["T"], 1)


def _trees(c):
    """parents [B,T] (-1 behind a tree's end): every node hangs under an earlier one, at most `depth` deep."""
    r = random.Random(c["shape_seed"] * 8 + 2)
    par = np.full((c["B"], c["T"]), -1, np.int32)
    for b, n in enumerate(_nodes(c)):
        level = [0]
        for i in range(1, n):
            p = r.randrange(max(0, i - 20), i)
            while level[p] >= c["depth"]:
                p = int(par[b, p])
            par[b, i] = p
            level.append(level[p] + 1)
    return par


def _paths(c, par):
    """Accepted paths: a way down each tree of which no row moves onto a row that has still to move, so that a pass may be made again."""
    r = random.Random(c["shape_seed"] * 8 + 3)
    length, path = np.zeros(c["B"], np.int32), np.full((c["B"], c["depth"] + 1), -1, np.int32)
    for b, n in enumerate(_nodes(c)):
        best = [0]
        for _ in range(40):
            way, i = [], r.randrange(n)
            while i > 0:
                way.append(i)
                i = int(par[b, i])
            way = [0] + way[::-1]
            if all(p == s or p >= len(way) for s, p in enumerate(way)) and len(way) > len(best):
                best = way
        length[b], path[b, :len(best)] = len(best) - 1, best
    return length, path


def _tables(c, rows, seed):
    """Block tables [B,M] of sequences that hold `rows` rows each, from a pool with a third more blocks in the order that the seed gives;
    free stack and its height."""
    R = c["R"]
    need = [-(-n // R) for n in rows]
    M = max(max(need), -(-(c["ctx_hi"] + c["T"]) // R)) + 1
    n_blocks = sum(need) + max(4, sum(need) // 3) + c["B"] * (-(-c["T"] // R) + 1)
    ids = list(range(n_blocks))
    random.Random(c["shape_seed"] * 65537 + int(seed)).shuffle(ids)
    table, at = np.full((c["B"], M), -1, np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    free = np.full(n_blocks, -1, np.int32)
    free[:n_blocks - at] = ids[at:]
    return table, np.array(need, np.int32), free, n_blocks - at, n_blocks


# ------------------------------------------------------------------ the format in plain torch

def _sections(cache, R, D):
    """Views of cache [..., n_blocks, H, bytes]: K codes [..., H, R, D/2], V codes [..., H, R/8, D/8, 8, 4], scales [..., H, R/8, D/32, 8]."""
    lead, half, sc = list(cache.shape[:-1]), R * D // 2, R * D // 32
    return (cache[..., :half].unflatten(-1, (R, D // 2)), cache[..., half:2 * half].unflatten(-1, (R // 8, D // 8, 8, 4)),
            cache[..., 2 * half:2 * half + sc].unflatten(-1, (R // 8, D // 32, 8)), cache[..., 2 * half + sc:].unflatten(-1, (R // 8, D // 32, 8)))


def _encode(x):
    """x float32 [..., D] -> codes u8 [..., D/2], scale bytes u8 [..., D/32]."""
    blk = x.unflatten(-1, (-1, 32))
    amax = blk.abs().amax(-1)
    sound = torch.isfinite(blk).all(-1)
    m, up = torch.frexp(torch.where(sound, amax, torch.ones_like(amax)))        # amax = m * 2^up, .5 <= m < 1
    e = torch.where(m < 0.875, up - 3, up - 2)
    e = torch.where(amax == 0, torch.full_like(e, -126), e).clamp(-126, 125)
    y = torch.where(sound[..., None], torch.ldexp(blk, -e[..., None]), torch.zeros_like(blk))
    a = y.abs()
    code = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int() + (a > 5.0).int())
    code = (code | (torch.signbit(y).int() << 3)).flatten(-2)
    packed = (code[..., 0::2] | (code[..., 1::2] << 4)).to(torch.uint8)
    return packed, torch.where(sound, e + 127, torch.full_like(e, 255)).to(torch.uint8)


def _decode(codes, scales):
    """codes u8 [..., D/2], scale bytes u8 [..., D/32] -> float32 [..., D]."""
    lut = torch.tensor(LUT + [-v for v in LUT], dtype=torch.float32, device=codes.device)
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    x = lut[c.int()].unflatten(-1, (-1, 32))
    f = torch.where(scales == 255, torch.full_like(scales, 0, dtype=torch.float32) + float("nan"),
                    torch.ldexp(torch.ones((), device=codes.device), scales.int() - 127))
    return (x * f[..., None]).flatten(-2)


def _get(cache, R, D, blk, row):
    """K and V codes and scales of rows (blk, row), both [n]: each [L, n, H, ...]; cache [L, n_blocks, H, bytes]."""
    kc, vc, ks, vs = _sections(cache, R, D)
    r8, r1 = row // 8, row % 8
    k = kc[:, blk, :, row]                                           # the indexed axes come first: [n, L, H, D/2]
    v = vc[:, blk, :, r8, :, r1].flatten(-2)
    return [t.transpose(0, 1) for t in (k, v, ks[:, blk, :, r8, :, r1], vs[:, blk, :, r8, :, r1])]


def _put(cache, R, D, blk, row, parts):
    kc, vc, ks, vs = _sections(cache, R, D)
    r8, r1 = row // 8, row % 8
    k, v, a, b = [t.transpose(0, 1) for t in parts]
    kc[:, blk, :, row] = k
    vc[:, blk, :, r8, :, r1] = v.unflatten(-1, (-1, 4))
    ks[:, blk, :, r8, :, r1] = a
    vs[:, blk, :, r8, :, r1] = b


# ------------------------------------------------------------------ the operators in plain torch

def _plain_blocks(s):
    R, M, n_blocks, T = s["R"], s["table"].shape[1], s["free"].numel(), s["T"]
    ctx, new, owned, n_free = s["ctx"].long(), s["nodes"].long(), s["owned"].long(), s["n_free"].long()
    want = torch.where(ctx < 0, torch.zeros_like(ctx), (ctx + new + R - 1) // R)
    fits = want <= M
    freed = torch.where(fits, (owned - want).clamp(min=0), torch.zeros_like(want))
    need = torch.where(fits, (want - owned).clamp(min=0), torch.zeros_like(want))
    there = (n_free + freed.sum()).clamp(max=n_blocks)
    granted = fits & ((need == 0) | (need.cumsum(0) <= there))
    at = torch.arange(M, device=ctx.device)[None]
    goes = (at >= want[:, None]) & (at < owned[:, None]) & fits[:, None]
    to = torch.where(goes, n_free + goes.flatten().cumsum(0).view_as(goes) - 1, torch.full_like(at, n_blocks)).clamp(max=n_blocks)
    stack = torch.cat((s["free"], s["free"][:1]))
    stack.scatter_(0, to.flatten(), s["table"].flatten())
    s["free"].copy_(stack[:n_blocks])
    comes = (at >= owned[:, None]) & (at < want[:, None]) & granted[:, None]
    rank = comes.flatten().cumsum(0).view_as(comes) - 1
    s["table"].copy_(torch.where(comes, s["free"][(there - 1 - rank).clamp(0, n_blocks - 1)], s["table"]))
    i = torch.arange(T, device=ctx.device)[None]
    pos = (ctx[:, None] + i).clamp(min=0)
    slot = s["table"].gather(1, (pos // R).clamp(max=M - 1)).long() * R + pos % R
    slots = torch.where((i < new[:, None]) & granted[:, None] & (ctx >= 0)[:, None], slot, torch.full_like(slot, -1)).int()
    owned_out = torch.where(granted, want, owned).int()
    return [slots, granted.int(), owned_out, (there - (need * granted).sum()).int().view(1), s["table"], s["free"]]


def _plain_append(s, slots):
    R, D = s["R"], s["D"]
    keep = slots.flatten() >= 0
    at = slots.flatten()[keep].long()
    k, ks = _encode(s["k"].flatten(0, -3)[keep].float())
    v, vs = _encode(s["v"].flatten(0, -3)[keep].float())
    _put(s["cache"], R, D, at // R, at % R, [t[None] for t in (k, v, ks, vs)])


def _plain_read(s, slots):
    at = slots.flatten().long()
    k, v, ks, vs = _get(s["cache"], s["R"], s["D"], at.clamp(min=0) // s["R"], at.clamp(min=0) % s["R"])
    keep = (at >= 0)[None, :, None, None]
    return [torch.where(keep, _decode(c, f), torch.zeros((), device=c.device)).to(torch.bfloat16) for c, f in ((k, ks), (v, vs))]


def _ancestors(parents, nodes):
    """[B,T,T]: whether node a is node i or an ancestor of it, by doubling."""
    B, T = parents.shape
    i = torch.arange(T, device=parents.device)
    p = torch.where((parents >= 0) & (parents < i) & (i < nodes[:, None]), parents.long(), torch.full_like(parents, T, dtype=torch.long))
    up = torch.zeros((B, T, T + 1), device=parents.device).scatter_(2, p[..., None], 1.0)[..., :T]
    up = up + torch.eye(T, device=parents.device)
    for _ in range(6):
        up = (up @ up).clamp(max=1.0)
    return up > 0


def _plain_attend(s, table):
    R, D, T = s["R"], s["D"], s["T"]
    q, ctx, nodes = s["q"], s["ctx"].long(), s["nodes"].long()
    B, _, Hq, _ = q.shape
    S = s["S"]
    at = torch.arange(S, device=q.device)
    there = at < (ctx + nodes)[:, None]                              # [B,S]
    blk = torch.where(there, table.gather(1, (at // R)[None].expand(B, S)).long(), torch.zeros((), dtype=torch.long, device=q.device))
    k, v, ks, vs = [t[0].unflatten(0, (B, S)) for t in _get(s["cache"], R, D, blk.flatten(), (at % R)[None].expand(B, S).flatten())]
    k, v = _decode(k, ks), _decode(v, vs)                            # [B,S,H,D]
    Hkv = k.shape[2]
    k = k.permute(0, 2, 3, 1).contiguous()
    v = torch.where(there[:, :, None, None], v, torch.zeros((), device=q.device)).permute(0, 2, 1, 3).contiguous()
    G = Hq // Hkv
    x = q.float().view(B, T, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * T, D).contiguous()
    scores = (x @ k) * (1.0 / math.sqrt(D))
    anc = _ancestors(s["parents"], s["nodes"])                       # [B,T,T]
    node = at[None] - ctx[:, None]                                   # [B,S]: the tree node of a row
    allow = (node < 0)[:, None] | (anc.gather(2, node.clamp(0, T - 1)[:, None].expand(B, T, S)) & (node >= 0)[:, None])
    allow = (allow & there[:, None])[:, None, None].expand(B, Hkv, G, T, S).reshape(B, Hkv, G * T, S)
    scores = torch.where(allow, scores, torch.full_like(scores, -math.inf))
    top = scores.amax(-1, keepdim=True)
    w = torch.exp(scores - top)
    total = w.sum(-1, keepdim=True)
    out = (w @ v) / total
    lse = (top + torch.log(total))[..., 0]
    out = out.view(B, Hkv, G, T, D).permute(0, 3, 1, 2, 4).reshape(B, T, Hq, D)
    lse = lse.view(B, Hkv, G, T).permute(0, 3, 1, 2).reshape(B, T, Hq)
    live = (torch.arange(T, device=q.device) < nodes[:, None])[:, :, None]
    zero = torch.zeros((), device=q.device)
    got = [torch.where(live[..., None], out, zero).to(torch.bfloat16)]
    return got + [torch.where(live, lse, zero)] if s["lse"] else got


def _plain_commit(s, table):
    R, D = s["R"], s["D"]
    ctx, n, path = s["ctx"].long(), s["length"].long(), s["path"].long()
    step = torch.arange(path.shape[1], device=ctx.device)[None].expand_as(path)
    b, t = torch.nonzero((step >= 1) & (step <= n[:, None]), as_tuple=True)
    src, dst = ctx[b] + path[b, t], ctx[b] + t
    _put(s["cache"], R, D, table[b, dst // R].long(), dst % R, _get(s["cache"], R, D, table[b, src // R].long(), src % R))
    return (ctx + n + 1).int()


# ------------------------------------------------------------------ inputs

def _i32(v):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(v, dtype=np.int32))).to("cuda")


def _fill(cache, R, D, gen, table, rows):
    """Rows of N(0,1) keys and values in layer 0 for every sequence's blocks."""
    H = cache.shape[2]
    for b, n in enumerate(rows):
        blk = torch.as_tensor(table[b, :-(-n // R)], device="cuda").long().repeat_interleave(R)
        row = torch.arange(R, device="cuda").repeat(len(blk) // R)
        k, ks = _encode(torch.randn((len(blk), H, D), generator=gen, device="cuda").bfloat16().float())
        v, vs = _encode(torch.randn((len(blk), H, D), generator=gen, device="cuda").bfloat16().float())
        _put(cache[:1], R, D, blk, row, [t[None] for t in (k, v, ks, vs)])


def _new_cache(layers, n_blocks, H, R, D):
    return torch.zeros((layers, n_blocks, H, R * (D + D // 16)), dtype=torch.uint8, device="cuda")


def _projected(s, gen, shape, Hq, Hkv, D):
    """Keys and values as a model has them: slices of one projection's output [..., (Hq + 2 Hkv) * D]."""
    x = torch.randn(tuple(shape) + (Hq + 2 * Hkv, D), generator=gen, device="cuda", dtype=torch.bfloat16)
    s["k"], s["v"] = x[..., Hq:Hq + Hkv, :], x[..., Hq + Hkv:, :]


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 29)
    kind, R = c["kind"], c["R"]
    s = dict(kind=kind, R=R, T=c.get("T"), D=c.get("D"), lse=c.get("lse", False), seed=int(seed))
    if kind == "append":
        N, H, D = c["N"], c["Hkv"], c["D"]
        n_blocks = -(-N // R) * 3 // 2 + 3
        r = random.Random(c["shape_seed"] * 8 + int(seed))
        ids = r.sample(range(n_blocks), -(-N // R))
        slots = np.array([ids[i // R] * R + i % R for i in range(N)], np.int32)
        slots[r.sample(range(N), c["unused"])] = -1
        s.update(slots=_i32(slots), cache=_new_cache(1, n_blocks, H, R, D))
        _projected(s, gen, (N,), c["Hq"], H, D)
        return _handles(c, s)
    ctx, nodes = _ctx(c), _nodes(c)
    s.update(S=c["ctx_hi"] + c["T"], ctx_list=ctx, nodes_list=nodes)
    par = _trees(c) if kind != "blocks" else None
    if kind in ("blocks", "step"):                                   # what the sequences held after the pass before
        r = random.Random(c["shape_seed"] * 8 + 5)
        held = [n + r.randint(0, R if kind == "step" else 2 * R) * (r.random() < 0.5) for n in ctx]
        table, owned, free, n_free, n_blocks = _tables(c, held, seed)
        for b in r.sample(range(c["B"]), c["ended"]):
            ctx[b] = -1
        s.update(owned=_i32(owned), free=_i32(free), n_free=_i32([n_free]), owned_out=_i32(owned), n_free_out=_i32([n_free]),
                 slots=_i32(np.zeros((c["B"], c["T"]))), granted=_i32(np.zeros(c["B"])))
    else:
        table, _, _, _, n_blocks = _tables(c, [a + n for a, n in zip(ctx, nodes)], seed)
    s.update(table=_i32(table), ctx=_i32(ctx), nodes=_i32(nodes))
    if kind == "blocks":
        return _handles(c, s)
    layers, H, D = c.get("layers", 1), c["Hkv"], c["D"]
    s["parents"] = _i32(par)
    s["cache"] = _new_cache(layers, n_blocks, H, R, D)
    if kind == "commit":                                             # any rows serve: codes at random, scales of values around one
        codes = R * D
        for one in s["cache"]:
            one.random_(0, 256, generator=gen)
            one[..., codes:] = torch.randint(122, 128, one[..., codes:].shape, generator=gen, device="cuda", dtype=torch.uint8)
    else:
        _fill(s["cache"], R, D, gen, table, [a + n for a, n in zip(ctx, nodes)] if kind == "attend" else ctx)
        s["q"] = torch.randn((c["B"], c["T"], c["Hq"], D), generator=gen, device="cuda", dtype=torch.bfloat16)
    if kind == "step":
        _projected(s, gen, (c["B"], c["T"]), c["Hq"], H, D)
    if kind in ("commit", "step"):
        length, path = _paths(c, par)
        s.update(length=_i32(length), path=_i32(path), new_ctx=_i32(ctx))
    if kind == "commit":                                             # slots of the rows that may be kept, root first, path by path
        D1 = path.shape[1]
        rows = np.asarray(ctx)[:, None] + np.arange(D1)[None]
        blk = np.take_along_axis(table, np.minimum(rows // R, table.shape[1] - 1), 1)
        s["kept"] = _i32(np.where(np.arange(D1)[None] <= length[:, None], blk * R + rows % R, -1))
    return _handles(c, s)


def _handles(c, s):
    """What a serving loop over fixed buffers keeps: its calls, marshalled once."""
    s["calls"] = None
    if own:
        s["calls"] = _calls(s)
    return s


def _calls(s):
    from paper_2512_14069_amd import binding as rb
    kind, calls = s["kind"], []
    tables = cache = None
    if kind in ("blocks", "step"):
        tables = rb.KvqTables(block_tables=s["table"], owned=s["owned"], free_blocks=s["free"], n_free=s["n_free"], block_rows=s["R"])
        calls.append(rb.radar_kvq_blocks(s["ctx"], tables, s["T"], n_new=s["nodes"], slots=s["slots"], granted=s["granted"],
                                         owned_out=s["owned_out"], n_free_out=s["n_free_out"], prepared=True))
    if kind != "blocks":
        cache = rb.KvqCache(data=s["cache"], block_rows=s["R"], D=s["D"])
    if kind in ("append", "step"):
        calls.append(rb.radar_kvq_append(cache, s["k"], s["v"], s["slots"], layer=0, prepared=True))
    if kind in ("attend", "step"):
        B, T, Hq, _ = s["q"].shape
        lse = torch.empty((B, T, Hq), dtype=torch.float32, device="cuda") if s["lse"] else None
        s["out"] = [torch.empty_like(s["q"])] + ([lse] if s["lse"] else [])
        calls.append(rb.radar_tree_attention_kvq(s["q"], cache, s["table"], s["ctx"], parents=s["parents"], n_nodes=s["nodes"], S_max=s["S"],
                                                 out=s["out"][0], lse_out=lse, prepared=True))
    if kind in ("commit", "step"):
        calls.append(rb.radar_kvq_commit(cache, s["table"], s["ctx"], s["length"], s["path"], new_ctx_lens=s["new_ctx"], prepared=True))
    if kind in ("append", "commit", "step"):
        read = rb.radar_kvq_read(cache, s["kept"] if kind == "commit" else s["slots"], prepared=True)
        s["rows"] = list(read.out)
        calls.append(read)
    return calls


# ------------------------------------------------------------------ one pass

def _own_run(s):
    calls = s["calls"] or _calls(s)
    for call in calls:
        call()
    kind, got = s["kind"], []
    if kind in ("blocks", "step"):
        got += [s["slots"], s["granted"], s["owned_out"], s["n_free_out"], s["table"], s["free"]]
    if kind in ("attend", "step"):
        got += s["out"]
    if kind in ("commit", "step"):
        got.append(s["new_ctx"])
    if kind in ("append", "commit", "step"):
        got += s["rows"]
    return got


def run(state):
    s = state
    if own:
        return _own_run(s)
    kind, got, slots = s["kind"], [], s.get("slots")
    if kind in ("blocks", "step"):
        got += _plain_blocks(s)
        slots = got[0]
    if kind in ("append", "step"):
        _plain_append(s, slots)
    if kind in ("attend", "step"):
        got += _plain_attend(s, s["table"])
    if kind in ("commit", "step"):
        got.append(_plain_commit(s, s["table"]))
    if kind in ("append", "commit", "step"):
        got += _plain_read(s, s["kept"] if kind == "commit" else slots)
    return got


# ------------------------------------------------------------------ from the definitions, in 64 bits

def _exact_blocks(table, owned, free, n_free, ctx, new, R, T):
    table, owned, free, n_free = table.copy(), [int(v) for v in owned], list(map(int, free)), int(n_free)
    B, M = table.shape
    want = [0 if l < 0 else -(-(l + n) // R) for l, n in zip(ctx, new)]
    for b in range(B):
        if want[b] <= M:
            for i in range(want[b], owned[b]):
                if n_free < len(free):
                    free[n_free] = int(table[b, i])
                    n_free += 1
    granted, short, at = [], False, n_free
    for b in range(B):
        need = max(0, want[b] - owned[b]) if want[b] <= M else 0
        short = short or (need > 0 and need > at)
        granted.append(int(want[b] <= M and (need == 0 or not short)))
        if granted[b]:
            for i in range(owned[b], want[b]):
                at -= 1
                table[b, i] = free[at]
            owned[b] = want[b]
    slots = np.full((B, T), -1, np.int32)
    for b in range(B):
        for i in range(new[b] if granted[b] and ctx[b] >= 0 else 0):
            slots[b, i] = table[b, (ctx[b] + i) // R] * R + (ctx[b] + i) % R
    return [slots, np.array(granted, np.int32), np.array(owned, np.int32), np.array([at], np.int32), table.astype(np.int32), np.array(free, np.int32)]


def _exact_values(x):
    """What rows x [..., D] become: float64, by distance to every code."""
    blk = x.double().reshape(x.shape[:-1] + (-1, 32))
    amax = blk.abs().max(-1).values
    e = torch.ceil(torch.log2(amax / 7.0).clamp(-200, 200))
    e = torch.where(amax >= 7.0 * torch.exp2(e), e + 1, e)
    e = torch.where(amax < 7.0 * torch.exp2(e - 1), e - 1, e).clamp(-126, 125)
    step = torch.exp2(e)[..., None]
    y = (blk / step).abs()
    lut = torch.tensor(LUT, dtype=torch.float64, device=x.device)
    best, code = torch.full_like(y, math.inf), torch.zeros_like(y)
    for i in [0, 2, 4, 6, 1, 3, 5, 7]:                               # an even code first: it keeps a tie
        d = (y - lut[i]).abs()
        code = torch.where(d < best, lut[i], code)
        best = torch.minimum(d, best)
    return (code * step * torch.sign(blk)).reshape(x.shape)


def _exact_rows(cache, R, D, table, n):
    """Rows 0 ... n-1 of one sequence as float64 [n, H, D], K and V, straight from the bytes of layer 0."""
    half, got = R * D // 2, []
    lut = torch.tensor(LUT + [-v for v in LUT], dtype=torch.float64, device=cache.device)
    blocks = cache[0][torch.as_tensor(table[:-(-n // R)], device=cache.device).long()]       # [m, H, bytes]
    m, H, _ = blocks.shape
    for kv in (0, 1):
        raw = blocks[..., kv * half:(kv + 1) * half]
        raw = raw.reshape(m, H, R, D // 2) if kv == 0 else raw.reshape(m, H, R // 8, D // 8, 8, 4).permute(0, 1, 2, 4, 3, 5).reshape(m, H, R, D // 2)
        sc = blocks[..., 2 * half + kv * (R * D // 32):][..., :R * D // 32].reshape(m, H, R // 8, D // 32, 8).permute(0, 1, 2, 4, 3)
        sc = torch.exp2(sc.reshape(m, H, R, D // 32).double() - 127.0).repeat_interleave(32, -1)
        x = torch.empty((m, H, R, D), dtype=torch.float64, device=cache.device)
        x[..., 0::2], x[..., 1::2] = lut[(raw % 16).int()], lut[(raw // 16).int()]
        got.append((x * sc).transpose(1, 2).reshape(m * R, H, D)[:n])
    return got


def _exact_attend(c, s, par, table):
    D, T, Hq, Hkv = c["D"], c["T"], c["Hq"], c["Hkv"]
    G = Hq // Hkv
    out = torch.zeros((c["B"], T, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((c["B"], T, Hq), dtype=torch.float64, device="cuda")
    for b, (l, n) in enumerate(zip(s["ctx_list"], s["nodes_list"])):
        k, v = _exact_rows(s["cache"], c["R"], D, table[b], l + n)
        allow = np.zeros((n, l + n), bool)
        allow[:, :l] = True
        for i in range(n):
            a = i
            while a >= 0:
                allow[i, l + a] = True
                a = int(par[b, a])
        bar = torch.from_numpy(np.where(allow, 0.0, -np.inf)).to("cuda")
        for h in range(Hq):
            x = s["q"][b, :n, h].double() @ k[:, h // G].t().contiguous() / math.sqrt(D) + bar
            lse[b, :n, h] = torch.logsumexp(x, -1)
            out[b, :n, h] = torch.exp(x - lse[b, :n, h, None]) @ v[:, h // G].contiguous()
    return [out, lse] if c.get("lse") else [out]


def exact(case, seed):
    global own
    c, was = dict(case), own
    own = False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    kind, R, got = c["kind"], c["R"], []
    table = s["table"].cpu().numpy() if "table" in s else None
    par = s["parents"].cpu().numpy() if "parents" in s else None
    if kind in ("blocks", "step"):
        got += _exact_blocks(table, s["owned"].cpu().numpy(), s["free"].cpu().numpy(), int(s["n_free"][0]), s["ctx_list"], s["nodes_list"], R, c["T"])
        table = got[4]
    if kind == "blocks":
        return got
    if kind == "attend":
        return _exact_attend(c, s, par, table)
    if kind == "append":
        keep = (s["slots"] >= 0)[:, None, None]
        return [torch.where(keep, _exact_values(s[x]), torch.zeros((), dtype=torch.float64, device="cuda"))[None] for x in ("k", "v")]
    if kind == "step":                                               # the new rows' values depend on nothing but themselves
        k, v = (_exact_values(s[x]) for x in ("k", "v"))
        slots = torch.from_numpy(got[0]).to("cuda").long().flatten()
        keep = slots >= 0
        _put(s["cache"], R, c["D"], slots[keep] // R, slots[keep] % R, _again(k, v, keep))
        got += _exact_attend(c, s, par, table)
    length, path = s["length"].cpu().numpy(), s["path"].cpu().numpy()
    got.append(np.asarray(s["ctx_list"], np.int32) + length + 1)
    if kind == "step":
        rows = [x.clone() for x in (k, v)]
        for b in range(c["B"]):
            for t in range(1, int(length[b]) + 1):
                for new, old in zip(rows, (k, v)):
                    new[b, t] = old[b, int(path[b, t])]
        return got + [torch.where(keep[:, None, None], x.flatten(0, 1), torch.zeros((), dtype=torch.float64, device="cuda"))[None] for x in rows]
    kept = s["kept"].cpu().numpy()
    L, H, D, D1 = c["layers"], c["Hkv"], c["D"], path.shape[1]
    rows = [torch.zeros((L, c["B"], D1, H, D), dtype=torch.float64, device="cuda") for _ in range(2)]
    for b, l in enumerate(s["ctx_list"]):
        n = l + int(path[b].max()) + 1
        for layer in range(L):
            kv = _exact_rows(s["cache"][layer:layer + 1], R, D, table[b], n)
            pick = torch.as_tensor(l + path[b, :int(length[b]) + 1], device="cuda").long()
            for x, r in zip(kv, rows):
                r[layer, b, :len(pick)] = x[pick]
    assert (kept >= 0).sum() == (length + 1).sum()
    return got + [r.flatten(1, 2) for r in rows]


def _again(k, v, keep):
    """Codes and scales that stand for the values k and v [B,T,H,D] exactly (a value of the format encodes to itself)."""
    a, b = (_encode(x.flatten(0, 1)[keep].float()) for x in (k, v))
    return [t[None] for t in (a[0], b[0], a[1], b[1])]


# ------------------------------------------------------------------ what a pass cannot do without

def _row(c):
    return c["Hkv"] * (c["D"] + c["D"] // 16)                        # bytes of a row of the cache, K and V


def _work(c, kind):
    if kind == "append":
        return (c["N"] - c["unused"]) * c["Hkv"] * c["D"] * 4 + c["N"] * 4 + (c["N"] - c["unused"]) * _row(c), 0.0
    nodes = _nodes(c)
    if kind == "blocks":
        moved = sum(-(-n // c["R"]) for n in nodes)
        return 4 * (c["B"] * (c["T"] + 5) + 2 * moved), 0.0
    if kind == "attend":
        rows = [a + n for a, n in zip(_ctx(c), nodes)]
        byt = sum(rows) * _row(c) + (sum(nodes) + c["B"] * c["T"]) * c["Hq"] * c["D"] * 2
        return byt, 4.0 * sum(r * n for r, n in zip(rows, nodes)) * c["Hq"] * c["D"]
    length, path = _paths(c, _trees(c))
    moved = int(sum((path[b, t] != t) for b in range(c["B"]) for t in range(1, int(length[b]) + 1)))
    return moved * c["layers"] * _row(c) * 2 + path.size * 4, 0.0


def _read_work(c, kind):
    if kind == "append":
        kept, all_ = c["N"] - c["unused"], c["N"]
    elif kind == "commit":
        length, path = _paths(c, _trees(c))
        kept, all_ = int(length.sum()) + c["B"], path.size
    else:
        kept, all_ = sum(_nodes(c)), c["B"] * c["T"]
    return c.get("layers", 1) * (kept * _row(c) + all_ * c["Hkv"] * c["D"] * 4)


def work(case):
    c = dict(case)
    kind = c["kind"]
    if kind != "step":
        byt, flops = _work(c, kind)
        return {"bytes": byt + (_read_work(c, kind) if kind in ("append", "commit") else 0), "flops": flops}
    rows = dict(c, N=sum(_nodes(c)), unused=0)
    parts = [_work(c, "blocks"), _work(rows, "append"), _work(c, "attend"), _work(c, "commit")]
    return {"bytes": sum(p[0] for p in parts) + _read_work(c, kind), "flops": sum(p[1] for p in parts)}
