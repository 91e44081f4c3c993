"""Rotary positions, rotated rows into the paged 4-bit cache, and chunks of new tokens over it, as measurable cases: plain form and the library's calls.

Four kinds of pass:

  rope     rows of q and k turned by their positions, for caches of any kind
  append   rows of a batch's new tokens: q turned, k turned and k and v into the paged 4-bit cache, and back out of it as the values they stand for
  chunk    one layer's attention of a batch's new tokens (prompts, pieces of prompts, single tokens) over the paged 4-bit cache
  step     one layer's part in a serving step: blocks and slots, rows in, attention, rows out

Rows are [B, T] with a count for each sequence ("padded"), or one sequence's behind the other's ("packed": sequence b has rows starts[b] ... starts[b+1] - 1).
Row i of sequence b is at cache row ctx[b] + i, and sees the cache rows up to itself.

Rotation.  Pair j of a row (values j and j + P of the first 2 P, or 2 j and 2 j + 1) is turned by t = (positions[axis of j] + ctx) * inv_freq[j], worked out in
64 bits, since a position of a million radians leaves 32 none for the fraction.  The turned values are rounded to 32 bits and then to bf16; so is k before it is encoded.

Format.  32 consecutive values of a row share a power of two 2^e and are e2m1 codes (0 .5 1 1.5 2 3 4 6 and a sign); e is the smallest
whole number with amax < 7 * 2^e, within [-126, 125]; codes round to nearest, ties to the even code; byte e + 127 is kept, or 255 for a block
with an infinity or NaN, which stands for 32 NaNs.  A block of R rows of one KV head is R * (D + D / 16) bytes:
K codes [R][D/2], V codes [R/8][D/8][8][4], K scales [R/8][D/32][8], V scales [R/8][D/32][8]; an even element is a byte's low half.

Lengths of a case come from its `shape_seed`, values from prepare()'s seed.
"""
import math
import random

import numpy as np
import torch

own = False

LUT = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
CAP = 4.0 * 64 * 128 * (16384 * 16384 / 2)                           # operations of the largest listed case, beyond which none is drawn


def listed():
    return [
        # the rows of one 60-node tree on an 8B-class target with a dense cache: positions are the nodes' depths behind the prefix; bound by the call
        dict(name="rope_tree", kind="rope", B=1, T=60, packed=False, n_lo=60, singles=0, ended=0, Hq=32, Hkv=8, D=128, pairs=64, axes=1, dealt=False, adjacent=False,
             ctx_lo=2048, ctx_hi=2048, shape_seed=1),
        # a video's patches with time, height and width, an odd number of them, out of a projection's fused output: bound by bytes
        dict(name="rope_video", kind="rope", B=3, T=3000, packed=True, n_lo=2000, singles=0, ended=0, Hq=32, Hkv=8, D=128, pairs=64, axes=3, dealt=False, adjacent=False,
             ctx_lo=0, ctx_hi=0, shape_seed=2),
        # plain decoding of a served batch of 64 conversations, a token each
        dict(name="append_tokens64", kind="append", B=64, T=1, packed=True, n_lo=1, singles=0, ended=0, Hq=32, Hkv=8, D=128, R=16, pairs=64, axes=1, dealt=False,
             adjacent=False, ctx_lo=512, ctx_hi=8192, shape_seed=3),
        # the trees of a served batch of 16, of different sizes
        dict(name="append_trees16", kind="append", B=16, T=60, packed=False, n_lo=2, singles=0, ended=0, Hq=32, Hkv=8, D=128, R=16, pairs=64, axes=1, dealt=False,
             adjacent=False, ctx_lo=512, ctx_hi=8192, shape_seed=4),
        # prompts with images in them, of odd lengths, one behind the other
        dict(name="append_prompts", kind="append", B=5, T=2047, packed=True, n_lo=1200, singles=0, ended=0, Hq=32, Hkv=8, D=128, R=32, pairs=64, axes=3, dealt=True,
             adjacent=False, ctx_lo=0, ctx_hi=0, shape_seed=5),
        # one new token of a single short conversation on the smallest layer that the repository configures: bound by the call itself
        dict(name="chunk_token_small", kind="chunk", B=1, T=1, packed=True, n_lo=1, singles=0, ended=0, Hq=4, Hkv=1, D=64, R=16, ctx_lo=256, ctx_hi=256, lse=True,
             shape_seed=6),
        # a first prompt of an 8B-class target
        dict(name="chunk_prompt", kind="chunk", B=1, T=2048, packed=False, n_lo=2048, singles=0, ended=0, Hq=32, Hkv=8, D=128, R=16, ctx_lo=0, ctx_hi=0, lse=False,
             shape_seed=7),
        # a piece of a long prompt behind what is cached of it
        dict(name="chunk_piece", kind="chunk", B=1, T=512, packed=True, n_lo=512, singles=0, ended=0, Hq=32, Hkv=8, D=128, R=64, ctx_lo=16384, ctx_hi=16384, lse=False,
             shape_seed=8),
        # a serving step of 48 conversations: a token of each but two, of which a prompt's piece
        dict(name="chunk_mixed48", kind="chunk", B=48, T=512, packed=True, n_lo=300, singles=46, ended=1, Hq=32, Hkv=8, D=128, R=16, ctx_lo=512, ctx_hi=8192, lse=False,
             shape_seed=9),
        # prompts of 16 conversations of odd lengths, some of them behind shared or earlier rows
        dict(name="chunk_ragged16", kind="chunk", B=16, T=2001, packed=True, n_lo=90, singles=0, ended=0, Hq=32, Hkv=8, D=128, R=16, ctx_lo=0, ctx_hi=1500, lse=True,
             shape_seed=10),
        # a long prompt on a 70B-class target, the largest layer configured: bound by the matrix products
        dict(name="chunk_prompt_70b", kind="chunk", B=1, T=16384, packed=True, n_lo=16384, singles=0, ended=0, Hq=64, Hkv=8, D=128, R=64, ctx_lo=0, ctx_hi=0, lse=False,
             shape_seed=11),
        # all of it in a row, as one layer of a serving step makes the calls: tokens of 14 conversations and pieces of two prompts
        dict(name="step_mixed16", kind="step", B=16, T=400, packed=True, n_lo=200, singles=14, ended=0, Hq=32, Hkv=8, D=128, R=16, pairs=64, axes=1, dealt=False,
             adjacent=False, ctx_lo=256, ctx_hi=4096, lse=False, shape_seed=12),
    ]


# ------------------------------------------------------------------ drawn cases

def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _heads(rng):
    Hkv = rng.choice([1, 2, 4, 5, 8])
    return Hkv * rng.choice([1, 2, 4, 5, 8]), Hkv, rng.choice([64, 128, 128])


def _turns(rng, D):
    axes = rng.choice([1, 1, 2, 3, 4])
    return dict(pairs=rng.choice([D // 2, D // 2, D // 4, 8, 24]), axes=axes, dealt=rng.random() < 0.5, adjacent=rng.random() < 0.4)


def _batch(rng, top):
    """Sequences and rows of them, at most `top` in all."""
    while True:
        B, T = _log(rng, 1, 64), _log(rng, 1, top)
        singles = rng.choice([0, 0, rng.randint(0, B - 1)])
        if (B - singles) * T + singles <= top:
            return dict(B=B, T=T, packed=rng.random() < 0.6 and singles >= 0 or singles > 0, n_lo=rng.choice([T, max(1, T // 4), 1]), singles=singles,
                        ended=rng.choice([0, 0, 1]) if B > 2 else 0, shape_seed=rng.randrange(1 << 20))


def _draw_rope(rng):
    Hq, Hkv, D = _heads(rng)
    hi = rng.choice([0, _log(rng, 1, 1 << 20)])
    return dict(_batch(rng, 8192), kind="rope", Hq=Hq, Hkv=Hkv, D=D, ctx_lo=hi // 2, ctx_hi=hi, **_turns(rng, D))


def _draw_append(rng):
    Hq, Hkv, D = _heads(rng)
    hi = rng.choice([0, _log(rng, 1, 8192)])
    return dict(_batch(rng, 8192), kind="append", Hq=Hq, Hkv=Hkv, D=D, R=rng.choice([16, 32, 64, 128]), ctx_lo=hi // 4, ctx_hi=hi, **_turns(rng, D))


def _draw_chunk(rng):
    while True:
        Hq, Hkv, D = _heads(rng)
        c = _batch(rng, 16384)
        hi = rng.choice([0, _log(rng, 1, 16384)])
        long = c["B"] - c["singles"]
        if c["B"] * (hi + c["T"]) * Hkv * D <= 64 * 8192 * 1024 and 4.0 * Hq * D * (long * c["T"] * (hi + c["T"] / 2) + c["singles"] * hi) <= CAP / 4:
            return dict(c, kind="chunk", Hq=Hq, Hkv=Hkv, D=D, R=rng.choice([16, 32, 64, 128]), ctx_lo=hi // rng.choice([1, 2, 16]), ctx_hi=hi,
                        lse=rng.random() < 0.5)


def _draw_step(rng):
    while True:
        Hq, Hkv, D = _heads(rng)
        c = _batch(rng, 2048)
        hi = _log(rng, 1, 4096)
        if c["B"] <= 32:
            return dict(c, kind="step", Hq=Hq, Hkv=Hkv, D=D, R=rng.choice([16, 32, 64, 128]), ctx_lo=hi // 4, ctx_hi=hi, lse=False, **_turns(rng, D))


def draw(rng):
    return rng.choice([_draw_chunk] * 4 + [_draw_rope, _draw_append, _draw_append, _draw_step])(rng)


# ------------------------------------------------------------------ shapes of a case

def _lens(c, lo, hi, what):
    """One whole number per sequence, spread over [lo, hi]; the largest is hi."""
    r = random.Random(c["shape_seed"] * 8 + what)
    v = [r.randint(lo, hi) for _ in range(c["B"])]
    v[r.randrange(c["B"])] = hi
    return v


def _ctx(c):
    v = _lens(c, c["ctx_lo"], c["ctx_hi"], 0)
    for b in random.Random(c["shape_seed"] * 8 + 2).sample(range(c["B"]), c["ended"]):
        v[b] = -1                                                    # a sequence that has ended
    return v


def _news(c):
    v = _lens(c, min(c["n_lo"], c["T"]), c["T"], 1)
    r = random.Random(c["shape_seed"] * 8 + 3)
    for b in r.sample([b for b in range(c["B"])], c["singles"]):
        v[b] = 1
    if c["kind"] != "chunk" or c["packed"]:
        return [0 if n < 0 else m for n, m in zip(_ctx(c), v)]
    return v


def _tables(c, rows, seed):
    """Block tables [B,M] of sequences that hold `rows` rows each, from a pool with a few more blocks in the order that the seed gives;
    free stack and its height."""
    R = c["R"]
    need = [-(-max(n, 0) // R) for n in rows]
    M = max(max(need), -(-(c["ctx_hi"] + c["T"]) // R)) + 1
    n_blocks = sum(need) + max(4, sum(need) // 8) + sum(-(-n // R) + 1 for n in _news(c))
    ids = list(range(n_blocks))
    random.Random(c["shape_seed"] * 65537 + int(seed)).shuffle(ids)
    table, at = np.full((c["B"], M), -1, np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    free = np.full(n_blocks, -1, np.int32)
    free[:n_blocks - at] = ids[at:]
    return table, np.array(need, np.int32), free, n_blocks - at, n_blocks


def _rows_of(c, news):
    """(sequence, row of it) of every row that there is, and where it is among the tensors' rows."""
    b = np.repeat(np.arange(c["B"]), news)
    i = np.concatenate([np.arange(n) for n in news]).astype(np.int64) if sum(news) else np.zeros(0, np.int64)
    return b, i, (np.arange(len(b)) if c["packed"] else b * c["T"] + i)


# ------------------------------------------------------------------ the cache's format in plain torch

def _sections(cache, R, D):
    """Views of cache [..., n_blocks, H, bytes]: K codes [..., H, R, D/2], V codes [..., H, R/8, D/8, 8, 4], scales [..., H, R/8, D/32, 8]."""
    half, sc = R * D // 2, R * D // 32
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
    """K and V codes and scales of rows (blk, row), both [n], of one layer's cache: each [n, H, ...]."""
    kc, vc, ks, vs = _sections(cache, R, D)
    r8, r1 = row // 8, row % 8
    return kc[blk, :, row], vc[blk, :, r8, :, r1].flatten(-2), ks[blk, :, r8, :, r1], vs[blk, :, r8, :, r1]


def _put(cache, R, D, blk, row, parts):
    kc, vc, ks, vs = _sections(cache, R, D)
    r8, r1 = row // 8, row % 8
    k, v, a, b = parts
    kc[blk, :, row] = k
    vc[blk, :, r8, :, r1] = v.unflatten(-1, (-1, 4))
    ks[blk, :, r8, :, r1] = a
    vs[blk, :, r8, :, r1] = b


# ------------------------------------------------------------------ the operators in plain torch

def _plain_rows(s):
    """Of every row of q: its sequence, its number in it, and whether it is there."""
    n = torch.arange(s["N"], device="cuda")
    if s["starts"] is None:
        b, i = n // s["T"], n % s["T"]
        there = i < s["news"].long()[b]
    else:
        b = torch.searchsorted(s["starts"][1:].contiguous(), n.int(), right=True).clamp(max=s["B"] - 1)
        i = n - s["starts"].long()[b]
        there = (n < s["starts"][-1]) & (i < s["T"])
    return b, i, there & (s["ctx"][b] >= 0)


def _plain_turn(s, x, cos, sin):
    """x [N,H,D] turned, rounded to 32 bits and to bf16."""
    P = s["pairs"]
    d = x.double()
    if s["adjacent"]:
        a, b = d[..., 0:2 * P:2], d[..., 1:2 * P:2]
        t = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = d[..., :P], d[..., P:2 * P]
        t = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return torch.cat((t.float().to(torch.bfloat16), x[..., 2 * P:]), -1)


def _plain_angles(s, b, i):
    pos = s["positions"].long() if s["positions"] is not None else i[None].expand(s["axes"], -1)
    pos = pos + s["ctx"].long()[b].clamp(min=0)
    t = pos[s["axis_of"]].t().double() * s["inv_freq"].double()      # [N,P]
    return torch.cos(t)[:, None], torch.sin(t)[:, None]


def _plain_rope(s, out, x, cos, sin, there):
    out.copy_(torch.where(there[:, None, None], _plain_turn(s, x, cos, sin), out))
    return out


def _plain_slots(s, slots, b, i, there):
    at = slots[b, i.clamp(max=s["T"] - 1)].long()
    return torch.where(there, at, torch.full_like(at, -1))


def _plain_append(s, slots):
    R, D = s["R"], s["D"]
    b, i, there = _plain_rows(s)
    cos, sin = _plain_angles(s, b, i)
    got = _plain_rope(s, s["q_out"], s["q"].flatten(0, -3), cos, sin, there)
    at = _plain_slots(s, slots, b, i, there)
    keep = at >= 0
    at = at[keep]
    k, ks = _encode(_plain_turn(s, s["k"].flatten(0, -3), cos, sin)[keep].float())
    v, vs = _encode(s["v"].flatten(0, -3)[keep].float())
    _put(s["cache"], R, D, at // R, at % R, (k, v, ks, vs))
    return got


def _plain_read(s, slots):
    at = slots.flatten().long()
    k, v, ks, vs = _get(s["cache"], s["R"], s["D"], at.clamp(min=0) // s["R"], at.clamp(min=0) % s["R"])
    keep = (at >= 0)[:, None, None]
    return [torch.where(keep, _decode(c, f), torch.zeros((), device=c.device)).to(torch.bfloat16)[None] for c, f in ((k, ks), (v, vs))]


def _plain_chunk(s, q, table):
    """q [N,Hq,D] -> out [N,Hq,D], log-sum-exps [N,Hq]; a sequence and 1024 rows of a KV head's queries at a time."""
    R, D, T, Hkv = s["R"], s["D"], s["T"], s["Hkv"]
    G, scale = s["Hq"] // Hkv, 1.0 / math.sqrt(s["D"])
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(q.shape[:2], dtype=torch.float32, device="cuda")
    first = 0
    for b, (l, n) in enumerate(zip(s["ctx_list"], s["news_list"])):
        row0 = first if s["starts"] is not None else b * T
        first += n
        if l < 0 or n == 0:
            continue
        at = torch.arange(l + n, device="cuda")
        k, v, ks, vs = _get(s["cache"], R, D, table[b, at // R].long(), at % R)
        k, v = _decode(k, ks).permute(1, 2, 0).contiguous(), _decode(v, vs).transpose(0, 1).contiguous()       # [H,D,S], [H,S,D]
        for i0 in range(0, n, 1024):
            m = min(1024, n - i0)
            rows, S = slice(row0 + i0, row0 + i0 + m), l + i0 + m
            x = q[rows].float().view(m, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, m * G, D).contiguous()
            bar = (torch.arange(S, device="cuda")[None] > l + i0 + torch.arange(m, device="cuda")[:, None]).repeat_interleave(G, 0)
            for h in range(Hkv):
                x_h = (x[h] @ k[h, :, :S]) * scale
                x_h.masked_fill_(bar, -math.inf)
                top = x_h.amax(-1, keepdim=True)
                w = torch.exp(x_h - top)
                total = w.sum(-1, keepdim=True)
                out[rows, h * G:(h + 1) * G] = ((w @ v[h, :S]) / total).to(torch.bfloat16).view(m, G, D)
                lse[rows, h * G:(h + 1) * G] = (top + torch.log(total)).view(m, G)
    return [out, lse] if s["lse"] else [out]


def _plain_blocks(s):
    R, M, n_blocks, T = s["R"], s["table"].shape[1], s["free"].numel(), s["T"]
    ctx, new, owned, n_free = s["ctx"].long(), s["news"].long(), s["owned"].long(), s["n_free"].long()
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


# ------------------------------------------------------------------ inputs

def _i32(v):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(v, dtype=np.int32))).to("cuda")


def _fill(cache, R, D, gen, table, rows):
    """Rows of N(0,1) keys and values for every sequence's blocks."""
    H = cache.shape[1]
    for b, n in enumerate(rows):
        blk = torch.as_tensor(table[b, :-(-n // R)] if n > 0 else [], device="cuda").long().repeat_interleave(R)
        row = torch.arange(R, device="cuda").repeat(len(blk) // R)
        if len(blk) == 0:
            continue
        k, ks = _encode(torch.randn((len(blk), H, D), generator=gen, device="cuda").bfloat16().float())
        v, vs = _encode(torch.randn((len(blk), H, D), generator=gen, device="cuda").bfloat16().float())
        _put(cache, R, D, blk, row, (k, v, ks, vs))


def _positions(c, news, seed):
    """[axes, rows]: of text the rows' numbers, or the depths of a tree's nodes; of images and video time, height and width, each image's behind what came before."""
    r = random.Random(c["shape_seed"] * 8 + int(seed) * 64 + 4)
    N = sum(news) if c["packed"] else c["B"] * c["T"]
    pos = np.zeros((c["axes"], max(N, 1)), np.int32)
    at = 0
    for b, n in enumerate(news):
        row0, wide = (at if c["packed"] else b * c["T"]), r.randint(3, 40)
        i = np.arange(n)
        if c["axes"] == 1:
            pos[0, row0:row0 + n] = np.minimum(i, [r.randint(0, 8) for _ in i]) if not c["packed"] and c["T"] <= 64 else i
        else:
            for a, v in enumerate([i // (wide * wide), i // wide % wide, i % wide, i][-c["axes"] if c["axes"] == 2 else 0:][:c["axes"]]):
                pos[a, row0:row0 + n] = v
        at += n
    return pos[:, :N]


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 31)
    kind, B, T, Hq, Hkv, D = (c[n] for n in ("kind", "B", "T", "Hq", "Hkv", "D"))
    ctx, news = _ctx(c), _news(c)
    N = sum(news) if c["packed"] else B * T
    s = dict(kind=kind, B=B, T=T, N=N, Hq=Hq, Hkv=Hkv, D=D, R=c.get("R"), lse=c.get("lse", False), ctx_list=ctx, news_list=news, ctx=_i32(ctx), news=_i32(news),
             starts=_i32(np.concatenate(([0], np.cumsum(news)))) if c["packed"] else None, S=c["ctx_hi"] + T, packed=c["packed"])
    lead = (N,) if c["packed"] else (B, T)
    fused = torch.randn(lead + (Hq + 2 * Hkv, D), generator=gen, device="cuda", dtype=torch.bfloat16)          # a projection's output
    s["q"], s["k"], s["v"] = fused[..., :Hq, :], fused[..., Hq:Hq + Hkv, :], fused[..., Hq + Hkv:, :]
    if kind != "chunk":
        P, axes = c["pairs"], c["axes"]
        axis_of = [j % axes if c["dealt"] else j * axes // P for j in range(P)]
        s.update(pairs=P, axes=axes, adjacent=c["adjacent"], axis_of=axis_of, positions=_i32(_positions(c, news, seed)),
                 inv_freq=(10000.0 ** (-torch.arange(P, dtype=torch.float64) / P)).float().to("cuda"))
        s["q_out"] = torch.zeros((N, Hq, D), dtype=torch.bfloat16, device="cuda")
    if kind == "rope":
        s["k_out"] = torch.zeros((N, Hkv, D), dtype=torch.bfloat16, device="cuda")
        return _handles(s)
    if kind == "step":                                               # what the sequences held after the step before
        r = random.Random(c["shape_seed"] * 8 + 5)
        held = [max(n, 0) + r.randint(0, c["R"]) * (r.random() < 0.5) for n in ctx]
    else:
        held = [l + n if l >= 0 else 0 for l, n in zip(ctx, news)]
    table, owned, free, n_free, n_blocks = _tables(c, held, seed)
    s["table"] = _i32(table)
    s["cache"] = torch.zeros((n_blocks, Hkv, c["R"] * (D + D // 16)), dtype=torch.uint8, device="cuda")
    if kind == "append":
        slots = np.full((B, T), -1, np.int32)
        for b, (l, n) in enumerate(zip(ctx, news)):
            j = l + np.arange(n)
            slots[b, :n] = table[b, j // c["R"]] * c["R"] + j % c["R"]
        s["slots"] = _i32(slots)
    else:
        _fill(s["cache"], c["R"], D, gen, table, held if kind == "chunk" else ctx)
    if kind == "step":
        s.update(owned=_i32(owned), free=_i32(free), n_free=_i32([n_free]), owned_out=_i32(owned), n_free_out=_i32([n_free]),
                 slots=_i32(np.zeros((B, T))), granted=_i32(np.zeros(B)))
    return _handles(s)


def _handles(s):
    """What a serving loop over fixed buffers keeps: its calls, marshalled once."""
    s["calls"] = None
    if own:
        s["calls"] = _calls(s)
    return s


def _calls(s):
    from paper_2512_14069_amd import binding as rb
    kind, calls, cache, q = s["kind"], [], None, s["q"]
    rows = dict(ctx_lens=s["ctx"], row_starts=s["starts"], n_new=None if s["packed"] else s["news"])
    if kind != "chunk":
        rope = rb.Rope(s["inv_freq"], axes=s["axes"], pair_axis=s["axis_of"], interleaved=s["adjacent"])
        q_out = s["q_out"].view(q.shape)
    if kind == "rope":
        return [rb.radar_rope(q, s["k"], rope, positions=s["positions"], T_max=s["T"], q_out=q_out, k_out=s["k_out"].view(s["k"].shape), prepared=True, **rows)]
    cache = rb.KvqCache(data=s["cache"][None], block_rows=s["R"], D=s["D"])
    if kind == "step":
        tables = rb.KvqTables(block_tables=s["table"], owned=s["owned"], free_blocks=s["free"], n_free=s["n_free"], block_rows=s["R"])
        calls.append(rb.radar_kvq_blocks(s["ctx"], tables, s["T"], n_new=s["news"], slots=s["slots"], granted=s["granted"], owned_out=s["owned_out"],
                                         n_free_out=s["n_free_out"], prepared=True))
    if kind != "chunk":
        calls.append(rb.radar_kvq_append_rope(cache, q, s["k"], s["v"], s["slots"], rope, positions=s["positions"], q_out=q_out, prepared=True, **rows))
        q = q_out
    if kind != "append":
        lse = torch.empty(q.shape[:-1], dtype=torch.float32, device="cuda") if s["lse"] else None
        out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
        calls.append(rb.radar_chunk_attention_kvq(q, cache, s["table"], T_max=s["T"], S_max=s["S"], out=out, lse_out=lse, prepared=True, **rows))
        s["out"] = [t.flatten(0, -3 if t is out else -2) for t in ([out, lse] if s["lse"] else [out])]
    if kind != "chunk":
        calls.append(rb.radar_kvq_read(cache, s["slots"], prepared=True))
        s["rows"] = list(calls[-1].out)
    return calls


# ------------------------------------------------------------------ one pass

def run(state):
    s, kind, got = state, state["kind"], []
    if own:
        for call in s["calls"] or _calls(s):
            call()
        if kind == "rope":
            return [s["q_out"], s["k_out"]]
        if kind == "step":
            got += [s["slots"], s["granted"], s["owned_out"], s["n_free_out"], s["table"], s["free"]]
        if kind != "chunk":
            got.append(s["q_out"])
        return got + (s["out"] if kind != "append" else []) + (s["rows"] if kind != "chunk" else [])
    slots, q = s.get("slots"), s["q"].flatten(0, -3)
    if kind == "rope":
        b, i, there = _plain_rows(s)
        cos, sin = _plain_angles(s, b, i)
        return [_plain_rope(s, s["q_out"], q, cos, sin, there), _plain_rope(s, s["k_out"], s["k"].flatten(0, -3), cos, sin, there)]
    if kind == "step":
        got += _plain_blocks(s)
        slots = got[0]
    if kind != "chunk":
        q = _plain_append(s, slots)
        got.append(q)
    if kind != "append":
        got += _plain_chunk(s, q, s["table"])
    if kind != "chunk":
        got += _plain_read(s, slots)
    return got


# ------------------------------------------------------------------ from the definitions, in 64 bits

def _exact_turn(c, s, x, rows):
    """x [N,H,D] -> float64, rows [(sequence, row of it)] of N that are there turned by complex numbers, the others zero."""
    b, i, at = rows
    P = c["pairs"]
    at = torch.as_tensor(at, device="cuda")
    ctx = torch.as_tensor([max(l, 0) for l in s["ctx_list"]], device="cuda", dtype=torch.float64)[torch.as_tensor(b, device="cuda")]
    pos = s["positions"].double()[:, at] + ctx
    freq = s["inv_freq"].double()
    out = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    y = x[at].double()
    for j in range(P):
        t = pos[s["axis_of"][j]] * freq[j]
        one, two = (2 * j, 2 * j + 1) if c["adjacent"] else (j, j + P)
        z = torch.complex(y[..., one], y[..., two]) * torch.polar(torch.ones_like(t), t)[:, None]
        y[..., one], y[..., two] = z.real, z.imag
    out[at] = y
    return out


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
    """Rows 0 ... n-1 of one sequence as float64 [n, H, D], K and V, straight from the bytes."""
    half, got = R * D // 2, []
    lut = torch.tensor(LUT + [-v for v in LUT], dtype=torch.float64, device=cache.device)
    blocks = cache[torch.as_tensor(table[:-(-n // R)], device=cache.device).long()]          # [m, H, bytes]
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


def _exact_chunk(c, s, q, table, kv_of):
    """q float64 [N,Hq,D]; kv_of(b): keys and values [ctx + n, Hkv, D] of a sequence."""
    D, Hq, G = c["D"], c["Hq"], c["Hq"] // c["Hkv"]
    out = torch.zeros((s["N"], Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((s["N"], Hq), dtype=torch.float64, device="cuda")
    first = 0
    for b, (l, n) in enumerate(zip(s["ctx_list"], s["news_list"])):
        row0 = first if c["packed"] else b * c["T"]
        first += n
        if l < 0 or n == 0:
            continue
        k, v = kv_of(b)
        for h in range(Hq):
            kh, vh = k[:, h // G].t().contiguous(), v[:, h // G].contiguous()
            for i0 in range(0, n, 4096):
                m = min(4096, n - i0)
                x = q[row0 + i0:row0 + i0 + m, h] @ kh / math.sqrt(D)
                x += torch.full((m, l + n), -math.inf, dtype=torch.float64, device="cuda").triu_(l + i0 + 1)
                norm = torch.logsumexp(x, -1)
                lse[row0 + i0:row0 + i0 + m, h] = norm
                out[row0 + i0:row0 + i0 + m, h] = torch.exp(x - norm[:, None]) @ vh
    return [out, lse] if c["lse"] else [out]


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


def exact(case, seed):
    global own
    c, was = dict(case), own
    own = False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    kind, R, D, got = c["kind"], c.get("R"), c["D"], []
    rows = _rows_of(c, s["news_list"])
    q, k, v = (s[n].flatten(0, -3) for n in "qkv")
    if kind == "rope":
        return [_exact_turn(c, s, q, rows), _exact_turn(c, s, k, rows)]
    table = s["table"].cpu().numpy()
    if kind == "chunk":
        return _exact_chunk(c, s, q.double(), table, lambda b: _exact_rows(s["cache"], R, D, table[b], s["ctx_list"][b] + s["news_list"][b]))
    slots = None
    if kind == "step":
        got += _exact_blocks(table, s["owned"].cpu().numpy(), s["free"].cpu().numpy(), int(s["n_free"][0]), s["ctx_list"], s["news_list"], R, c["T"])
        slots, table = got[0], got[4]
    turned = _exact_turn(c, s, q, rows)
    got.append(turned)
    new_k = _exact_values(_exact_turn(c, s, k, rows).float().to(torch.bfloat16))      # (k is rounded to bf16 before it is encoded, by definition)
    new_v = _exact_values(v)
    b, i, at = rows
    if kind == "step":
        first = np.concatenate(([0], np.cumsum(s["news_list"])))

        def kv_of(x):
            l, n = s["ctx_list"][x], s["news_list"][x]
            old = _exact_rows(s["cache"], R, D, table[x], l) if l > 0 else [torch.zeros((0, c["Hkv"], D), dtype=torch.float64, device="cuda")] * 2
            mine = torch.as_tensor(at[first[x]:first[x] + n], device="cuda")
            return [torch.cat((o, w[mine])) for o, w in zip(old, (new_k, new_v))]
        got += _exact_chunk(c, s, turned.float().to(torch.bfloat16).double(), table, kv_of)      # (and so is q, before attention)
    back = [torch.zeros((c["B"] * c["T"], c["Hkv"], D), dtype=torch.float64, device="cuda") for _ in range(2)]
    to = torch.as_tensor(b * c["T"] + i, device="cuda")
    if slots is not None:
        keep = torch.as_tensor(slots.flatten(), device="cuda")[to] >= 0
        to, at = to[keep], torch.as_tensor(at, device="cuda")[keep]
    for o, w in zip(back, (new_k, new_v)):
        o[to] = w[at]
    return got + [o[None] for o in back]


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = dict(case)
    kind, Hq, Hkv, D = c["kind"], c["Hq"], c["Hkv"], c["D"]
    ctx, news = _ctx(c), _news(c)
    live = [(l, n) for l, n in zip(ctx, news) if l >= 0]
    rows = sum(n for _, n in live)
    cached = Hkv * (D + D // 16)                                     # bytes of a row of the cache, K and V
    byt, flops = 0, 0.0
    if kind == "rope":
        byt += rows * (Hq + Hkv) * D * 4
    if kind in ("append", "step"):
        byt += rows * (Hq * D * 4 + Hkv * D * 4 + cached) + rows * cached + c["B"] * c["T"] * Hkv * D * 4      # rows in, and back out
    if kind != "chunk":
        byt += rows * 4 * c["axes"]
        flops += rows * (Hq + Hkv) * c["pairs"] * 6.0
    if kind in ("chunk", "step"):
        byt += sum(l + n for l, n in live) * cached + (rows + (rows if c["packed"] else c["B"] * c["T"])) * Hq * D * 2
        flops += 4.0 * Hq * D * sum(n * l + n * (n + 1) / 2 for l, n in live)
    if kind == "step":
        byt += 4 * (c["B"] * (c["T"] + 5) + 2 * sum(-(-n // c["R"]) for n in news))
    return {"bytes": byt, "flops": flops}
