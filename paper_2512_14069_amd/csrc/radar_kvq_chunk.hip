// Attention of chunks of new tokens over the paged 4-bit cache (radar_chunk_attention_kvq), for gfx950.
//
// Transposed as in radar_kvq_attention.hip, with its step of 32 keys (radar_kvq_step.h): a KV head's queries are counted through as columns,
// c = row * G + head of the group, and 64 of them are a wavefront's.  Row i sees keys up to ctx + i, so a column's keys are the first so many and only
// the last steps of a block of columns have anything to mask.
//
// Long chunks are bound by vector issue beside the matrix pipe: a step of 32 keys by 64 columns is 64 products and 249 vector instructions, of which about 110 turn
// codes into operands and as many are the softmax (16384 rows, 64 heads on 8, D = 128: 3.43 to 3.57 ms by machine, 1.23 to 1.28 PFLOP/s of what the mask leaves, the vector units issue in 77% of
// the cycles, the matrix pipe is busy in 57%; a large library product of bf16 reaches 1.37).  So a block is as wide as the registers allow, 64 columns, wherever there are rows
// enough.  Short chunks are bound by the way in and out of a block (finding it 0.6 to 2.6 us, its first loads 2 to 4, the merge 3 to 4: 2048 rows of 32 heads 48 us, of which 27
// would be steps), single tokens by the rows' bytes (64 of them behind 304824 rows 61 us, 5.45 TB/s; a copy of large buffers reaches 5.1, reading and writing).
// Two or four blocks side by side in one workgroup, for the L1's sake, gained nothing (a lighter batch of 16 chunks 369 us for 366, 16384 rows of 32 heads 1775 for 1779).
#include <algorithm>
#include <atomic>
#include <cmath>

#include "radar_host.h"
#include "radar_kvq_step.h"
#include "radar_rows.h"

namespace radar {

constexpr int kKcCols = 64;                    // columns of the widest block
constexpr int kKcTarget = 1024;                // most workgroups that what is divided is dealt to, and most parts
constexpr int kKcPlanned = 512;                // most sequences whose work every workgroup counts through.  Nothing is divided beyond (512 single tokens, one of them behind
                                               // 65536 rows, 71 us; 513 352)
constexpr int kKcArrived = 16;                 // counters are 64 bytes apart: atomics on one line wait for each other

struct KcArgs {
    int rbits, n_blocks;
    int64_t block_bytes;                       // of a block, all heads
    float scale_log2;
    const __bf16 *q;
    const unsigned char *cache;
    const int32_t *tables;
    __bf16 *out;
    float *lse;
    int Hq, M;
    int64_t q_sb, q_st, q_sh, o_sb, o_st, o_sh;
    float *part;                               // [kKcTarget] partial results: outputs, maxima (log2 units) and sums, in fp32
    unsigned int *arrived;                     // of a block's workgroups, kKcArrived words apart
};
// What a workgroup finds its work by: the kernel's leading arguments, which are in registers when it starts.
struct KcWork {
    const int32_t *ctx_lens, *row_starts, *n_new;
    int B, T, N, S;
    uint32_t heads;                            // KV heads, and their queries' heads above the 16th bit
    uint32_t dealt;                            // workgroups that divided work is dealt to (0: nothing is divided), and log2 of a level's keys above the 16th bit
    int least;                                 // least steps of a part (of four times as many nothing is divided: handing over and joining takes 6 us or so)
    uint32_t by_G;                             // 2^16 / G, rounded up
    __host__ __device__ int Hkv() const { return (int)(heads & 0xffff); }
    __host__ __device__ int G() const { return (int)(heads >> 16); }
    __host__ __device__ int target() const { return (int)(dealt & 0xffff); }
    __host__ __device__ int level_bits() const { return (int)(dealt >> 16); }
};
constexpr size_t kKcArgsAt = (sizeof(KcWork) + alignof(KcArgs) - 1) / alignof(KcArgs) * alignof(KcArgs);      // of the block behind them

// A sequence: rows of its prefix, new rows, rows that the tensors have for it, keys that its last row sees; the first of its rows.
struct KcSeq { int L, n, rows, total, row0; };
// Keys that row i behind L >= 0 others sees, of `most`: the sum may pass 31 bits.
__device__ __forceinline__ int kc_seen(int L, int i, int most) { return (int)min((uint32_t)L + (uint32_t)i + 1u, (uint32_t)most); }
template <bool UNIFORM = false>                // the same sequence in every lane
__device__ __forceinline__ KcSeq kc_seq(const KcWork &a, int b) {
    auto word = [](const int32_t *p, int i) { return UNIFORM ? uniform_word(p, i) : p[i]; };
    KcSeq s;
    if (a.row_starts) {
        const int from = min(max(word(a.row_starts, b), 0), a.N), to = min(max(word(a.row_starts, b + 1), from), a.N);
        s.rows = min(to - from, a.T);
        s.row0 = from;
        s.n = s.rows;
    } else {
        s.rows = a.T;
        s.row0 = b * a.T;
        s.n = a.n_new ? min(max(word(a.n_new, b), 0), a.T) : a.T;
    }
    s.L = min(word(a.ctx_lens, b), a.S);
    if (s.L < 0) s.n = 0, s.L = -1;
    s.total = s.n > 0 ? kc_seen(s.L, s.n - 1, a.S) : 0;
    return s;
}

// n / d, n < 2^23, by the reciprocal and one step either way.
__device__ __forceinline__ uint32_t kc_quotient(uint32_t n, uint32_t d) {
    int q = (int)((float)n * __builtin_amdgcn_rcpf((float)d)), r = (int)(n - (uint32_t)q * d);
    if (r < 0) --q;
    else if (r >= (int)d) ++q;
    return (uint32_t)q;
}
// (r0 + c) / G for a place r0 < G in a row and a column c < 64 behind it: at most 127 by 64 (exact with 16 bits), or at most once.
__device__ __forceinline__ int kc_rows_on(int t, const KcWork &a) {
    if (a.G() > kKcCols) return t >= a.G() ? 1 : 0;
    return (int)((uint32_t)t * a.by_G >> 16);
}

// What a workgroup does: a block of columns of a KV head, the first of them of row i0, and the steps [s0, s1) of it, one of `parts` such, whose results lie one behind the other
// from `slot` on.
struct KcItem { int b, hk, cg, i0, n, rows, row0, L, limit, s0, s1, part, parts, slot, unit; };
constexpr int kKcState = 16;

// Every item in one line, those with the most keys first, so that the workgroups that start last have little to do: by level (eighths or so of the longest
// context that a block's first row sees), in it sequence by sequence, from the last block of columns to the first, part by part and KV head by KV head (workgroups go
// to the eight XCDs in turn: a head's rows then stay in one L2).  A sequence's blocks are divided into parts of about `per` steps, none of fewer than `least`; `per` is the batch's
// work over the workgroups that it is dealt to, so that there are no more items than blocks and workgroups, and no more parts than workgroups.  A step
// of 16 columns counts for half a step of 64.  The quotients are by reciprocals, rounded to the safe side, as this is a chain that every workgroup goes through.
// All lanes call; the result is the same in all of them.
constexpr int kKcLevels = 8;
template <int COLS>
__device__ __forceinline__ int kc_blocks(int rows, int G) { return (rows * G + COLS - 1) / COLS; }                 // (rows * G < 2^28)
// Blocks of a sequence whose first row sees `keys` keys of others or more.
template <int COLS>
__device__ __forceinline__ int kc_beyond(const KcSeq &s, int cgs, int G, int keys) { return cgs - kc_blocks<COLS>(min(max(keys - s.L, 0), s.rows), G); }
template <int COLS>
__device__ __forceinline__ int kc_cost(const KcSeq &s, int G) {      // of a block of the sequence, in steps
    const int steps = (s.total + 31) >> 5;
    return COLS == 64 && s.n * G <= 16 ? steps >> 1 : steps;
}
template <int COLS>
__device__ __forceinline__ bool kc_find(KcItem &x, const KcWork &a, uint32_t item) {
    const int lane = lane_id(), Hkv = a.Hkv(), G = a.G();
    int p = 1, cgs, back = 0;                  // back: blocks behind this one
    uint32_t rel, slot0 = 0, unit0 = 0;        // rel: of the block's items; the sequence's first partial result and counter
    KcSeq s;
    if (a.B == 1) {                            // one sequence: nothing to count through, all of it in scalar registers
        s = kc_seq<true>(a, 0);
        cgs = kc_blocks<COLS>(s.rows, G);
        const uint32_t units = (uint32_t)(Hkv * cgs);
        const int cost = (s.total + 31) >> 5;
        if (cost >= 4 * a.least) p = max(min(a.target() / (int)max(units, 1u), cost / a.least), 1);
        if (item >= units * (uint32_t)p) return false;
        x.b = 0;
        rel = item;
    } else if (a.target() > 0) {
        auto seq = [&](int b0) { return kc_seq(a, min(b0 + lane, a.B - 1)); };
        s = seq(0);
        float work = 0.f;
        for (int b0 = 0; b0 < a.B; b0 += kWave) {
            const KcSeq t = b0 == 0 ? s : seq(b0);
            if (b0 + lane < a.B) work += (float)(kc_blocks<COLS>(t.rows, G) * Hkv) * (float)kc_cost<COLS>(t, G);
        }
        // (rounded up and down by more than what the sums and the reciprocal are off)
        const float per = fmaxf(wave_sum_f32(work) * 1.001f * __builtin_amdgcn_rcpf((float)a.target()), (float)a.least), inv = 0.999f * __builtin_amdgcn_rcpf(per);
        auto parts = [&](const KcSeq &t) { return (t.total + 31) >> 5 < 4 * a.least ? 1 : max((int)((float)kc_cost<COLS>(t, G) * inv), 1); };
        // the level: the highest on or above which there are more items than this one's number
        const int bits = a.level_bits();
        int level = 0;
        uint32_t first = 0;                    // items above the level
        if (bits < 31) {                       // (64 sequences at most)
            const int c = kc_blocks<COLS>(s.rows, G);
            const uint32_t each = lane < a.B ? (uint32_t)(Hkv * parts(s)) : 0u;
            int most = kKcLevels;              // no items there
            while (most - level > 1) {
                const int mid = (level + most) >> 1;
                const uint32_t n = readlane_u32(wave_scan_u32(each * (uint32_t)kc_beyond<COLS>(s, c, G, mid << bits)), kWave - 1);
                if (n > item) level = mid;
                else { most = mid; first = n; }
            }
        }
        int b0 = 0, hit = -1;
        for (; b0 < a.B; b0 += kWave) {
            if (b0 > 0) s = seq(b0);
            cgs = kc_blocks<COLS>(s.rows, G);
            p = parts(s);
            const bool there = b0 + lane < a.B;
            int lower = cgs, upper = 0;        // blocks on the level or above, and above
            if (bits < 31) {
                if (level > 0) lower = kc_beyond<COLS>(s, cgs, G, level << bits);
                if (level + 1 < kKcLevels) upper = kc_beyond<COLS>(s, cgs, G, (level + 1) << bits);
            }
            const uint32_t mine = there ? (uint32_t)(Hkv * cgs) : 0u, items = there ? (uint32_t)(Hkv * (lower - upper) * p) : 0u;
            const uint32_t incl = wave_scan_u32(items);
            uint32_t split = 0, whole = 0;
            if (__ballot(p > 1) != 0) {
                split = wave_scan_u32(p > 1 ? mine * (uint32_t)p : 0u);
                whole = wave_scan_u32(p > 1 ? mine : 0u);
            }
            const uint64_t behind = __ballot(first + incl > item);
            if (behind != 0) {
                hit = __ffsll((unsigned long long)behind) - 1;
                rel = item - (first + readlane_u32(incl, hit) - readlane_u32(items, hit));
                if (rel >= readlane_u32(items, hit)) return false;   // (only where row_starts falls)
                p = (int)readlane_u32((uint32_t)p, hit);
                cgs = (int)readlane_u32((uint32_t)cgs, hit);
                back = (int)readlane_u32((uint32_t)upper, hit);
                if (p > 1) {
                    const uint32_t m = readlane_u32(mine, hit);
                    slot0 += readlane_u32(split, hit) - m * (uint32_t)p;
                    unit0 += readlane_u32(whole, hit) - m;
                }
                break;
            }
            first += readlane_u32(incl, kWave - 1);
            slot0 += readlane_u32(split, kWave - 1);
            unit0 += readlane_u32(whole, kWave - 1);
        }
        if (hit < 0) return false;
        x.b = b0 + hit;
        s.L = (int)readlane_u32((uint32_t)s.L, hit); s.n = (int)readlane_u32((uint32_t)s.n, hit); s.rows = (int)readlane_u32((uint32_t)s.rows, hit);
        s.total = (int)readlane_u32((uint32_t)s.total, hit); s.row0 = (int)readlane_u32((uint32_t)s.row0, hit);
    } else {
        // too many sequences to count through: blocks of columns begin at first row * G / COLS + b, which leaves every sequence room
        const int block = (int)kc_quotient(item, (uint32_t)Hkv);
        int off;
        if (a.row_starts) {
            auto begin = [&](int b) { return (int64_t)min(max(a.row_starts[b], 0), a.N) * G / COLS + b; };
            x.b = max(last_at_most(a.B, block, begin), 0);
            off = (int)begin(x.b);
        } else {
            const int each = kc_blocks<COLS>(a.T, G);
            x.b = block / each;
            off = x.b * each;
        }
        x.b = __builtin_amdgcn_readfirstlane(x.b);
        if (x.b >= a.B) return false;
        s = kc_seq(a, x.b);
        cgs = kc_blocks<COLS>(s.rows, G);
        rel = item - (uint32_t)off * (uint32_t)Hkv;
        if (block < off || block - off >= cgs) return false;
    }
    const uint32_t turn = kc_quotient(rel, (uint32_t)Hkv), nth = p > 1 ? kc_quotient(turn, (uint32_t)p) : turn;
    x.hk = (int)(rel - turn * (uint32_t)Hkv);
    x.cg = cgs - 1 - back - (int)nth;
    const int part = (int)(turn - nth * (uint32_t)p);
    x.n = s.n; x.rows = s.rows; x.row0 = s.row0; x.L = s.L;
    const int c0 = x.cg * COLS;
    x.i0 = c0 / G;
    const int i1 = min(x.i0 + kc_rows_on(c0 - x.i0 * G + COLS - 1, a), s.n - 1);
    x.limit = x.i0 < s.n ? kc_seen(s.L, i1, s.total) : 0;
    const int steps = (x.limit + 31) >> 5;
    x.unit = (int)unit0 + x.cg * Hkv + x.hk;
    x.slot = 0;
    x.parts = 1;
    int each = steps, short_ones = 1;          // of x.parts parts the first short_ones have `each` steps, the others one more
    if (p > 1) {
        // of a sequence that is divided, as many parts as are as long as its last block's, but none of fewer keys than a.least steps have (so the part with the
        // last keys, whose last step may be half empty, is a longer one where there are any)
        const int longest = (s.total + 31) >> 5, wanted_steps = (longest + p - 1) / p;
        int wanted = max(min(min((steps + wanted_steps - 1) / max(wanted_steps, 1), p), (x.limit >> 5) / a.least), 1);
        x.slot = (int)(slot0 + (uint32_t)(x.cg * Hkv + x.hk) * (uint32_t)p);
        // (there is room by the bounds above; row_starts that falls may break them)
        if (x.cg < 0 || x.slot < 0 || x.slot > kKcTarget - wanted || (uint32_t)x.unit >= (uint32_t)kKcTarget) wanted = 1;
        x.parts = wanted;
        each = steps / wanted;
        short_ones = wanted - (steps - each * wanted);
    }
    if (x.cg < 0 || part >= x.parts) return false;
    x.part = part;
    x.s0 = part * each + max(part - short_ones, 0);
    x.s1 = x.s0 + each + (part >= short_ones ? 1 : 0);
    return true;
}

// An item waits in LDS, of which every wavefront has its own copy: taken from there it is in scalar registers, and nothing that was worked out to find it
// is kept in vector registers through the loop (which would spill).
template <typename T>
__device__ __forceinline__ T kc_recall(const int *from) {            // the same in every lane
    constexpr int N = sizeof(T) / 4;
    int v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __builtin_amdgcn_readfirstlane(from[i]);
    return __builtin_bit_cast(T, v);
}
__device__ __forceinline__ void kc_remember(int *to, KcItem x) {
    constexpr int N = sizeof(KcItem) / 4;
    static_assert(N <= kKcState);
    int v[N];
    __builtin_memcpy(v, &x, sizeof(x));
#pragma unroll
    for (int i = 0; i < N; ++i) to[i] = v[i];
}

// The arguments, read where a phase of the kernel needs them.
__device__ __forceinline__ KcWork kc_args_work() {
    const ArgBlock<KcWork> g = args_from_here<KcWork>(0);
    KcWork a;
    a.row_starts = g->row_starts; a.heads = g->heads; a.by_G = g->by_G;
    return a;
}
__device__ __forceinline__ KcArgs kc_args_loop() {
    const ArgBlock<KcArgs> g = args_from_here<KcArgs>(kKcArgsAt);
    KcArgs a;
    a.tables = g->tables; a.cache = g->cache; a.M = g->M; a.rbits = g->rbits; a.n_blocks = g->n_blocks; a.block_bytes = g->block_bytes;
    a.scale_log2 = g->scale_log2; a.q = g->q; a.q_sb = g->q_sb; a.q_st = g->q_st; a.q_sh = g->q_sh;
    return a;
}
__device__ __forceinline__ KcArgs kc_args_end() {
    const ArgBlock<KcArgs> g = args_from_here<KcArgs>(kKcArgsAt);
    KcArgs a;
    a.out = g->out; a.o_sb = g->o_sb; a.o_st = g->o_st; a.o_sh = g->o_sh; a.lse = g->lse; a.Hq = g->Hq; a.part = g->part; a.arrived = g->arrived;
    a.scale_log2 = g->scale_log2;
    return a;
}

// Where row i, head h of an item's sequence is in out, and its place in lse.
__device__ __forceinline__ __bf16 *kc_out(const KcArgs &a, bool packed, const KcItem &x, int i, int h) {
    const size_t row = packed ? (size_t)(x.row0 + i) * a.o_st : (size_t)x.b * a.o_sb + (size_t)i * a.o_st;
    return a.out + row + (size_t)h * a.o_sh;
}
template <int N>
__device__ __forceinline__ void kc_write(const KcArgs &a, bool packed, const KcItem &x, int i, int h, int d, const float (&acc)[N], float M, float l) {
    const float inv = l == 0.f ? 0.f : 1.0f / l;                     // (no key seen)
    __bf16 o[N] __attribute__((aligned(16)));
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = (__bf16)(acc[e] * inv);
    typedef uint32_t words __attribute__((ext_vector_type(N / 2)));
    words w;
    __builtin_memcpy(&w, o, sizeof(w));
    *reinterpret_cast<words *>(kc_out(a, packed, x, i, h) + d) = w;
    if (a.lse && d == 0) a.lse[(size_t)(x.row0 + i) * a.Hq + h] = l == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(l)) * kqLn2;
}

template <int D, int NC, int KW>
struct KcShape {
    static constexpr int NM = D / 16, CH = D / 32, COLS = 16 * NC;
    static constexpr int PASSES = NC * D > 256 ? 2 : 1, EP = 4 / PASSES, DP = D / PASSES, ROW = DP + 4;       // of the merge in LDS
    // The merge is each wavefront's for a share of the columns (2048 rows, four wavefronts: 48.8 us, 50.8 with all of it through LDS; eight: registers spill).
    static constexpr bool SPREAD = NC == 4 && (KW == 2 || KW == 4);
    static constexpr bool AS_HELD = SPREAD || KW == 1;               // partial results as registers hold them: [column block][output][lane], else [column][D]
    static constexpr int room() {                                    // queries' operands, then the merge's buffer (spread: behind them, as others may still read them)
        const int q = COLS * D * 2, merge = KW > 1 ? KW * COLS * ROW * 4 : 0;
        return SPREAD ? q + NC * (KW - 1) * NM / 2 * kWave * 16 : q > merge ? q : merge;
    }
    static constexpr int PART = COLS * D + 2 * COLS;                 // floats of a partial result
};
// Of a kernel whose blocks are 16 * MOST columns wide, or a half or a quarter of that.
template <int D, int MOST, int KW>
constexpr int kc_room() {
    const int half = KcShape<D, MOST == 1 ? 1 : 2, KW>::room(), all = KcShape<D, MOST, KW>::room(), one = KcShape<D, 1, KW>::room();
    return all > half ? (all > one ? all : one) : (half > one ? half : one);
}
template <int D, int MOST, int KW>
constexpr int kc_lds_bytes() { return kc_room<D, MOST, KW>() + (KW + 1) * 16 * MOST * 8 + 16 * MOST * 4 + KW * kKcState * 4; }

// One item.  KW wavefronts take its steps in turn and meet in LDS at the end.
template <int D, int NC, int MOST, int KW, bool FAR>
__device__ __forceinline__ void kc_item(unsigned char *smem, const int *state) {
    using S = KcShape<D, NC, KW>;
    constexpr int THREADS = KW * kWave;
    static_assert(S::room() <= kc_room<D, MOST, KW>());
    u32x4 *const s_q = reinterpret_cast<u32x4 *>(smem);              // [column block][chunk][lane], the lanes' operands
    float *const s_o = reinterpret_cast<float *>(smem);              // [wavefront][column][ROW]
    float *const s_m = reinterpret_cast<float *>(smem + kc_room<D, MOST, KW>()), *const s_l = s_m + KW * 16 * MOST;
    float *const s_M = s_l + KW * 16 * MOST, *const s_L = s_M + 16 * MOST;
    int *const s_lim = reinterpret_cast<int *>(s_L + 16 * MOST);       // keys that a column sees
    const int lane = lane_id(), w = KW > 1 ? __builtin_amdgcn_readfirstlane(wave_id()) : 0, r = lane & 15, grp = lane >> 4;

    KcItem p = kc_recall<KcItem>(state);
    KcArgs a = kc_args_loop();
    const KcWork g = kc_args_work();
    const int32_t *const table = (const int32_t *)(uintptr_t)kq_scalar(a.tables + (size_t)p.b * a.M);
    const kq_bytes base = (kq_bytes)(uintptr_t)kq_scalar(a.cache + (size_t)p.hk * KvqChunk<D>::bytes(1 << a.rbits));
    const int mine = p.s0 + w, hidden = kc_seen(p.L, p.i0, p.limit);          // (keys that the first column sees)
    const bool active = mine < p.s1;
    KqK<D> k;
    KqV v;
    KqIds id{0, 0}, nid{0, 0};
    if (active) {
        id = kq_ids(a, table, mine * 32, p.limit);
        nid = kq_ids(a, table, min(mine + KW, p.s1 - 1) * 32, p.limit);
    }
    // the queries are asked for while the blocks' numbers are on their way, and the first step's codes behind them
    constexpr int QS = (NC * S::CH + KW - 1) / KW;
    u32x4 y[QS];
    {
        const int G = g.G(), r0 = p.cg * 16 * MOST - p.i0 * G;
        const __bf16 *const q0 = a.q + (g.row_starts ? (size_t)p.row0 * a.q_st : (size_t)p.b * a.q_sb) + (size_t)(p.hk * G) * a.q_sh;
#pragma unroll
        for (int j = 0; j < QS; ++j) {
            const int x = w + j * KW, t = r0 + x / S::CH * 16 + r, on = kc_rows_on(t, g), i = p.i0 + on;
            y[j] = u32x4{0, 0, 0, 0};
            if (i < p.n && x < NC * S::CH) y[j] = *reinterpret_cast<const u32x4 *>(q0 + (size_t)i * a.q_st + (size_t)(t - on * G) * a.q_sh + (D / 4) * grp + 8 * (x % S::CH));
        }
        if (w == 0 && lane < S::COLS) {
            const int i = p.i0 + kc_rows_on(r0 + lane, g);
            s_lim[lane] = i < p.n ? kc_seen(p.L, i, p.limit) : 0;
        }
    }
    if (active) {
        const KqBase at = kq_base<D>(a, base, id, mine * 32);
        int lane2 = lane;
        asm volatile("" : "+v"(lane2));
        kq_load_k<D, FAR>(k, at, lane2);
        kq_load_v<D, FAR>(v, a, at, lane2);
    }
#pragma unroll
    for (int j = 0; j < QS; ++j)
        if (w + j * KW < NC * S::CH) s_q[(w + j * KW) * kWave + lane] = y[j];
    if (lane < S::COLS) s_m[w * S::COLS + lane] = -kKqNone;          // the references of this wavefront's columns, as scores
    floatx4 oacc[S::NM][NC];
    float negref[NC], l_run[NC];
#pragma unroll
    for (int n = 0; n < NC; ++n) {
        negref[n] = kKqNone;
        l_run[n] = 0.f;
#pragma unroll
        for (int m = 0; m < S::NM; ++m) oacc[m][n] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    __syncthreads();
    auto qop = [&](int n, int ch) { return __builtin_bit_cast(bf16x8, s_q[(n * S::CH + ch) * kWave + lane]); };
    const int last = p.s1 - 1;                                       // (past it, rows that are there are asked for once more, in vain)
    for (int s = mine; s < p.s1; s += KW) {
        const int next = min(s + KW, last);
        KqIds nnid;
        kq_step<D, NC, FAR || NC == 1 ? 2 : 4>(k, v, id, qop, [&] {
            nnid = kq_ids(a, table, min(s + 2 * KW, last) * 32, p.limit);
            kq_load_k<D, FAR>(k, kq_base<D>(a, base, nid, next * 32), lane);
        }, oacc, negref, l_run, [&](int col, int) {
            const int sees = s_lim[col] - s * 32;
            return sees >= 32 ? ~0u : sees <= 0 ? 0u : (1u << sees) - 1;
        }, s_m, a, s * 32, hidden, p.limit);
        kq_load_v<D, FAR>(v, a, kq_base<D>(a, base, nid, next * 32), lane);
        id = nid;
        nid = nnid;
    }
    __builtin_amdgcn_s_setprio(0);

    a = kc_args_end();
    const KcWork e = kc_args_work();
    const int G = e.G();
    const bool packed = e.row_starts != nullptr;
    p = kc_recall<KcItem>(state);
    const int r0 = p.cg * 16 * MOST - p.i0 * G;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));                                    // (addresses are worked out here, and not kept from the start)
    const int r2 = tid & 15, grp2 = (tid >> 4) & 3;
    const int live = min(p.n * G - p.cg * 16 * MOST, S::COLS);       // columns of the block that there are
    float *const to = a.part + (size_t)(p.slot + p.part) * KcShape<D, MOST, KW>::PART;
    auto hand_over = [&](int at, float x0, float x1) {
        store_shared_result(reinterpret_cast<uint64_t *>(to + at), (uint64_t)__float_as_uint(x1) << 32 | __float_as_uint(x0));
    };
    auto hand_over_sum = [&](int col, float M, float l) {
        store_shared_result(reinterpret_cast<uint64_t *>(to + S::COLS * D + 2 * col), (uint64_t)__float_as_uint(l) << 32 | __float_as_uint(M));
    };
    // a column's reference in log2 units (a far one is good to 2^-24 of itself, as the scores are)
    auto reference = [&](int n, float l) {
        const float m = s_m[w * S::COLS + n * 16 + r2];
        return l == 0.f ? -kKqNone : kq_is_far(negref[n]) ? fminf(fmaxf(m * a.scale_log2, -kKqNone), kKqNone) : -negref[n];
    };
    // a lane's outputs of its column in block n
    auto leave = [&](int n, float M, float l) {
        const int col = n * 16 + r2, on = kc_rows_on(r0 + col, e), i = p.i0 + on, h = p.hk * G + r0 + col - on * G;
        if (col >= live) return;
        if (p.parts > 1) {
#pragma unroll
            for (int m = 0; m < S::NM; ++m) {
                const floatx4 x = oacc[m][n];
                const int at = ((n * S::NM + m) * kWave + (tid & (kWave - 1))) * 4;
                hand_over(at, x[0], x[1]);
                hand_over(at + 2, x[2], x[3]);
            }
            if (grp2 == 0) hand_over_sum(col, M, l);
            return;
        }
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            float x[S::NM];
#pragma unroll
            for (int m = 0; m < S::NM; ++m) x[m] = oacc[m][n][y];
            kc_write(a, packed, p, i, h, D / 4 * grp2 + y * S::NM, x, M, l);
        }
    };
    if constexpr (KW == 1) {
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            const float l = kq_column_sum(l_run[n]);
            leave(n, reference(n, l), l);
        }
    } else {
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            const float l = kq_column_sum(l_run[n]), M = reference(n, l);
            if (grp2 == 0) {
                s_m[w * S::COLS + n * 16 + r2] = M;
                s_l[w * S::COLS + n * 16 + r2] = l;
            }
        }
        if constexpr (S::SPREAD) {
            // Every wavefront adds up 16 of the columns, or 32.  The others' shares of them come through LDS as they lie in the registers, half the outputs at a time, and are
            // scaled where they are added.
            constexpr int OWN = NC / KW;                             // column blocks of a wavefront
            floatx4 *const s_x = reinterpret_cast<floatx4 *>(smem + S::COLS * D * 2);                // [column block][wavefront behind the owner][output][lane]
            auto place = [&](int n, int behind, int m) { return ((n * (KW - 1) + behind - 1) * (S::NM / 2) + m) * kWave + (tid & (kWave - 1)); };
            float scl[OWN][KW], M[OWN], l[OWN];
            auto one_half = [&](auto which) {
                constexpr int M0 = decltype(which)::value;
                if (M0 > 0) __syncthreads();
#pragma unroll
                for (int n = 0; n < NC; ++n)
#pragma unroll
                    for (int m = 0; m < S::NM / 2; ++m)
                        if (w != n / OWN) s_x[place(n, (w - n / OWN) & (KW - 1), m)] = oacc[M0 + m][n];
                __syncthreads();
#pragma unroll
                for (int n = 0; n < NC; ++n) {
                    if (w != n / OWN) continue;
                    const int o = n % OWN, col = n * 16 + r2;
                    if constexpr (M0 == 0) {
                        M[o] = -kKqNone;
                        l[o] = 0.f;
#pragma unroll
                        for (int x = 0; x < KW; ++x) M[o] = fmaxf(M[o], scl[o][x] = s_m[((w + x) & (KW - 1)) * S::COLS + col]);
#pragma unroll
                        for (int x = 0; x < KW; ++x) {
                            scl[o][x] = __builtin_amdgcn_exp2f(scl[o][x] - M[o]);
                            l[o] += s_l[((w + x) & (KW - 1)) * S::COLS + col] * scl[o][x];
                        }
                    }
#pragma unroll
                    for (int m = 0; m < S::NM / 2; ++m) {
                        oacc[M0 + m][n] *= scl[o][0];
#pragma unroll
                        for (int x = 1; x < KW; ++x) oacc[M0 + m][n] += s_x[place(n, x, m)] * scl[o][x];
                    }
                    if constexpr (M0 > 0) leave(n, M[o], l[o]);
                }
            };
            one_half(std::integral_constant<int, 0>{});
            one_half(std::integral_constant<int, S::NM / 2>{});
        } else {
        __syncthreads();
        if (tid < S::COLS) {
            float m[KW], M = -kKqNone, l = 0.f;
#pragma unroll
            for (int x = 0; x < KW; ++x) m[x] = s_m[x * S::COLS + tid];
#pragma unroll
            for (int x = 0; x < KW; ++x) M = fmaxf(M, m[x]);
#pragma unroll
            for (int x = 0; x < KW; ++x) l += s_l[x * S::COLS + tid] * __builtin_amdgcn_exp2f(m[x] - M);
            s_M[tid] = M;
            s_L[tid] = l;
        }
        __syncthreads();
        float scl[NC];
#pragma unroll
        for (int n = 0; n < NC; ++n) scl[n] = __builtin_amdgcn_exp2f(s_m[w * S::COLS + n * 16 + r2] - s_M[n * 16 + r2]);
        constexpr int Q4 = S::DP / 4, TPC = THREADS / S::COLS < Q4 ? THREADS / S::COLS : Q4, IPT = Q4 / TPC;      // fours of a pass; lanes of a column
#pragma unroll
        for (int pass = 0; pass < S::PASSES; ++pass) {               // of a column: d = D/4 * part + (4 / PASSES * pass + e) * NM + m
            if (pass > 0) __syncthreads();
#pragma unroll
            for (int n = 0; n < NC; ++n)
#pragma unroll
                for (int e = 0; e < S::EP; ++e)
#pragma unroll
                    for (int m = 0; m < S::NM; m += 4) {
                        floatx4 x;
#pragma unroll
                        for (int y = 0; y < 4; ++y) x[y] = oacc[m + y][n][pass * S::EP + e] * scl[n];
                        *reinterpret_cast<floatx4 *>(s_o + (w * S::COLS + n * 16 + r2) * S::ROW + (grp2 * S::EP + e) * S::NM + m) = x;
                    }
            __syncthreads();
            int lane2 = threadIdx.x;
            asm volatile("" : "+v"(lane2));
            const int col = lane2 / TPC, mx = lane2 % TPC * 4, on = kc_rows_on(r0 + col, e), i = p.i0 + on, h = p.hk * G + r0 + col - on * G;
            if (col < live) {
                const float M = s_M[col], l = s_L[col];
#pragma unroll
                for (int z = 0; z < IPT; ++z) {
                    const int x = z * TPC * 4 + mx, d = D / 4 * (x / (S::EP * S::NM)) + pass * S::EP * S::NM + x % (S::EP * S::NM);
                    floatx4 acc = *reinterpret_cast<const floatx4 *>(s_o + col * S::ROW + x);
#pragma unroll
                    for (int y = 1; y < KW; ++y) acc += *reinterpret_cast<const floatx4 *>(s_o + (y * S::COLS + col) * S::ROW + x);
                    if (p.parts > 1) {
                        hand_over(col * D + d, acc[0], acc[1]);
                        hand_over(col * D + d + 2, acc[2], acc[3]);
                        if (d == 0) hand_over_sum(col, M, l);
                    } else {
                        const float o[4] = {acc[0], acc[1], acc[2], acc[3]};
                        kc_write(a, packed, p, i, h, d, o, M, l);
                    }
                }
            }
        }
        }
    }
    if (p.parts == 1) return;
    // The block's workgroup that arrives last has all the parts, its own among them, join.
    __syncthreads();
    unsigned int *const counter = a.arrived + p.unit * kKcArrived;
    if ((int)publish_then_ticket(counter, reinterpret_cast<unsigned int *>(s_m)) != p.parts - 1) return;
    if (threadIdx.x == 0) store_shared_result(counter, 0u);
    const float *const from = a.part + (size_t)p.slot * KcShape<D, MOST, KW>::PART;
    constexpr size_t apart = KcShape<D, MOST, KW>::PART;
    int first = threadIdx.x;
    asm volatile("" : "+v"(first));
    // M and l are the column's, o four outputs of it from each part, in turn
    struct Sum { float M = -kKqNone, l = 0.f; };
    auto join = [&](int col, auto &acc, auto place) {                // acc: fours, the x-th of them at place(x)
        constexpr int Q = sizeof(acc) / sizeof(floatx4), U = Q == 1 ? 4 : 1;
        Sum t;
#pragma unroll
        for (int x = 0; x < Q; ++x) acc[x] = floatx4{0.f, 0.f, 0.f, 0.f};
        for (int y0 = 0; y0 < p.parts; y0 += U) {
            uint64_t ml[U], lo[U][Q], hi[U][Q];
#pragma unroll
            for (int y = 0; y < U; ++y) {
                const float *const part = from + (size_t)min(y0 + y, p.parts - 1) * apart;
                ml[y] = load_shared_result(reinterpret_cast<const uint64_t *>(part + S::COLS * D + 2 * col));
#pragma unroll
                for (int x = 0; x < Q; ++x) {
                    lo[y][x] = load_shared_result(reinterpret_cast<const uint64_t *>(part + place(x)));
                    hi[y][x] = load_shared_result(reinterpret_cast<const uint64_t *>(part + place(x) + 2));
                }
            }
            float Mn = t.M;
#pragma unroll
            for (int y = 0; y < U; ++y) Mn = fmaxf(Mn, __uint_as_float((uint32_t)ml[y]));
            const float f0 = __builtin_amdgcn_exp2f(t.M - Mn);
            t.M = Mn;
            t.l *= f0;
#pragma unroll
            for (int x = 0; x < Q; ++x) acc[x] *= f0;
#pragma unroll
            for (int y = 0; y < U; ++y) {
                if (y0 + y >= p.parts) break;                        // (the last part once more)
                const float f = __builtin_amdgcn_exp2f(__uint_as_float((uint32_t)ml[y]) - Mn);
                t.l += __uint_as_float((uint32_t)(ml[y] >> 32)) * f;
#pragma unroll
                for (int x = 0; x < Q; ++x)
                    acc[x] += floatx4{__uint_as_float((uint32_t)lo[y][x]), __uint_as_float((uint32_t)(lo[y][x] >> 32)), __uint_as_float((uint32_t)hi[y][x]),
                                      __uint_as_float((uint32_t)(hi[y][x] >> 32))} * f;
            }
        }
        return t;
    };
    if constexpr (S::AS_HELD) {
        constexpr int Q = S::NM / 2;                                 // a lane's turn: half the outputs of its column and quarter
        for (int x = first; x < NC * 2 * kWave; x += THREADS) {
            const int n = x / (2 * kWave), half = x / kWave % 2, l2 = x % kWave, col = n * 16 + l2 % 16;
            if (col >= live) continue;
            floatx4 acc[Q];
            const Sum t = join(col, acc, [&](int y) { return ((n * S::NM + half * Q + y) * kWave + l2) * 4; });
            const int on = kc_rows_on(r0 + col, e), i = p.i0 + on, h = p.hk * G + r0 + col - on * G;
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                float o[Q];
#pragma unroll
                for (int m = 0; m < Q; ++m) o[m] = acc[m][y];
                kc_write(a, packed, p, i, h, D / 4 * (l2 / 16) + y * S::NM + half * Q, o, t.M, t.l);
            }
        }
    } else {
        for (int x = first; x < live * (D / 4); x += THREADS) {
            const int col = x / (D / 4), d = x % (D / 4) * 4, on = kc_rows_on(r0 + col, e), i = p.i0 + on, h = p.hk * G + r0 + col - on * G;
            floatx4 acc[1];
            const Sum t = join(col, acc, [&](int) { return col * D + d; });
            const float o[4] = {acc[0][0], acc[0][1], acc[0][2], acc[0][3]};
            kc_write(a, packed, p, i, h, d, o, t.M, t.l);
        }
    }
}

// MOST: blocks of 16, 32 or 64 columns.  With 16, for single tokens and where there are few rows, registers are left for twice as many wavefronts.
template <int D, int MOST, int KW, bool FAR>
__global__ __launch_bounds__(KW * kWave, MOST == 1 ? 4 : 2) void kvq_chunk_kernel(const int32_t *ctx_lens, const int32_t *row_starts, const int32_t *n_new, int B, int T, int N,
                                                                                 int S, uint32_t heads, uint32_t dealt, int least, uint32_t by_G, KcArgs) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    int *const state = reinterpret_cast<int *>(smem + kc_lds_bytes<D, MOST, KW>() - KW * kKcState * 4) + (KW > 1 ? wave_id() : 0) * kKcState;
    const KcWork work{ctx_lens, row_starts, n_new, B, T, N, S, heads, dealt, least, by_G};
    KcItem p;
    constexpr int COLS = 16 * MOST;
    if (!kc_find<COLS>(p, work, blockIdx.x)) return;                       // (the same in all wavefronts)
    kc_remember(state, p);
    const int G = work.G(), c0 = p.cg * COLS, live = min(max(p.n * G - c0, 0), COLS), there = min(p.rows * G - c0, COLS);
    if (live < there && p.s0 == 0) {                                 // rows that are not there, of sequences that are not there: zeros
        const KcArgs e = kc_args_end();
        for (int x = threadIdx.x; x < (there - live) * (D / 8); x += KW * kWave) {
            const int t = c0 - p.i0 * G + live + x / (D / 8), on = kc_rows_on(t, work), i = p.i0 + on, h = p.hk * G + t - on * G;
            *reinterpret_cast<u32x4 *>(kc_out(e, row_starts != nullptr, p, i, h) + x % (D / 8) * 8) = u32x4{0, 0, 0, 0};
            if (e.lse && x % (D / 8) == 0) e.lse[(size_t)(p.row0 + i) * e.Hq + h] = 0.f;
        }
    }
    if (live == 0) return;
    if (MOST == 1 || __builtin_amdgcn_readfirstlane(live) <= 16) kc_item<D, 1, MOST, KW, FAR>(smem, state);
    else if (MOST == 2 || __builtin_amdgcn_readfirstlane(live) <= 32) kc_item<D, MOST == 1 ? 1 : 2, MOST, KW, FAR>(smem, state);
    else kc_item<D, MOST, MOST, KW, FAR>(smem, state);
}

}  // namespace radar

using namespace radar;

static radar_status check_chunk(const radar_kvq_chunk_desc *d) {
    if (!d) return RADAR_INVALID_ARG;
    const radar_status st = kvq_check(&d->cache);
    if (st != RADAR_OK) return st;
    if (d->B < 1 || d->T_max < 1 || d->N < 0 || d->Hq < 1 || d->max_blocks < 1 || d->S_max < 1 || d->Hq % d->cache.Hkv != 0) return RADAR_INVALID_ARG;
    if ((d->S_max - 1) / d->cache.block_rows >= d->max_blocks) return RADAR_INVALID_ARG;
    if (d->rows_per_split < 0 || d->rows_per_split % 64 != 0) return RADAR_INVALID_ARG;
    if (!(d->softmax_scale >= 0.f)) return RADAR_INVALID_ARG;
    if (d->B > 65535 || d->Hq > 65535 || d->S_max > INT32_MAX - 4096 || d->N > INT32_MAX) return RADAR_UNSUPPORTED_SHAPE;
    return RADAR_OK;
}

// Blocks of columns of a KV head, at most: of [B,T_max], or of N rows in B sequences.
static int64_t chunk_blocks(const radar_kvq_chunk_desc *d, bool packed, int cols) {
    const int64_t G = d->Hq / d->cache.Hkv;
    return packed ? d->N * G / cols + d->B : (int64_t)d->B * (((int64_t)d->T_max * G + cols - 1) / cols);
}

struct KcRoom { size_t off_part, bytes; };
static KcRoom chunk_room(int D) {
    KcRoom r;
    r.off_part = (size_t)kKcTarget * kKcArrived * sizeof(unsigned int);       // counters first: all calls leave them at zero
    r.bytes = r.off_part + (size_t)kKcTarget * kKcCols * (D + 2) * sizeof(float);
    return r;
}

// Columns of a block, wavefronts of a workgroup, and whether long blocks are divided: whichever takes least by a model of rounds (a step of every wavefront), what a block costs
// besides and what a part costs to join.  Its figures are a fit to the times of all seven kinds, divided and whole, in 155 shapes (1 to 16384 rows in 1 to 256 sequences behind 0 to
// 100000, single tokens, trees, prompts and mixtures; groups of 1, 4 and 8, D = 64 and 128, one MI355X); what it picks took 1.5% longer than the best of them in the mean, 29% at most (one
// piece of a prompt among 15 tokens).  us, best and worst kind: 64 rows 5.6 (16 columns, four wavefronts) to 12; 64 behind 16384 29 (32, eight) to 104; 512 behind 16384 123 (64, eight) to
// 215; 2048 47 (64, four) to 89; 16384 1764 (64, one) to 3298.  Divided and whole: 128 rows behind 2048 16.7 and 12.8, five rows each of eight sequences behind 2048 16.0 and 13.5, a single
// token behind 2048 9.2 and 10.9.
struct KcKind {
    int most, kw, slots;                                   // blocks of 16 * most columns; wavefronts; workgroups that the chip holds at once (at D = 128: D = 64 has registers
                                                           // for up to 1.75 times as many of 16 columns and twice as many of 32, which the plan leaves unused)
    double alone, full, end;                               // us: a round of a workgroup that is alone, and with as many as there is room for; what a block costs besides
};
constexpr KcKind kKcKinds[] = {{1, 8, 512, 0.68, 1.33, 4.56}, {1, 4, 1024, 0.81, 1.31, 3.87}, {2, 8, 256, 0.71, 1.01, 5.21},
                               {4, 8, 256, 1.24, 1.44, 8.8}, {4, 4, 512, 1.0, 1.53, 4.92}, {4, 2, 1024, 1.26, 1.42, 7.42}, {4, 1, 2048, 1.05, 1.38, 6.5}};
constexpr double kKcAlone = 0.31;                          // a round is as long as alone up to this share of the workgroups that there is room for
constexpr int kKcWhole = 1 << 28;                          // least steps of a part where nothing is divided
struct KcPlan {
    int kind, target, least, level_bits;
    int64_t items;
};
static KcPlan plan_chunk(const radar_kvq_chunk_desc *d, bool packed) {
    KcPlan p;
    const int64_t G = d->Hq / d->cache.Hkv;
    const double hi = (double)(((int64_t)d->S_max + 31) / 32), lo = (double)(std::max(d->S_max - d->T_max, 0) / 32), mid = 0.5 * (hi + lo);
    // the least steps of a part: a part costs about a third of a round to join, so that the longest context is best divided by the root of its steps
    // (us, one sequence of 16384 rows, a single token, parts of 16 / 32 steps: 13.4 12.6; 2048 rows 9.2 10.9, 64 rows behind them 20.1 23.2)
    auto least = [&](const KcKind &k) { return d->rows_per_split ? d->rows_per_split / 32 : std::max(2 * k.kw, (int)(1.5 * std::sqrt(hi))); };
    double best = 1e300;
    p.kind = 0;
    p.items = 0;
    for (int x = 0; x < (int)(sizeof(kKcKinds) / sizeof(kKcKinds[0])); ++x) {
        const KcKind &k = kKcKinds[x];
        int64_t units = chunk_blocks(d, packed, 16 * k.most) * d->cache.Hkv;
        if (packed && d->B <= kKcPlanned) units = std::min(units, chunk_blocks(d, false, 16 * k.most) * d->cache.Hkv);      // (counted through, not looked up by where they begin)
        if (units >= (1 << 22) || (k.most > 1 && p.items > 0 && (int64_t)d->T_max * G <= 8 * k.most)) continue;      // (half empty: only where others are too many)
        const int64_t dealt = std::min(kKcTarget, k.slots) / units, long_enough = (int64_t)hi / least(k);
        const int64_t divided = hi < 4.0 * least(k) ? 1 : std::max<int64_t>(std::min(dealt, long_enough), 1);
        for (int64_t parts = divided; parts > 0; parts = parts > 1 && !d->rows_per_split ? 1 : 0) {
            const double fill = (double)(units * parts) / k.slots, round = k.alone + (k.full - k.alone) * std::max(std::min(fill, 1.0) - kKcAlone, 0.0) / (1.0 - kKcAlone);
            const double end = k.end + (parts > 1 ? 0.52 + 0.54 * (double)parts * k.most : 0.0), steps = 1.0 / (double)parts / k.kw;
            const double us = std::max(std::ceil(hi * steps) * round + end, fill * (mid * steps * round + end));          // the longest block; all of them
            if (us < best) { best = us; p.kind = x; p.items = units; p.least = parts == 1 && divided > 1 ? kKcWhole : least(k); }
        }
    }
    const KcKind &k = kKcKinds[p.kind];
    p.target = d->B <= kKcPlanned ? std::min(kKcTarget, k.slots) : 0;
    p.level_bits = 31;
    if (d->B > 1 && d->B <= kWave)                         // (one sequence's blocks are in that order anyway)
        for (p.level_bits = 5; ((int64_t)d->S_max >> p.level_bits) >= kKcLevels; ++p.level_bits) {}
    p.items += p.target;
    return p;
}

extern "C" size_t radar_chunk_attention_kvq_workspace_bytes(const radar_kvq_chunk_desc *d) {
    if (check_chunk(d) != RADAR_OK) return 0;
    return chunk_room(d->cache.D).bytes;
}

template <int D, int MOST, int KW, bool FAR>
static hipError_t launch_chunk(const char *name, const KcWork &w, const KcArgs &a, int64_t items, hipStream_t s) {
    constexpr int bytes = kc_lds_bytes<D, MOST, KW>();
    static std::atomic<uint64_t> configured{0};            // devices on which the kernel may have so much LDS (two threads may both say so)
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    const uint64_t bit = 1ull << (device & 63);
    if (device > 63 || !(configured.load(std::memory_order_relaxed) & bit)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void *>(&kvq_chunk_kernel<D, MOST, KW, FAR>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
        configured.fetch_or(bit, std::memory_order_relaxed);
    }
    return launch(name, kvq_chunk_kernel<D, MOST, KW, FAR>, dim3((unsigned)items), dim3(KW * kWave), bytes, s, w.ctx_lens, w.row_starts, w.n_new,
                  w.B, w.T, w.N, w.S, w.heads, w.dealt, w.least, w.by_G, a);
}
template <int D, bool FAR>
static hipError_t launch_chunk(const KcWork &w, const KcArgs &a, const KcPlan &p, hipStream_t s) {
    switch (p.kind) {
        case 0: return launch_chunk<D, 1, 8, FAR>("kvq_chunk_16x8", w, a, p.items, s);
        case 1: return launch_chunk<D, 1, 4, FAR>("kvq_chunk_16x4", w, a, p.items, s);
        case 2: return launch_chunk<D, 2, 8, FAR>("kvq_chunk_32x8", w, a, p.items, s);
        case 3: return launch_chunk<D, 4, 8, FAR>("kvq_chunk_64x8", w, a, p.items, s);
        case 4: return launch_chunk<D, 4, 4, FAR>("kvq_chunk_64x4", w, a, p.items, s);
        case 5: return launch_chunk<D, 4, 2, FAR>("kvq_chunk_64x2", w, a, p.items, s);
        default: return launch_chunk<D, 4, 1, FAR>("kvq_chunk_64x1", w, a, p.items, s);
    }
}

extern "C" radar_status radar_chunk_attention_kvq(const void *q, const void *cache, const int32_t *block_tables, const int32_t *ctx_lens,
                                                  const int32_t *row_starts, const int32_t *n_new, void *out, float *lse_out,
                                                  const radar_kvq_chunk_desc *d, void *workspace, size_t workspace_bytes, void *stream) {
    if (!q || !cache || !block_tables || !ctx_lens || !out || !workspace || out == q || (row_starts && n_new)) return RADAR_INVALID_ARG;
    const radar_status st = check_chunk(d);
    if (st != RADAR_OK) return st;
    if (!row_starts && d->N != (int64_t)d->B * d->T_max) return RADAR_INVALID_ARG;
    const int64_t Hkv = d->cache.Hkv;
    if (chunk_blocks(d, row_starts != nullptr, kKcCols) * Hkv >= (1 << 22)) return RADAR_UNSUPPORTED_SHAPE;
    const KcRoom room = chunk_room(d->cache.D);
    if (workspace_bytes < room.bytes) return RADAR_WORKSPACE_TOO_SMALL;
    if (((uintptr_t)workspace & 255) != 0) return RADAR_INVALID_ARG;
    KcArgs a;
    a.q = static_cast<const __bf16 *>(q); a.cache = static_cast<const unsigned char *>(cache);
    a.tables = block_tables;
    a.out = static_cast<__bf16 *>(out); a.lse = lse_out;
    a.Hq = d->Hq; a.M = d->max_blocks;
    a.rbits = kvq_log2(d->cache.block_rows); a.n_blocks = d->cache.n_blocks;
    const int64_t D = d->cache.D;
    a.block_bytes = Hkv * d->cache.block_rows * (D + D / 16);
    a.q_sh = d->q_stride_h ? d->q_stride_h : D;
    a.q_st = d->q_stride_t ? d->q_stride_t : D * d->Hq;
    a.q_sb = d->q_stride_b ? d->q_stride_b : D * d->Hq * d->T_max;
    a.o_sh = d->out_stride_h ? d->out_stride_h : D;
    a.o_st = d->out_stride_t ? d->out_stride_t : D * d->Hq;
    a.o_sb = d->out_stride_b ? d->out_stride_b : D * d->Hq * d->T_max;
    const uintptr_t al = (uintptr_t)q | (uintptr_t)cache | (uintptr_t)out;
    const int64_t strides = a.q_sh | a.q_st | a.q_sb | a.o_sh | a.o_st | a.o_sb;
    if ((al & 15) != 0 || (strides & 7) != 0 || strides < 0) return RADAR_INVALID_ARG;
    if (d->N == 0) return RADAR_OK;
    a.scale_log2 = (d->softmax_scale != 0.f ? d->softmax_scale : 1.0f / sqrtf((float)D)) * kqLog2e;
    char *ws = static_cast<char *>(workspace);
    a.arrived = reinterpret_cast<unsigned int *>(ws);
    a.part = reinterpret_cast<float *>(ws + room.off_part);
    const KcPlan p = plan_chunk(d, row_starts != nullptr);
    const KcWork w{ctx_lens, row_starts, n_new, d->B, d->T_max, (int)d->N, d->S_max, (uint32_t)Hkv | (uint32_t)(d->Hq / d->cache.Hkv) << 16,
                   (uint32_t)p.target | (uint32_t)p.level_bits << 16, p.least, (uint32_t)((65535 + d->Hq / Hkv) / (d->Hq / Hkv))};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool far = (int64_t)a.n_blocks * a.block_bytes > UINT32_MAX;
    const hipError_t e = D == 128 ? (far ? launch_chunk<128, true>(w, a, p, s) : launch_chunk<128, false>(w, a, p, s))
                                  : (far ? launch_chunk<64, true>(w, a, p, s) : launch_chunk<64, false>(w, a, p, s));
    return e == hipSuccess ? RADAR_OK : RADAR_HIP_ERROR;
}
