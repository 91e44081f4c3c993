// Tree-verify attention over the paged 4-bit cache (radar_tree_attention_kvq), for gfx950.
//
// As in radar_attention.hip everything is kept transposed: S^T = K Q^T (keys x queries) and O^T = V^T P^T, so that a lane owns one
// query column and the exponentiated scores sit in its registers as the next product wants them.  The queries of a KV head's group
// are counted through as columns, c = node * G + head of the group, so that a tree's live columns are the first ones.
//
// Codes turn into MFMA operands in registers (16x16x32, bf16: what a code stands for is exact there).  A lane of the K operand
// takes a whole stretch of its key's codes, 16 bytes at D = 128: the sum over d may run in any order, so its eights are dealt to the
// products as they lie.  A lane of the V operand holds eight keys of one d, and the layout puts the codes of eight keys for the
// same eight d side by side: 32 bytes are the operands of eight products.
//
// What bounds it (one MI355X, D = 128, blocks of 16 rows): 64 single tokens over 512 to 8192 rows, 283 MB, the rows' bytes (69 us; 55 at a copy's
// rate); four sequences of 16384 rows with 64 heads, 129 GFLOP, vector instructions (72% of the SIMDs' cycles) beside the matrix pipe (51%): 119 us,
// 1.09 PFLOP/s; 16 ragged trees over 512 to 8192 rows 66 us, a third of it the ends of pieces and the second launch; one tree over 2048 rows 12.0
// us, 240 workgroups of five rounds that join in pairs; one token over 256 rows 6.1 us, a launch.
#include <algorithm>
#include <atomic>
#include <cmath>

#include "radar_host.h"
#include "radar_kvq_step.h"

namespace radar {

struct KqArgs {
    const __bf16 *q;
    const unsigned char *cache;
    const int32_t *tables, *parents, *ctx_lens, *n_nodes;
    __bf16 *out;
    float *lse;
    int B, T, Hq, Hkv, G, M, S, rbits, n_blocks;
    int64_t q_sb, q_st, q_sh, o_sb, o_st, o_sh;
    float scale_log2;
    int64_t block_bytes;                       // of a block, all heads
    int workgroups, least, shift, max_cgs;     // least share of the line; log2 steps per unit of it; column blocks of a KV head
    int unit_cost, whole;                      // what a unit costs besides its steps; whole: no line, 2^(whole - 1) workgroups for each unit
    float *part;                               // [2 * workgroups] partial results: outputs, maxima (log2 units), sums, in fp32
    uint32_t *unit_tab;                        // first and last workgroup of a unit; where they are the same it is written already
    unsigned int *arrived;                     // of a unit's workgroups, kKqArrived words apart
};

// A sequence: rows of its prefix, nodes of its tree, rows that may be attended to.  There is none: nn = 0.
struct KqSeq { int L, nn, total; };
__device__ __forceinline__ KqSeq kq_seq(const KqArgs &a, int b) {
    KqSeq s;
    s.L = min(a.ctx_lens[b], a.S);                                   // (so that the tree's rows can be added in 32 bits)
    s.nn = a.n_nodes ? max(1, min(a.n_nodes[b], a.T)) : a.T;
    if (s.L < 0) s.nn = 0;
    s.total = s.L < 0 ? 0 : min(s.L + s.nn, a.S);
    return s;
}

// Ancestor word of tree row `lane` (bit a set <=> a is the row or an ancestor of it), by doubling; a parent counts only if it is an
// earlier row.  All lanes call.
__device__ __forceinline__ uint64_t kq_ancestors(const int32_t *parents, int nn) {
    const int lane = lane_id();
    int p = parents ? parents[min(lane, max(nn, 1) - 1)] : lane - 1;
    uint32_t lo = lane < 32 ? 1u << lane : 0u, hi = lane < 32 ? 0u : 1u << (lane - 32);
    p = (lane < nn && p < lane) ? p : -1;
    while (__ballot(p >= 0) != 0ull) {
        const int src = max(p, 0);
        const uint32_t l2 = (uint32_t)__shfl((int)lo, src), h2 = (uint32_t)__shfl((int)hi, src);
        const int p2 = __shfl(p, src);
        if (p >= 0) { lo |= l2; hi |= h2; p = p2; }
    }
    return (uint64_t)hi << 32 | lo;
}

// Four outputs of a row, from their weighted sum, the reference and the weights' sum; with the first four the row's log-sum-exp.
__device__ __forceinline__ void kq_write(const KqArgs &a, int b, int i, int h, int d, floatx4 acc, float M, float l) {
    const float inv = l == 0.f ? 0.f : 1.0f / l;                     // (no key seen)
    bf16x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (__bf16)(acc[e] * inv);
    *reinterpret_cast<bf16x4 *>(a.out + (size_t)b * a.o_sb + (size_t)i * a.o_st + (size_t)h * a.o_sh + d) = o;
    if (a.lse && d == 0) a.lse[((size_t)b * a.T + i) * a.Hq + h] = l == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(l)) * kqLn2;
}

// Which of the step's 32 keys a column sees.  first: the step's first key, counted from the tree's first row.
__device__ __forceinline__ uint32_t kq_allowed(uint64_t anc, int first) {
    if (first >= 64) return 0;
    if (first >= 0) return (uint32_t)(anc >> first);
    if (first <= -32) return ~0u;
    return (uint32_t)(anc << -first) | ((1u << -first) - 1);
}
// ===================================================================== one workgroup
// A workgroup takes one KV head's rows, or a range of them, for 16 * NC query columns; its eight wavefronts take the steps of 32 keys in turn and
// meet in LDS at the end.  Nobody waits for anybody before that: there is no tile to share.  What a wavefront spends on turning codes into
// operands (about 115 vector instructions a step) is shared by its columns only, hence as many as registers allow: with 64 columns the outputs
// take 128 registers, and the queries' operands stay in LDS.
constexpr int kKqWaves = 8, kKqThreads = kKqWaves * kWave;
constexpr int kKqArrived = 16;                 // counters are 64 bytes apart: atomics on one line wait for each other
constexpr int kKqJoined = 256;                 // most workgroups of units that several take
constexpr int kq_line_workgroups(int nc) { return nc == 1 ? 512 : 256; }       // what the chip holds at once
template <int D, int NC>
struct KqShape {
    static constexpr int NM = D / 16, CH = D / 32, COLS = 16 * NC;   // output tiles; steps of the scores' product; columns
    static constexpr int PASSES = NC * D > 256 ? 2 : 1;              // the merge goes over the outputs in so many passes (its buffer is 139 KB at most)
    static constexpr int EP = 4 / PASSES, DP = D / PASSES;           // registers, values of a pass
    static constexpr int ROW = DP + 4;                               // of the merge's buffer: rows 16 bytes apart from a multiple of the banks
    static constexpr int q_bytes() { return COLS * D * 2; }
    static constexpr int merge_bytes() { return kKqWaves * COLS * ROW * 4; }
    static constexpr int lds_bytes() { return merge_bytes() + (kKqWaves + 2) * COLS * 8 + kKqWaves * 64 + q_bytes(); }
    static constexpr int PART = COLS * D + 2 * COLS;                 // floats of a partial result: outputs, maxima and sums in pairs
};

// --------------------------------------------------------------------- dealing the rows out
// The batch's work is one line: sequence by sequence, KV head by KV head, block of columns by block of columns (a unit), each as long as its
// steps and a constant for what a unit costs besides.  Workgroup w takes the w-th of equal shares of the line, wherever the cuts
// fall, one piece after the other.  A unit that one workgroup has all of is written at once; otherwise every piece of it leaves a
// partial result: in the workgroup's second place if the unit goes on behind its share, else in its first.  Whatever the lengths, all
// workgroups end together.  Workgroups go to the eight XCDs in turn, so their numbers are dealt such that an XCD takes a stretch of the
// line: the column blocks of a KV head then find its rows in one L2.

struct KqChunkPlan {                           // lane = sequence b0 + lane; the same in every wavefront
    int b0;
    uint32_t base, end;                        // the chunk's stretch of the line
    int L, nn, total, cgs;
    uint32_t len, start;                       // of a unit; where the sequence begins on the line
};

// The share that a workgroup takes, of n; n: it takes none.  An XCD takes shares that follow each other, every XCD as many.
__device__ __forceinline__ uint32_t kq_share_of(uint32_t n) {
    const uint32_t each = (n + 7) >> 3, i = blockIdx.x >> 3;
    return i < each ? min((blockIdx.x & 7) * each + i, n) : n;
}

template <int NC>
__device__ __forceinline__ void kq_plan_chunk(KqChunkPlan &c, const KqArgs &a, int b0, uint32_t base) {
    const int lane = lane_id(), b = min(b0 + lane, a.B - 1);
    const KqSeq s = kq_seq(a, b);
    c.b0 = b0; c.base = base;
    c.L = s.L; c.nn = s.nn; c.total = s.total;
    c.cgs = (s.nn * a.G + 16 * NC - 1) / (16 * NC);
    const int steps = (s.total + 31) >> 5;
    c.len = (uint32_t)((steps + (1 << a.shift) - 1) >> a.shift) + (uint32_t)a.unit_cost;
    const uint32_t mine = b0 + lane < a.B && s.nn > 0 ? c.len * (uint32_t)(a.Hkv * c.cgs) : 0u;
    if (mine == 0) c.len = 0;
    const uint32_t incl = wave_scan_u32(mine);
    c.start = base + incl - mine;
    c.end = base + readlane_u32(incl, kWave - 1);
}

// A workgroup's place on the line and its piece, which wait in LDS (every wavefront has its own copy) while the loop needs the scalar registers.
struct KqPlace { uint32_t pos, end, share; int b0; uint32_t base, number; };       // number: of its share
struct KqPiece { int b, hk, cg, nn, slot, L, total, s0, s1, parts; };        // slot: of its partial result, -1: it is all of its unit
constexpr int kKqState = 16;                   // words of a wavefront's copy: the place, then the piece
template <typename T>
__device__ __forceinline__ T kq_recall(const int *from) {            // the same in every lane
    constexpr int N = sizeof(T) / 4;
    int v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __builtin_amdgcn_readfirstlane(from[i]);
    return __builtin_bit_cast(T, v);
}
template <typename T>
__device__ __forceinline__ void kq_remember(int *to, T x) {
    constexpr int N = sizeof(T) / 4;
    int v[N];
    __builtin_memcpy(v, &x, sizeof(T));
#pragma unroll
    for (int i = 0; i < N; ++i) to[i] = v[i];
}

// The arguments, read where a phase of the kernel needs them: all of them at once are more than the scalar registers hold beside its state.
__device__ __forceinline__ KqArgs kq_args_plan() {
    const ArgBlock<KqArgs> g = args_from_here<KqArgs>(0);
    KqArgs a;
    a.ctx_lens = g->ctx_lens; a.n_nodes = g->n_nodes; a.B = g->B; a.T = g->T; a.Hkv = g->Hkv; a.G = g->G; a.S = g->S;
    a.workgroups = g->workgroups; a.least = g->least; a.shift = g->shift; a.max_cgs = g->max_cgs; a.unit_tab = g->unit_tab;
    a.unit_cost = g->unit_cost; a.whole = g->whole;
    return a;
}
__device__ __forceinline__ KqArgs kq_args_loop() {
    const ArgBlock<KqArgs> g = args_from_here<KqArgs>(0);
    KqArgs a;
    a.tables = g->tables; a.cache = g->cache; a.M = g->M; a.rbits = g->rbits; a.n_blocks = g->n_blocks; a.block_bytes = g->block_bytes;
    a.scale_log2 = g->scale_log2;
    return a;
}
__device__ __forceinline__ KqArgs kq_args_query() {
    const ArgBlock<KqArgs> g = args_from_here<KqArgs>(0);
    KqArgs a;
    a.q = g->q; a.q_sb = g->q_sb; a.q_st = g->q_st; a.q_sh = g->q_sh; a.G = g->G; a.T = g->T; a.parents = g->parents;
    return a;
}
__device__ __forceinline__ KqArgs kq_args_end() {
    const ArgBlock<KqArgs> g = args_from_here<KqArgs>(0);
    KqArgs a;
    a.out = g->out; a.o_sb = g->o_sb; a.o_st = g->o_st; a.o_sh = g->o_sh; a.lse = g->lse; a.G = g->G; a.T = g->T; a.Hq = g->Hq; a.part = g->part;
    a.ctx_lens = g->ctx_lens; a.n_nodes = g->n_nodes; a.S = g->S; a.B = g->B; a.workgroups = g->workgroups;
    a.whole = g->whole; a.arrived = g->arrived; a.scale_log2 = g->scale_log2;
    return a;
}

template <int D, int NC, bool FAR>
__global__ __launch_bounds__(kKqThreads, NC == 1 ? 4 : 2) void kvq_attn_kernel(KqArgs) {
    using S = KqShape<D, NC>;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    float *const s_o = reinterpret_cast<float *>(smem);                               // [wavefront][column][ROW]
    float *const s_m = reinterpret_cast<float *>(smem + S::merge_bytes()), *const s_l = s_m + kKqWaves * S::COLS;
    float *const s_M = s_l + kKqWaves * S::COLS, *const s_L = s_M + S::COLS;          // of all wavefronts
    uint64_t *const s_anc = reinterpret_cast<uint64_t *>(s_L + S::COLS);              // the columns' ancestors
    int *const s_state = reinterpret_cast<int *>(s_anc + S::COLS);
    u32x4 *const s_q = reinterpret_cast<u32x4 *>(s_state + kKqWaves * kKqState);      // [column block][chunk][lane], the lanes' operands
    const int lane = lane_id(), w = __builtin_amdgcn_readfirstlane(wave_id()), r = lane & 15, grp = lane >> 4;
    int *const state = s_state + w * kKqState;

    // A workgroup, or as many as `parts`, for each unit: nothing to work out but which, and the only sequence's lengths.
    auto whole_piece = [&]() -> bool {
        const KqArgs a = kq_args_plan();
        const int bits = a.whole - 1;
        const uint32_t n = (uint32_t)(a.B * a.Hkv * a.max_cgs) << bits, u = kq_share_of(n), unit = u >> bits;
        if (u >= n) return false;
        KqPiece p;
        const uint32_t bh = unit / (uint32_t)a.max_cgs;
        p.cg = (int)__builtin_amdgcn_readfirstlane(unit - bh * (uint32_t)a.max_cgs);
        p.b = (int)__builtin_amdgcn_readfirstlane(bh / (uint32_t)a.Hkv);
        p.hk = (int)__builtin_amdgcn_readfirstlane(bh) - p.b * a.Hkv;
        p.L = min(uniform_word(a.ctx_lens, p.b), a.S);               // (kq_seq)
        p.nn = a.n_nodes ? max(1, min(uniform_word(a.n_nodes, p.b), a.T)) : a.T;
        if (p.L < 0) p.nn = 0;
        p.total = p.L < 0 ? 0 : min(p.L + p.nn, a.S);
        const int steps = p.cg * S::COLS < p.nn * a.G ? (p.total + 31) >> 5 : 0, per = (steps + (1 << bits) - 1) >> bits;
        p.s0 = (int)(u & ((1u << bits) - 1)) * max(per, 1);
        p.s1 = min(p.s0 + per, steps);
        if (p.s0 > 0 && p.s0 >= steps) return false;                 // (a unit without steps has its first workgroup, for the zeros)
        p.parts = per > 0 ? (int)__builtin_amdgcn_readfirstlane((uint32_t)(steps + per - 1) / (uint32_t)per) : 1;
        p.slot = p.parts > 1 ? (int)u : -1;
        kq_remember(state + sizeof(KqPlace) / 4, p);
        return true;
    };
    // the line's length, and this workgroup's share of it
    auto plan = [&] {
        const KqArgs a = kq_args_plan();
        KqChunkPlan c;
        uint32_t line = 0;
        for (int b0 = 0; b0 < a.B; b0 += kWave) {
            kq_plan_chunk<NC>(c, a, b0, line);
            line = c.end;
        }
        const uint32_t share = max((line + a.workgroups - 1) / a.workgroups, (uint32_t)a.least);
        const uint32_t pos = min((uint64_t)kq_share_of((line + share - 1) / share) * share, (uint64_t)line);
        kq_remember(state, KqPlace{pos, (uint32_t)min((uint64_t)pos + share, (uint64_t)line), share, 0, 0, pos / share});
    };
    auto next_piece = [&]() -> bool {                                // all values the same in every lane
        KqPlace x = kq_recall<KqPlace>(state);
        if (x.pos >= x.end) return false;
        const KqArgs a = kq_args_plan();
        const uint32_t cost = (uint32_t)a.unit_cost;
        KqChunkPlan c;
        kq_plan_chunk<NC>(c, a, x.b0, x.base);
        while (x.pos < x.end) {
            while (x.pos >= c.end) kq_plan_chunk<NC>(c, a, c.b0 + kWave, c.end);
            const uint64_t before = __ballot(c.len > 0 && c.start <= x.pos);
            const int q = 63 - __clzll((long long)before);
            const uint32_t len = readlane_u32(c.len, q), first = readlane_u32(c.start, q);
            const uint32_t u = __builtin_amdgcn_readfirstlane((x.pos - first) / len), at = first + u * len;  // (a quotient comes out of vector registers)
            const uint32_t from = x.pos - at, to = min(x.end - at, len);
            x.pos = at + to;
            if (to <= cost) continue;                                // (of the unit's own cost nobody has anything to do)
            const int cgs = (int)readlane_u32((uint32_t)c.cgs, q);
            KqPiece p;
            p.b = c.b0 + q;
            p.hk = __builtin_amdgcn_readfirstlane((int)u / cgs);
            p.cg = (int)u - p.hk * cgs;
            p.L = (int)readlane_u32((uint32_t)c.L, q);
            p.nn = (int)readlane_u32((uint32_t)c.nn, q);
            p.total = (int)readlane_u32((uint32_t)c.total, q);
            const int steps = (p.total + 31) >> 5;
            p.s0 = min((int)(from > cost ? (from - cost) << a.shift : 0u), steps);
            p.s1 = min((int)((to - cost) << a.shift), steps);
            p.parts = 1;
            p.slot = from <= cost && to == len ? -1 : 2 * (int)x.number + (to < len ? 1 : 0);
            if (from <= cost && threadIdx.x == 0)       // for the merge: first and last workgroup
                a.unit_tab[(p.b * a.Hkv + p.hk) * a.max_cgs + p.cg] = p.slot < 0 ? 0u : x.number << 16 | ((at + len - 1) / x.share);
            x.b0 = c.b0; x.base = c.base;
            kq_remember(state, x);
            kq_remember(state + sizeof(KqPlace) / 4, p);
            return true;
        }
        return false;
    };

    const bool whole = args_from_here<KqArgs>(0)->whole != 0;
    if (!whole) plan();
    for (bool more = true; more; more = !whole) {
        if (!(whole ? whole_piece() : next_piece())) break;
        KqPiece p = kq_recall<KqPiece>(state + sizeof(KqPlace) / 4);
        KqArgs a = kq_args_loop();
        // (the same in every lane, which the compiler does not see behind the search for the piece)
        const int32_t *const table = (const int32_t *)(uintptr_t)kq_scalar(a.tables + (size_t)p.b * a.M);
        const kq_bytes base = (kq_bytes)(uintptr_t)kq_scalar(a.cache + (size_t)p.hk * KvqChunk<D>::bytes(1 << a.rbits));
        const int mine = p.s0 + w;
        const bool active = mine < p.s1;
        // the first step's loads, before the queries (two steps ahead took as long or longer: 64 single tokens 71 us, 69 with one)
        KqK<D> k;
        KqV v;
        KqIds id{0, 0}, nid{0, 0};
        if (active) {
            id = kq_ids(a, table, mine * 32, p.total);
            nid = kq_ids(a, table, min(mine + kKqWaves, p.s1 - 1) * 32, p.total);
            const KqBase at = kq_base<D>(a, base, id, mine * 32);
            int lane2 = lane;
            asm volatile("" : "+v"(lane2));                          // (a mask of lanes less to keep)
            kq_load_k<D, FAR>(k, at, lane2);
            kq_load_v<D, FAR>(v, a, at, lane2);
        }
        // this lane's columns: their queries' operands (d = D/4 * grp + 8 * c + 0..7) and ancestors
        const KqArgs aq = kq_args_query();
        auto query = [&](int n, int ch) {
            const KqArgs &a = aq;
            const int col = (p.cg * NC + n) * 16 + r, i = col / a.G;
            u32x4 x = {0, 0, 0, 0};
            if (i < p.nn) x = *reinterpret_cast<const u32x4 *>(a.q + (size_t)p.b * a.q_sb + (size_t)i * a.q_st + (size_t)(p.hk * a.G + col - i * a.G) * a.q_sh + (D / 4) * grp + 8 * ch);
            return x;
        };
        for (int x = w; x < NC * S::CH; x += kKqWaves) s_q[x * kWave + lane] = query(x / S::CH, x % S::CH);
        if (w < NC && p.s1 * 32 > p.L) {
            const uint64_t words = kq_ancestors(aq.parents ? aq.parents + (size_t)p.b * aq.T : nullptr, p.nn);
            const int i = ((p.cg * NC + w) * 16 + r) / aq.G, ii = min(i, RADAR_T_MAX - 1);
            const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)words, ii), hi = (uint32_t)__shfl((int)(uint32_t)(words >> 32), ii);
            if (grp == 0) s_anc[w * 16 + r] = i < p.nn ? (uint64_t)hi << 32 | lo : 0ull;
        }
        if (lane < S::COLS) s_m[w * S::COLS + lane] = -kKqNone;      // the references of this wavefront's columns, as scores
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
        const int last = p.s1 - 1;                                   // (past it, rows that are there are asked for once more, in vain)
        for (int s = mine; s < p.s1; s += kKqWaves) {
            const int next = min(s + kKqWaves, last);
            KqIds nnid;
            kq_step<D, NC, FAR || NC == 1 ? 2 : 4>(k, v, id, qop, [&] {
                nnid = kq_ids(a, table, min(s + 2 * kKqWaves, last) * 32, p.total);
                kq_load_k<D, FAR>(k, kq_base<D>(a, base, nid, next * 32), lane);
            }, oacc, negref, l_run, [&](int col, int first) { return kq_allowed(s_anc[col], first); }, s_m, a, s * 32, p.L, p.total);
            kq_load_v<D, FAR>(v, a, kq_base<D>(a, base, nid, next * 32), lane);
            id = nid;
            nid = nnid;
        }
        __builtin_amdgcn_s_setprio(0);
        // the wavefronts' results, added up against their common reference
        a = kq_args_end();
        p = kq_recall<KqPiece>(state + sizeof(KqPlace) / 4);
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));                                // (addresses are worked out here, and not kept from the start)
        const int r = tid & 15, grp = (tid >> 4) & 3;
        // A lane's outputs after the merge: of one column, IPT times four.  (Wavefronts that had no step add zeros.)
        constexpr int Q4 = S::DP / 4, TPC = kKqThreads / S::COLS < Q4 ? kKqThreads / S::COLS : Q4, IPT = Q4 / TPC;      // fours of a pass; lanes of a column
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            const float l = kq_column_sum(l_run[n]);
            float *const m = s_m + w * S::COLS + n * 16 + r;
            if (grp == 0) {                                          // (a far reference in log2 units is good to 2^-24 of itself, as the scores are)
                *m = l == 0.f ? -kKqNone : kq_is_far(negref[n]) ? fminf(fmaxf(*m * a.scale_log2, -kKqNone), kKqNone) : -negref[n];
                s_l[w * S::COLS + n * 16 + r] = l;
            }
        }
        __syncthreads();
        if (tid < S::COLS) {
            float m[kKqWaves], M = -kKqNone, l = 0.f;
#pragma unroll
            for (int x = 0; x < kKqWaves; ++x) m[x] = s_m[x * S::COLS + tid];
#pragma unroll
            for (int x = 0; x < kKqWaves; ++x) M = fmaxf(M, m[x]);
#pragma unroll
            for (int x = 0; x < kKqWaves; ++x) l += s_l[x * S::COLS + tid] * __builtin_amdgcn_exp2f(m[x] - M);
            s_M[tid] = M;
            s_L[tid] = l;
        }
        __syncthreads();
        float scl[NC];
#pragma unroll
        for (int n = 0; n < NC; ++n) scl[n] = __builtin_amdgcn_exp2f(s_m[w * S::COLS + n * 16 + r] - s_M[n * 16 + r]);
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
                        *reinterpret_cast<floatx4 *>(s_o + (w * S::COLS + n * 16 + r) * S::ROW + (grp * S::EP + e) * S::NM + m) = x;
                    }
            __syncthreads();
            int lane2 = threadIdx.x;
            asm volatile("" : "+v"(lane2));
            const int mc = lane2 / TPC, mx = lane2 % TPC * 4, gc = p.cg * S::COLS + mc, mi = gc / a.G, mh = p.hk * a.G + gc - mi * a.G;
            if (whole && mc < S::COLS && mi >= p.nn) {               // rows behind the tree's end: zeros
#pragma unroll
                for (int z = 0; z < IPT; ++z) {
                    const int x = z * TPC * 4 + mx, d = D / 4 * (x / (S::EP * S::NM)) + pass * S::EP * S::NM + x % (S::EP * S::NM);
                    if (mi < a.T && p.s0 == 0) {
                        *reinterpret_cast<u32x2 *>(a.out + (size_t)p.b * a.o_sb + (size_t)mi * a.o_st + (size_t)mh * a.o_sh + d) = u32x2{0, 0};
                        if (a.lse && d == 0) a.lse[((size_t)p.b * a.T + mi) * a.Hq + mh] = 0.f;
                    }
                }
            } else if (mc < S::COLS && (p.slot >= 0 || mi < p.nn)) {
                const float M = s_M[mc], l = s_L[mc];
                floatx4 o[IPT][kKqWaves];
#pragma unroll
                for (int z = 0; z < IPT; ++z)
#pragma unroll
                    for (int y = 0; y < kKqWaves; ++y) o[z][y] = *reinterpret_cast<const floatx4 *>(s_o + (y * S::COLS + mc) * S::ROW + z * TPC * 4 + mx);
#pragma unroll
                for (int z = 0; z < IPT; ++z) {
                    const int x = z * TPC * 4 + mx, d = D / 4 * (x / (S::EP * S::NM)) + pass * S::EP * S::NM + x % (S::EP * S::NM);
                    floatx4 acc = o[z][0];
#pragma unroll
                    for (int y = 1; y < kKqWaves; ++y) acc += o[z][y];
                    float *const to = a.part + (size_t)p.slot * S::PART;
                    if (p.parts > 1) {
                        const float a0 = acc[0], a1 = acc[1], a2 = acc[2], a3 = acc[3];
                        store_shared_result(reinterpret_cast<uint64_t *>(to + mc * D + d), (uint64_t)__float_as_uint(a1) << 32 | __float_as_uint(a0));
                        store_shared_result(reinterpret_cast<uint64_t *>(to + mc * D + d + 2), (uint64_t)__float_as_uint(a3) << 32 | __float_as_uint(a2));
                        if (d == 0) store_shared_result(reinterpret_cast<uint64_t *>(to + S::COLS * D + 2 * mc), (uint64_t)__float_as_uint(l) << 32 | __float_as_uint(M));
                    } else if (p.slot >= 0) {
                        *reinterpret_cast<floatx4 *>(to + mc * D + d) = acc;
                        if (d == 0) { to[S::COLS * D + 2 * mc] = M; to[S::COLS * D + 2 * mc + 1] = l; }
                    } else {
                        kq_write(a, p.b, mi, mh, d, acc, M, l);
                    }
                }
            }
        }
        __syncthreads();
        if (p.parts > 1) {
            // The unit's workgroup that arrives last has all the parts, its own among them, join.
            const int bits = a.whole - 1, unit = p.slot >> bits;
            unsigned int *const counter = a.arrived + unit * kKqArrived;
            if ((int)publish_then_ticket(counter, reinterpret_cast<unsigned int *>(s_m)) != p.parts - 1) return;
            if (threadIdx.x == 0) store_shared_result(counter, 0u);
            const float *const from = a.part + (size_t)(unit << bits) * S::PART;
            int first = threadIdx.x;
            asm volatile("" : "+v"(first));                          // (what comes of it is worked out here, and not kept from the start)
            for (int x = first; x < S::COLS * D / 4; x += kKqThreads) {
                const int mc = x / (D / 4), d = x % (D / 4) * 4, gc = p.cg * S::COLS + mc, mi = gc / a.G, mh = p.hk * a.G + gc - mi * a.G;
                if (mi >= p.nn) continue;
                float M = -kKqNone, l = 0.f;
                floatx4 acc = {0.f, 0.f, 0.f, 0.f};
                constexpr int U = 4;
                for (int y0 = 0; y0 < p.parts; y0 += U) {
                    uint64_t ml[U], lo[U], hi[U];
#pragma unroll
                    for (int y = 0; y < U; ++y) {
                        const float *const part = from + (size_t)min(y0 + y, p.parts - 1) * S::PART;
                        ml[y] = load_shared_result(reinterpret_cast<const uint64_t *>(part + S::COLS * D + 2 * mc));
                        lo[y] = load_shared_result(reinterpret_cast<const uint64_t *>(part + mc * D + d));
                        hi[y] = load_shared_result(reinterpret_cast<const uint64_t *>(part + mc * D + d + 2));
                    }
                    float Mn = M;
#pragma unroll
                    for (int y = 0; y < U; ++y) Mn = fmaxf(Mn, __uint_as_float((uint32_t)ml[y]));
                    const float f0 = __builtin_amdgcn_exp2f(M - Mn);
                    M = Mn;
                    l *= f0;
                    acc *= f0;
#pragma unroll
                    for (int y = 0; y < U; ++y) {
                        if (y0 + y >= p.parts) break;                // (the last part once more)
                        const float f = __builtin_amdgcn_exp2f(__uint_as_float((uint32_t)ml[y]) - Mn);
                        l += __uint_as_float((uint32_t)(ml[y] >> 32)) * f;
                        acc += floatx4{__uint_as_float((uint32_t)lo[y]), __uint_as_float((uint32_t)(lo[y] >> 32)), __uint_as_float((uint32_t)hi[y]),
                                       __uint_as_float((uint32_t)(hi[y] >> 32))} * f;
                    }
                }
                kq_write(a, p.b, mi, mh, d, acc, M, l);
            }
        }
    }

    if (whole) return;
    // rows behind a tree's end, and of sequences that are not there: zeros (a lane looks at one row, the wavefront fills those that are found)
    const KqArgs a = kq_args_end();
    const int rows = a.B * a.T, step = a.workgroups * kKqWaves;
    for (int x0 = (int)blockIdx.x + a.workgroups * w; x0 < rows; x0 += step * kWave) {
        const int x = (int)min((int64_t)x0 + (int64_t)step * lane, (int64_t)rows - 1);
        uint64_t empty = __ballot((int64_t)x0 + (int64_t)step * lane < rows && x % a.T >= kq_seq(a, x / a.T).nn);
        for (; empty != 0; empty &= empty - 1) {
            const int y = x0 + step * (__ffsll((unsigned long long)empty) - 1), b = y / a.T, i = y - b * a.T;
            __bf16 *const row = a.out + (size_t)b * a.o_sb + (size_t)i * a.o_st;
            for (int z = lane; z < a.Hq * (D / 8); z += kWave) *reinterpret_cast<u32x4 *>(row + (size_t)(z / (D / 8)) * a.o_sh + z % (D / 8) * 8) = u32x4{0, 0, 0, 0};
            if (a.lse)
                for (int z = lane; z < a.Hq; z += kWave) a.lse[(size_t)y * a.Hq + z] = 0.f;
        }
    }
}

// The units that several workgroups had parts of.  A lane takes 4 (D = 64) or 8 outputs of a column.  GROUPS = 1: a workgroup has 16 columns, a lane
// goes over the parts.  GROUPS = 16, for units in many parts (a long context of one sequence): a workgroup has 4 columns and a wavefront
// every 16th part, four at a time; they meet in LDS (64 parts of a unit: 4.6 us, 25 by one lane).
template <int D, int NC, int GROUPS>
__global__ __launch_bounds__(GROUPS == 1 ? 256 : 1024) void kvq_merge_kernel(KqArgs a) {
    using S = KqShape<D, NC>;
    constexpr int PER = D / 16, CW = GROUPS == 1 ? 16 : 4, U = GROUPS == 1 ? 1 : 4, Q = PER / 4;
    const int unit = blockIdx.x, b = unit / (a.Hkv * a.max_cgs), hk = unit / a.max_cgs % a.Hkv, cg = unit % a.max_cgs, n = blockIdx.y;
    const KqSeq s = kq_seq(a, b);
    if ((cg * S::COLS + n * CW) >= s.nn * a.G) return;
    const uint32_t tab = a.unit_tab[unit];
    const int w0 = tab >> 16, w1 = tab & 0xffff;
    if (w0 == w1) return;
    const int group = GROUPS == 1 ? 0 : __builtin_amdgcn_readfirstlane(wave_id()), mine = GROUPS == 1 ? threadIdx.x / 16 : lane_id() / 16;
    const int col = n * CW + mine, d = threadIdx.x % 16 * PER;
    float M = -kKqNone, l = 0.f;
    floatx4 acc[Q];
#pragma unroll
    for (int x = 0; x < Q; ++x) acc[x] = floatx4{0.f, 0.f, 0.f, 0.f};
    auto add = [&](const float (&m)[U], const float (&ls)[U], const floatx4 (&o)[U][Q]) {
        float Mn = M;
#pragma unroll
        for (int u = 0; u < U; ++u) Mn = fmaxf(Mn, m[u]);
        const float f0 = __builtin_amdgcn_exp2f(M - Mn);
        M = Mn;
        l *= f0;
#pragma unroll
        for (int x = 0; x < Q; ++x) acc[x] *= f0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float f = __builtin_amdgcn_exp2f(m[u] - Mn);
            l += ls[u] * f;
#pragma unroll
            for (int x = 0; x < Q; ++x) acc[x] += o[u][x] * f;
        }
    };
    for (int w = w0 + group; w <= w1; w += U * GROUPS) {
        float m[U], ls[U];
        floatx4 o[U][Q];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool there = w + u * GROUPS <= w1;                 // (the same in every lane; otherwise the last part once more, as nothing)
            const int part = min(w + u * GROUPS, w1);
            const float *const from = a.part + (size_t)(2 * part + (part < w1 ? 1 : 0)) * S::PART;
            m[u] = there ? from[S::COLS * D + 2 * col] : -kKqNone;
            ls[u] = there ? from[S::COLS * D + 2 * col + 1] : 0.f;
#pragma unroll
            for (int x = 0; x < Q; ++x) o[u][x] = there ? *reinterpret_cast<const floatx4 *>(from + (size_t)col * D + d + 4 * x) : floatx4{0.f, 0.f, 0.f, 0.f};
        }
        add(m, ls, o);
    }
    if constexpr (GROUPS > 1) {
        __shared__ float s_m[GROUPS][CW], s_l[GROUPS][CW];
        __shared__ __attribute__((aligned(16))) float s_o[GROUPS][CW][D];
        if (d == 0) { s_m[group][mine] = M; s_l[group][mine] = l; }
#pragma unroll
        for (int x = 0; x < Q; ++x) *reinterpret_cast<floatx4 *>(&s_o[group][mine][d + 4 * x]) = acc[x];
        __syncthreads();
        if (group != 0) return;
        for (int g = 1; g < GROUPS; g += U) {                        // (the last of the 15 is counted once: beyond it nothing)
            float m[U], ls[U];
            floatx4 o[U][Q];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool there = g + u < GROUPS;
                const int y = min(g + u, GROUPS - 1);
                m[u] = there ? s_m[y][mine] : -kKqNone;
                ls[u] = there ? s_l[y][mine] : 0.f;
#pragma unroll
                for (int x = 0; x < Q; ++x) o[u][x] = there ? *reinterpret_cast<const floatx4 *>(&s_o[y][mine][d + 4 * x]) : floatx4{0.f, 0.f, 0.f, 0.f};
            }
            add(m, ls, o);
        }
    }
    const int gc = cg * S::COLS + col, i = gc / a.G, h = hk * a.G + gc - i * a.G;
    if (i >= s.nn) return;
#pragma unroll
    for (int x = 0; x < Q; ++x) kq_write(a, b, i, h, d + 4 * x, acc[x], M, l);
}

}  // namespace radar

using namespace radar;

static radar_status check_kvq_attn(const radar_kvq_attn_desc *d) {
    if (!d) return RADAR_INVALID_ARG;
    const radar_status st = kvq_check(&d->cache);
    if (st != RADAR_OK) return st;
    if (d->B < 1 || d->T_max < 1 || d->Hq < 1 || d->max_blocks < 1 || d->S_max < 1 || d->Hq % d->cache.Hkv != 0) return RADAR_INVALID_ARG;
    if ((d->S_max - 1) / d->cache.block_rows >= d->max_blocks) return RADAR_INVALID_ARG;
    if (d->rows_per_split < 0 || d->rows_per_split % 64 != 0) return RADAR_INVALID_ARG;
    if (!(d->softmax_scale >= 0.f)) return RADAR_INVALID_ARG;
    if (d->T_max > RADAR_T_MAX || d->B > 65535 || d->Hq > 65535 || d->S_max > INT32_MAX - 4096) return RADAR_UNSUPPORTED_SHAPE;
    // a launch has less than 2^32 lanes, a unit of 16 columns up to 512 of them
    if ((int64_t)d->B * d->cache.Hkv * ((d->Hq / d->cache.Hkv * d->T_max + 15) / 16) > (1 << 23) - 8) return RADAR_UNSUPPORTED_SHAPE;
    return RADAR_OK;
}

struct KqPlan {
    int nc, max_cgs, workgroups, least, shift, unit_cost;
    int whole;                                             // as in KqArgs: no line, no second launch
    size_t off_arrived, off_tab, off_part, bytes;
};

static KqPlan plan_kvq(const radar_kvq_attn_desc *d) {
    KqPlan p;
    const int cols = d->Hq / d->cache.Hkv * d->T_max, D = d->cache.D;
    const int64_t steps = ((int64_t)d->S_max + 31) / 32;
    // Columns a workgroup, and how units are given out: whole; to 2, 4, ... 64 workgroups each, the last of which joins their parts; or all of them in a
    // line, in equal shares.  Whichever takes least, from what rounds of steps and the rest took (us, one MI355X, D = 128, beside the 6 of any call;
    // D = 64 goes by the same figures, which were not measured there).
    // The line costs 13 more (9 with few units), a second launch and two pieces a workgroup, and pays where units differ or are more than the joined
    // ones may be (the host knows the longest only; half of it is taken for the others).  us with 16 / 32 / 64 columns, "-" where there are too many units to join:
    //                                         whole       joined, by 2 ... 32                   line
    //   1 token, 32 heads on 8, 2048 rows       13          10.8  9.3  8.9 10.2 11.4              12.5
    //   16000 rows                              60          34  21  15.5  13.3  15.5              17
    //   128000 rows                                         by 32 34                              33
    //   60 tree rows, 2048 rows                 14 17 24    12.5 15.9 22.9, by 4 - 14.0 20.2      21 21 25
    //   12000 rows                              50 57 84    32 37 53, by 4 - 26 36, by 8 - - 31   38 33 34
    //   4 sequences of 2000 rows                23 18 26    - - 25                                33 22 32
    //   4 of 9000                               69 54 69    - - 51                                78 55 56
    //   16 of 250 .. 2048                       70 63 49    - - -                                 62 57 55
    //   16 of 500 .. 5000                                   - - -                                 99 82 74
    p.whole = 0;
    double best = 1e300;
    const double rounds = (double)((steps + 7) / 8);
    for (int x = 0; x < 3; ++x) {
        const int nc = 1 << x;
        if (nc > 1 && cols <= 8 * nc) continue;
        const double units = (double)d->B * d->cache.Hkv * ((cols + 16 * nc - 1) / (16 * nc));
        const double alone[] = {0.91, 1.05, 1.7}, shared[] = {0.8, 1.27, 2.2}, end[] = {0.0, 2.3, 4.0}, divided[] = {13.2, 12.7, 16.0};
        const double few[] = {0.83, 1.0, 1.65}, many[] = {0.95, 1.27, 2.05}, join[] = {0.2, 0.35, 0.5};        // (many: more workgroups than half the CUs)
        auto take = [&](double us, int whole) { if (us < best) { best = us; p.nc = nc; p.whole = whole; } };
        take((units <= 32 ? 9.0 : divided[x]) + units / 256.0 * ((d->B > 1 ? 0.5 : 1.0) * rounds * shared[x] + 3.0 + end[x]), 0);
        if (d->rows_per_split != 0) continue;
        take(std::ceil(units / 256.0) * (rounds * alone[x] + end[x]), 1);
        for (int bits = 1; bits <= 6 && units * (1 << bits) <= kKqJoined; ++bits)
            take((d->B > 1 ? 0.88 : 1.0) * (std::ceil(rounds / (1 << bits)) * (units * (1 << bits) > 128 ? many[x] : few[x]) + end[x] + 1.4 + join[x] * (1 << bits)), 1 + bits);
    }
    p.max_cgs = (cols + 16 * p.nc - 1) / (16 * p.nc);
    const int64_t units = (int64_t)d->B * d->cache.Hkv * p.max_cgs;
    const int64_t parts = p.whole ? units << (p.whole - 1) : 0;
    p.workgroups = p.whole ? (int)((parts + 7) / 8 * 8) : kq_line_workgroups(p.nc);
    p.least = d->rows_per_split ? d->rows_per_split / 32 : 8;
    // what a unit costs besides its steps, in steps of a wavefront of eight: the merge in LDS, the way in and out (64 single tokens with 0 / 16 / 24 / 48:
    // 86 72 70 73 us; 16 ragged trees by 64 columns with 0 / 24 / 48 / 96: 109 80 71 74; by 32 with 16 / 48 / 96: 94 80 88)
    p.unit_cost = p.nc == 1 ? 24 : p.nc == 2 ? 48 : 56;
    // positions on the line stay within 31 bits
    p.shift = 0;
    while (units * ((steps >> p.shift) + 1 + p.unit_cost) >= (int64_t(1) << 31) && p.shift < 31) ++p.shift;
    // The workspace has room for any plan of these heads with as many sequences and nodes or fewer, since a program that has one for its largest
    // shape makes calls of all smaller ones, and these may be given out in another way and need more: units of 16 columns in the table, and as many
    // columns of partial results as a line leaves, two pieces a workgroup (joined units leave less).
    static_assert(kKqJoined <= 2 * kq_line_workgroups(4));
    const int widest = cols > 32 ? 4 : cols > 16 ? 2 : 1;
    const size_t units16 = (size_t)d->B * d->cache.Hkv * ((cols + 15) / 16), left = std::max(2 * kq_line_workgroups(1), 2 * kq_line_workgroups(widest) * widest) * 16;
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off += (bytes + 255) & ~size_t(255); return o; };
    p.off_arrived = take(kKqJoined * kKqArrived * sizeof(unsigned int));      // first, whatever the shape: all calls leave them at zero
    p.off_tab = take(units16 * sizeof(uint32_t));
    p.off_part = take(left * (D + 2) * sizeof(float));
    p.bytes = off;
    return p;
}

extern "C" size_t radar_tree_attention_kvq_workspace_bytes(const radar_kvq_attn_desc *d) {
    if (check_kvq_attn(d) != RADAR_OK) return 0;
    return plan_kvq(d).bytes;
}

template <int D, int NC, bool FAR>
static hipError_t launch_kvq(const KqArgs &a, const KqPlan &p, hipStream_t s) {
    constexpr int bytes = KqShape<D, NC>::lds_bytes();
    static std::atomic<uint64_t> configured{0};            // devices on which the kernel may have so much LDS (two threads may both say so)
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    const uint64_t bit = 1ull << (device & 63);
    if (device > 63 || !(configured.load(std::memory_order_relaxed) & bit)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void *>(&kvq_attn_kernel<D, NC, FAR>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
        configured.fetch_or(bit, std::memory_order_relaxed);
    }
    e = launch("kvq_attention", kvq_attn_kernel<D, NC, FAR>, dim3((unsigned)p.workgroups), dim3(kKqThreads), bytes, s, a);
    if (e != hipSuccess) return e;
    if (p.whole) return e;
    const unsigned units = (unsigned)(a.B * a.Hkv * a.max_cgs);
    // units in more than four parts or so
    if (4 * units <= (unsigned)p.workgroups) return launch("kvq_merge", kvq_merge_kernel<D, NC, 16>, dim3(units, 4 * NC), dim3(1024), 0, s, a);
    return launch("kvq_merge", kvq_merge_kernel<D, NC, 1>, dim3(units, NC), dim3(256), 0, s, a);
}

extern "C" radar_status radar_tree_attention_kvq(const void *q, const void *cache, const int32_t *block_tables, const int32_t *parents,
                                                 const int32_t *ctx_lens, const int32_t *n_nodes, void *out, float *lse_out,
                                                 const radar_kvq_attn_desc *d, void *workspace, size_t workspace_bytes, void *stream) {
    if (!q || !cache || !block_tables || !ctx_lens || !out || !workspace) return RADAR_INVALID_ARG;
    const radar_status st = check_kvq_attn(d);
    if (st != RADAR_OK) return st;
    const KqPlan p = plan_kvq(d);
    if (workspace_bytes < p.bytes) return RADAR_WORKSPACE_TOO_SMALL;
    if (((uintptr_t)workspace & 255) != 0) return RADAR_INVALID_ARG;
    KqArgs a;
    a.q = static_cast<const __bf16 *>(q); a.cache = static_cast<const unsigned char *>(cache);
    a.tables = block_tables; a.parents = parents; a.ctx_lens = ctx_lens; a.n_nodes = n_nodes;
    a.out = static_cast<__bf16 *>(out); a.lse = lse_out;
    a.B = d->B; a.T = d->T_max; a.Hq = d->Hq; a.Hkv = d->cache.Hkv; a.G = a.Hq / a.Hkv; a.M = d->max_blocks; a.S = d->S_max;
    a.rbits = kvq_log2(d->cache.block_rows); a.n_blocks = d->cache.n_blocks;
    const int64_t D = d->cache.D;
    a.block_bytes = (int64_t)a.Hkv * d->cache.block_rows * (D + D / 16);
    a.q_sh = d->q_stride_h ? d->q_stride_h : D;
    a.q_st = d->q_stride_t ? d->q_stride_t : D * d->Hq;
    a.q_sb = d->q_stride_b ? d->q_stride_b : D * d->Hq * d->T_max;
    a.o_sh = d->out_stride_h ? d->out_stride_h : D;
    a.o_st = d->out_stride_t ? d->out_stride_t : D * d->Hq;
    a.o_sb = d->out_stride_b ? d->out_stride_b : D * d->Hq * d->T_max;
    const uintptr_t al = (uintptr_t)q | (uintptr_t)cache | (uintptr_t)out;
    const int64_t strides = a.q_sh | a.q_st | a.q_sb | a.o_sh | a.o_st | a.o_sb;
    if ((al & 15) != 0 || (strides & 7) != 0 || strides < 0) return RADAR_INVALID_ARG;
    a.scale_log2 = (d->softmax_scale != 0.f ? d->softmax_scale : 1.0f / sqrtf((float)D)) * kqLog2e;
    a.workgroups = p.workgroups; a.least = p.least; a.shift = p.shift; a.max_cgs = p.max_cgs;
    a.unit_cost = p.unit_cost; a.whole = p.whole;
    char *ws = static_cast<char *>(workspace);
    a.arrived = reinterpret_cast<unsigned int *>(ws + p.off_arrived);
    a.unit_tab = reinterpret_cast<uint32_t *>(ws + p.off_tab);
    a.part = reinterpret_cast<float *>(ws + p.off_part);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool far = (int64_t)a.n_blocks * a.block_bytes > UINT32_MAX;
    auto go = [&](auto near_kernel, auto far_kernel) { return far ? far_kernel(a, p, s) : near_kernel(a, p, s); };
    const hipError_t e = D == 128 ? (p.nc == 1   ? go(launch_kvq<128, 1, false>, launch_kvq<128, 1, true>)
                                     : p.nc == 2 ? go(launch_kvq<128, 2, false>, launch_kvq<128, 2, true>)
                                                 : go(launch_kvq<128, 4, false>, launch_kvq<128, 4, true>))
                                  : (p.nc == 1   ? go(launch_kvq<64, 1, false>, launch_kvq<64, 1, true>)
                                     : p.nc == 2 ? go(launch_kvq<64, 2, false>, launch_kvq<64, 2, true>)
                                                 : go(launch_kvq<64, 4, false>, launch_kvq<64, 4, true>));
    return e == hipSuccess ? RADAR_OK : RADAR_HIP_ERROR;
}
