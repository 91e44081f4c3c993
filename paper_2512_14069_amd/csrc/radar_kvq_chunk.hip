// Attention of chunks of new tokens over the paged 4-bit cache (radar_chunk_attention_kvq), for gfx950.
//
// Transposed as in radar_kvq_attention.hip, with its step of 32 keys (radar_kvq_step.h): a KV head's queries are counted through as columns,
// c = row * G + head of the group, and 64 of them are a wavefront's.  Row i sees keys up to ctx + i, so a column's keys are the first so many and only
// the last steps of a block of columns have anything to mask.
#include <algorithm>
#include <atomic>
#include <cmath>

#include "radar_host.h"
#include "radar_kvq_step.h"
#include "radar_rows.h"

namespace radar {

constexpr int kKcCols = 64;                    // columns of a block
constexpr int kKcTarget = 512;                 // what long contexts are divided into, workgroups
constexpr int kKcPlanned = 512;                // most sequences whose work every workgroup counts through
constexpr int kKcArrived = 16;                 // counters are 64 bytes apart: atomics on one line wait for each other

struct KcArgs : KqCache {
    const __bf16 *q;
    const unsigned char *cache;
    const int32_t *tables, *ctx_lens, *row_starts, *n_new;
    __bf16 *out;
    float *lse;
    int B, T, Hq, Hkv, G, M, S, N;
    int64_t q_sb, q_st, q_sh, o_sb, o_st, o_sh;
    int target, least;                         // workgroups that divided work is dealt to (0: nothing is divided); least steps of one
    float *part;                               // [2 * kKcTarget] partial results: outputs, maxima (log2 units) and sums, in fp32
    unsigned int *arrived;                     // of a block's workgroups, kKcArrived words apart
};

// A sequence: rows of its prefix, new rows, rows that the tensors have for it, keys that its last row sees; the first of its rows.
struct KcSeq { int L, n, rows, total, row0; };
__device__ __forceinline__ KcSeq kc_seq(const KcArgs &a, int b) {
    KcSeq s;
    if (a.row_starts) {
        const int from = min(max(a.row_starts[b], 0), a.N), to = min(max(a.row_starts[b + 1], from), a.N);
        s.rows = min(to - from, a.T);
        s.row0 = from;
        s.n = s.rows;
    } else {
        s.rows = a.T;
        s.row0 = b * a.T;
        s.n = a.n_new ? min(max(a.n_new[b], 0), a.T) : a.T;
    }
    s.L = min(a.ctx_lens[b], a.S);             // (so that the new rows can be added in 32 bits)
    if (s.L < 0) s.n = 0;
    s.total = s.n > 0 ? min(s.L + s.n, a.S) : 0;
    return s;
}

// What a workgroup does: a block of columns of a KV head and the steps [s0, s1) of it, one of `parts` such.
struct KcItem { int b, hk, cg, n, rows, row0, L, limit, s0, s1, parts, slot, unit; };
constexpr int kKcState = 16;

// Every item in one line: sequence by sequence, from the last block of columns, which has the most keys, to the first, part by part and KV head by KV head
// (workgroups go to the eight XCDs in turn: a head's rows then stay in one L2).  A sequence's blocks are divided into parts of `per` steps, which is
// the batch's work over what it is dealt to, so that there are no more items than blocks and that, and no more parts than twice that.
// All lanes call; the result is the same in all of them.
__device__ __forceinline__ bool kc_find(KcItem &x, const KcArgs &a, uint32_t item) {
    const int lane = lane_id();
    auto blocks_of = [&](int rows) { return (int)(((int64_t)rows * a.G + kKcCols - 1) / kKcCols); };
    int per = INT32_MAX, p = 1, cgs;
    uint32_t rel, slots = 0, units = 0;
    KcSeq s;
    if (a.target > 0) {
        double work = 0.0;                     // (whole numbers below 2^53)
        for (int b0 = 0; b0 < a.B; b0 += kWave) {
            const KcSeq t = kc_seq(a, min(b0 + lane, a.B - 1));
            if (b0 + lane < a.B) work += (double)blocks_of(t.rows) * (double)a.Hkv * (double)((t.total + 31) >> 5);
        }
        per = max((int)fmin(ceil(wave_sum_f64(work) / (double)a.target), 1e9), a.least);
        uint32_t first = 0;
        int b0 = 0, hit = -1;
        for (; b0 < a.B; b0 += kWave) {
            s = kc_seq(a, min(b0 + lane, a.B - 1));
            cgs = blocks_of(s.rows);
            p = max((((s.total + 31) >> 5) + per - 1) / per, 1);
            const uint32_t mine = b0 + lane < a.B ? (uint32_t)(a.Hkv * cgs) : 0u, items = mine * (uint32_t)p;
            const uint32_t incl = wave_scan_u32(items), split = wave_scan_u32(p > 1 ? items : 0u), whole = wave_scan_u32(p > 1 ? mine : 0u);
            const uint64_t behind = __ballot(first + incl > item);
            if (behind != 0) {
                hit = __ffsll((unsigned long long)behind) - 1;
                rel = item - (first + readlane_u32(incl, hit) - readlane_u32(items, hit));
                if (rel >= readlane_u32(items, hit)) return false;   // (only where row_starts falls)
                p = (int)readlane_u32((uint32_t)p, hit);
                cgs = (int)readlane_u32((uint32_t)cgs, hit);
                if (p > 1) {
                    slots += readlane_u32(split, hit) - readlane_u32(items, hit);
                    units += readlane_u32(whole, hit) - readlane_u32(mine, hit);
                }
                break;
            }
            first += readlane_u32(incl, kWave - 1);
            slots += readlane_u32(split, kWave - 1);
            units += readlane_u32(whole, kWave - 1);
        }
        if (hit < 0) return false;
        x.b = b0 + hit;
        s.L = (int)readlane_u32((uint32_t)s.L, hit); s.n = (int)readlane_u32((uint32_t)s.n, hit); s.rows = (int)readlane_u32((uint32_t)s.rows, hit);
        s.total = (int)readlane_u32((uint32_t)s.total, hit); s.row0 = (int)readlane_u32((uint32_t)s.row0, hit);
    } else {
        // too many sequences to count through: blocks of columns begin at first row * G / 64 + b, which leaves every sequence room
        const int block = (int)(item / (uint32_t)a.Hkv);
        int off;
        if (a.row_starts) {
            auto begin = [&](int b) { return (int64_t)min(max(a.row_starts[b], 0), a.N) * a.G / kKcCols + b; };
            x.b = max(last_at_most(a.B, block, begin), 0);
            off = (int)begin(x.b);
        } else {
            const int each = blocks_of(a.T);
            x.b = block / each;
            off = x.b * each;
        }
        x.b = __builtin_amdgcn_readfirstlane(x.b);
        if (x.b >= a.B) return false;
        s = kc_seq(a, x.b);
        cgs = blocks_of(s.rows);
        rel = (uint32_t)(block - off) * (uint32_t)a.Hkv + item % (uint32_t)a.Hkv;
        if (block < off || block - off >= cgs) return false;
    }
    const uint32_t turn = rel / (uint32_t)a.Hkv, back = turn / (uint32_t)p;
    x.hk = (int)(rel - turn * (uint32_t)a.Hkv);
    x.cg = cgs - 1 - (int)back;
    const int part = (int)(turn - back * (uint32_t)p);
    x.n = s.n; x.rows = s.rows; x.row0 = s.row0; x.L = s.L;
    const int c0 = x.cg * kKcCols, i0 = c0 / a.G, i1 = min((c0 + kKcCols - 1) / a.G, s.n - 1);
    x.limit = i0 < s.n ? min(s.L + i1 + 1, s.total) : 0;
    const int steps = (x.limit + 31) >> 5;
    int wanted = p > 1 ? max((steps + per - 1) / per, 1) : 1;
    x.unit = (int)units + x.cg * a.Hkv + x.hk;
    // (there is room by the bounds above; row_starts that falls may break them)
    const int64_t slot0 = (int64_t)slots + rel - (int64_t)part * a.Hkv;
    if (slot0 < 0 || slot0 + (int64_t)(wanted - 1) * a.Hkv >= 2 * kKcTarget || (uint32_t)x.unit >= (uint32_t)kKcTarget) wanted = 1;
    const int each = (steps + wanted - 1) / wanted;
    x.parts = steps > 0 ? (steps + each - 1) / each : 1;
    if (part >= x.parts) return false;
    x.s0 = part * each;
    x.s1 = min(x.s0 + each, steps);
    x.slot = (int)(slots + rel);
    return true;
}

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
__device__ __forceinline__ KcArgs kc_args_plan() {
    const ArgBlock<KcArgs> g = args_from_here<KcArgs>(0);
    KcArgs a;
    a.ctx_lens = g->ctx_lens; a.row_starts = g->row_starts; a.n_new = g->n_new; a.B = g->B; a.T = g->T; a.Hkv = g->Hkv; a.G = g->G; a.S = g->S; a.N = g->N;
    a.target = g->target; a.least = g->least;
    return a;
}
__device__ __forceinline__ KcArgs kc_args_loop() {
    const ArgBlock<KcArgs> g = args_from_here<KcArgs>(0);
    KcArgs a;
    a.tables = g->tables; a.cache = g->cache; a.M = g->M; a.rbits = g->rbits; a.n_blocks = g->n_blocks; a.block_bytes = g->block_bytes;
    a.scale_log2 = g->scale_log2; a.G = g->G;
    return a;
}
__device__ __forceinline__ KcArgs kc_args_query() {
    const ArgBlock<KcArgs> g = args_from_here<KcArgs>(0);
    KcArgs a;
    a.q = g->q; a.q_sb = g->q_sb; a.q_st = g->q_st; a.q_sh = g->q_sh; a.G = g->G; a.row_starts = g->row_starts;
    return a;
}
__device__ __forceinline__ KcArgs kc_args_end() {
    const ArgBlock<KcArgs> g = args_from_here<KcArgs>(0);
    KcArgs a;
    a.out = g->out; a.o_sb = g->o_sb; a.o_st = g->o_st; a.o_sh = g->o_sh; a.lse = g->lse; a.G = g->G; a.Hq = g->Hq; a.part = g->part;
    a.row_starts = g->row_starts; a.arrived = g->arrived; a.scale_log2 = g->scale_log2;
    return a;
}

// Where row i, head h of an item's sequence is in out, and its place in lse.
__device__ __forceinline__ __bf16 *kc_out(const KcArgs &a, const KcItem &x, int i, int h) {
    const size_t row = a.row_starts ? (size_t)(x.row0 + i) * a.o_st : (size_t)x.b * a.o_sb + (size_t)i * a.o_st;
    return a.out + row + (size_t)h * a.o_sh;
}
template <int N>
__device__ __forceinline__ void kc_write(const KcArgs &a, const KcItem &x, int i, int h, int d, const float (&acc)[N], float M, float l) {
    const float inv = l == 0.f ? 0.f : 1.0f / l;                     // (no key seen)
    __bf16 o[N] __attribute__((aligned(16)));
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = (__bf16)(acc[e] * inv);
    typedef uint32_t words __attribute__((ext_vector_type(N / 2)));
    words w;
    __builtin_memcpy(&w, o, sizeof(w));
    *reinterpret_cast<words *>(kc_out(a, x, i, h) + d) = w;
    if (a.lse && d == 0) a.lse[(size_t)(x.row0 + i) * a.Hq + h] = l == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(l)) * kqLn2;
}

template <int D, int NC, int KW>
struct KcShape {
    static constexpr int NM = D / 16, CH = D / 32, COLS = 16 * NC;
    static constexpr int PASSES = NC * D > 256 ? 2 : 1, EP = 4 / PASSES, DP = D / PASSES, ROW = DP + 4;       // of the merge in LDS
    static constexpr int room() {                                    // queries' operands, then the merge's buffer
        const int q = COLS * D * 2, merge = KW > 1 ? KW * COLS * ROW * 4 : 0;
        return q > merge ? q : merge;
    }
    static constexpr int PART = COLS * D + 2 * COLS;                 // floats of a partial result
};
template <int D, int KW>
constexpr int kc_lds_bytes() { return KcShape<D, 4, KW>::room() + (KW + 1) * kKcCols * 8 + kKcCols * 4 + KW * kKcState * 4; }

// One item.  KW wavefronts take its steps in turn and meet in LDS at the end.
template <int D, int NC, int KW, bool FAR>
__device__ __forceinline__ void kc_item(unsigned char *smem, const int *state) {
    using S = KcShape<D, NC, KW>;
    constexpr int THREADS = KW * kWave;
    u32x4 *const s_q = reinterpret_cast<u32x4 *>(smem);              // [column block][chunk][lane], the lanes' operands
    float *const s_o = reinterpret_cast<float *>(smem);              // [wavefront][column][ROW]
    float *const s_m = reinterpret_cast<float *>(smem + KcShape<D, 4, KW>::room()), *const s_l = s_m + KW * kKcCols;
    float *const s_M = s_l + KW * kKcCols, *const s_L = s_M + kKcCols;
    int *const s_lim = reinterpret_cast<int *>(s_L + kKcCols);       // keys that a column sees
    const int lane = lane_id(), w = KW > 1 ? __builtin_amdgcn_readfirstlane(wave_id()) : 0, r = lane & 15, grp = lane >> 4;

    KcItem p = kc_recall<KcItem>(state);
    KcArgs a = kc_args_loop();
    const int32_t *const table = (const int32_t *)(uintptr_t)kq_scalar(a.tables + (size_t)p.b * a.M);
    const kq_bytes base = (kq_bytes)(uintptr_t)kq_scalar(a.cache + (size_t)p.hk * KvqChunk<D>::bytes(1 << a.rbits));
    const int mine = p.s0 + w;
    const int hidden = min(p.L + p.cg * kKcCols / a.G + 1, p.limit);           // of the first column
    KqK<D> k;
    KqV v;
    KqIds id{0, 0}, nid{0, 0};
    if (mine < p.s1) {
        id = kq_ids(a, table, mine * 32, p.limit);
        nid = kq_ids(a, table, min(mine + KW, p.s1 - 1) * 32, p.limit);
        const KqBase at = kq_base<D>(a, base, id, mine * 32);
        int lane2 = lane;
        asm volatile("" : "+v"(lane2));
        kq_load_k<D, FAR>(k, at, lane2);
        kq_load_v<D, FAR>(v, a, at, lane2);
    }
    {
        const KcArgs aq = kc_args_query();
        const __bf16 *const q0 = aq.q + (aq.row_starts ? (size_t)p.row0 * aq.q_st : (size_t)p.b * aq.q_sb) + (size_t)(p.hk * aq.G) * aq.q_sh;
        for (int x = w; x < NC * S::CH; x += KW) {
            const int col = p.cg * kKcCols + x / S::CH * 16 + r, i = col / aq.G;
            u32x4 y = {0, 0, 0, 0};
            if (i < p.n) y = *reinterpret_cast<const u32x4 *>(q0 + (size_t)i * aq.q_st + (size_t)(col - i * aq.G) * aq.q_sh + (D / 4) * grp + 8 * (x % S::CH));
            s_q[x * kWave + lane] = y;
        }
        if (w == 0 && lane < S::COLS) {
            const int i = (p.cg * kKcCols + lane) / aq.G;
            s_lim[lane] = i < p.n ? min(p.L + i + 1, p.limit) : 0;
        }
    }
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
        }, oacc, negref, l_run, [&](int col) {
            const int sees = s_lim[col] - s * 32;
            return sees >= 32 ? ~0u : sees <= 0 ? 0u : (1u << sees) - 1;
        }, s_m, a, s * 32, hidden, p.limit);
        kq_load_v<D, FAR>(v, a, kq_base<D>(a, base, nid, next * 32), lane);
        id = nid;
        nid = nnid;
    }
    __builtin_amdgcn_s_setprio(0);

    a = kc_args_end();
    p = kc_recall<KcItem>(state);
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));                                    // (addresses are worked out here, and not kept from the start)
    const int r2 = tid & 15, grp2 = (tid >> 4) & 3;
    const int live = min(p.n * a.G - p.cg * kKcCols, S::COLS);       // columns of the block that there are
    float *const to = a.part + (size_t)p.slot * KcShape<D, 4, KW>::PART;
    auto hand_over = [&](int col, int d, float x0, float x1) {
        store_shared_result(reinterpret_cast<uint64_t *>(to + col * D + d), (uint64_t)__float_as_uint(x1) << 32 | __float_as_uint(x0));
    };
    auto hand_over_sum = [&](int col, float M, float l) {
        store_shared_result(reinterpret_cast<uint64_t *>(to + S::COLS * D + 2 * col), (uint64_t)__float_as_uint(l) << 32 | __float_as_uint(M));
    };
    // a column's reference in log2 units (a far one is good to 2^-24 of itself, as the scores are)
    auto reference = [&](int n, float l) {
        const float m = s_m[w * S::COLS + n * 16 + r2];
        return l == 0.f ? -kKqNone : kq_is_far(negref[n]) ? fminf(fmaxf(m * a.scale_log2, -kKqNone), kKqNone) : -negref[n];
    };
    if constexpr (KW == 1) {
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            const int col = n * 16 + r2, gc = p.cg * kKcCols + col, i = gc / a.G, h = p.hk * a.G + gc - i * a.G;
            const float l = kq_column_sum(l_run[n]), M = reference(n, l);
            if (col >= live) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int d = D / 4 * grp2 + e * S::NM;
                float x[S::NM];
#pragma unroll
                for (int m = 0; m < S::NM; ++m) x[m] = oacc[m][n][e];
                if (p.parts > 1) {
#pragma unroll
                    for (int m = 0; m < S::NM; m += 2) hand_over(col, d + m, x[m], x[m + 1]);
                    if (d == 0) hand_over_sum(col, M, l);
                } else {
                    kc_write(a, p, i, h, d, x, M, l);
                }
            }
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
            const int col = lane2 / TPC, mx = lane2 % TPC * 4, gc = p.cg * kKcCols + col, i = gc / a.G, h = p.hk * a.G + gc - i * a.G;
            if (col < live) {
                const float M = s_M[col], l = s_L[col];
#pragma unroll
                for (int z = 0; z < IPT; ++z) {
                    const int x = z * TPC * 4 + mx, d = D / 4 * (x / (S::EP * S::NM)) + pass * S::EP * S::NM + x % (S::EP * S::NM);
                    floatx4 acc = *reinterpret_cast<const floatx4 *>(s_o + col * S::ROW + x);
#pragma unroll
                    for (int y = 1; y < KW; ++y) acc += *reinterpret_cast<const floatx4 *>(s_o + (y * S::COLS + col) * S::ROW + x);
                    if (p.parts > 1) {
                        hand_over(col, d, acc[0], acc[1]);
                        hand_over(col, d + 2, acc[2], acc[3]);
                        if (d == 0) hand_over_sum(col, M, l);
                    } else {
                        const float o[4] = {acc[0], acc[1], acc[2], acc[3]};
                        kc_write(a, p, i, h, d, o, M, l);
                    }
                }
            }
        }
    }
    if (p.parts == 1) return;
    // The block's workgroup that arrives last has all the parts, its own among them, join.  (A part's slots lie Hkv items apart, as the items do.)
    __syncthreads();
    unsigned int *const counter = a.arrived + p.unit * kKcArrived;
    if ((int)publish_then_ticket(counter, reinterpret_cast<unsigned int *>(s_m)) != p.parts - 1) return;
    if (threadIdx.x == 0) store_shared_result(counter, 0u);
    const KcArgs b = kc_args_plan();
    const int each = (((p.limit + 31) >> 5) + p.parts - 1) / p.parts, first_slot = p.slot - p.s0 / each * b.Hkv;
    const float *const from = a.part + (size_t)first_slot * KcShape<D, 4, KW>::PART;
    const size_t apart = (size_t)b.Hkv * KcShape<D, 4, KW>::PART;
    int first = threadIdx.x;
    asm volatile("" : "+v"(first));
    for (int x = first; x < live * (D / 4); x += THREADS) {
        const int col = x / (D / 4), d = x % (D / 4) * 4, gc = p.cg * kKcCols + col, i = gc / a.G, h = p.hk * a.G + gc - i * a.G;
        float M = -kKqNone, l = 0.f;
        floatx4 acc = {0.f, 0.f, 0.f, 0.f};
        constexpr int U = 4;
        for (int y0 = 0; y0 < p.parts; y0 += U) {
            uint64_t ml[U], lo[U], hi[U];
#pragma unroll
            for (int y = 0; y < U; ++y) {
                const float *const part = from + (size_t)min(y0 + y, p.parts - 1) * apart;
                ml[y] = load_shared_result(reinterpret_cast<const uint64_t *>(part + S::COLS * D + 2 * col));
                lo[y] = load_shared_result(reinterpret_cast<const uint64_t *>(part + col * D + d));
                hi[y] = load_shared_result(reinterpret_cast<const uint64_t *>(part + col * D + d + 2));
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
                if (y0 + y >= p.parts) break;                        // (the last part once more)
                const float f = __builtin_amdgcn_exp2f(__uint_as_float((uint32_t)ml[y]) - Mn);
                l += __uint_as_float((uint32_t)(ml[y] >> 32)) * f;
                acc += floatx4{__uint_as_float((uint32_t)lo[y]), __uint_as_float((uint32_t)(lo[y] >> 32)), __uint_as_float((uint32_t)hi[y]),
                               __uint_as_float((uint32_t)(hi[y] >> 32))} * f;
            }
        }
        const float o[4] = {acc[0], acc[1], acc[2], acc[3]};
        kc_write(a, p, i, h, d, o, M, l);
    }
}

template <int D, int KW, bool FAR>
__global__ __launch_bounds__(KW * kWave, 2) void kvq_chunk_kernel(KcArgs) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    int *const state = reinterpret_cast<int *>(smem + kc_lds_bytes<D, KW>() - KW * kKcState * 4) + (KW > 1 ? wave_id() : 0) * kKcState;
    KcItem p;
    {
        const KcArgs a = kc_args_plan();
        if (!kc_find(p, a, blockIdx.x)) return;                      // (the same in all wavefronts)
        kc_remember(state, p);
        const int c0 = p.cg * kKcCols, live = min(max(p.n * a.G - c0, 0), kKcCols), there = min(p.rows * a.G - c0, kKcCols);
        if (live < there && p.s0 == 0) {                             // rows that are not there, of sequences that are not there: zeros
            const KcArgs e = kc_args_end();
            for (int x = threadIdx.x; x < (there - live) * (D / 8); x += KW * kWave) {
                const int gc = c0 + live + x / (D / 8), i = gc / a.G, h = p.hk * a.G + gc - i * a.G;
                *reinterpret_cast<u32x4 *>(kc_out(e, p, i, h) + x % (D / 8) * 8) = u32x4{0, 0, 0, 0};
                if (e.lse && x % (D / 8) == 0) e.lse[(size_t)(p.row0 + i) * e.Hq + h] = 0.f;
            }
        }
        if (live == 0) return;
    }
    const int live = p.n * kc_args_plan().G - p.cg * kKcCols;
    if (__builtin_amdgcn_readfirstlane(live) <= 16) kc_item<D, 1, KW, FAR>(smem, state);
    else kc_item<D, 4, KW, FAR>(smem, state);
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
static int64_t chunk_blocks(const radar_kvq_chunk_desc *d, bool packed) {
    const int64_t G = d->Hq / d->cache.Hkv;
    return packed ? d->N * G / kKcCols + d->B : (int64_t)d->B * (((int64_t)d->T_max * G + kKcCols - 1) / kKcCols);
}

struct KcRoom { size_t off_part, bytes; };
static KcRoom chunk_room(int D) {
    KcRoom r;
    r.off_part = (size_t)kKcTarget * kKcArrived * sizeof(unsigned int);       // counters first: all calls leave them at zero
    r.bytes = r.off_part + (size_t)2 * kKcTarget * kKcCols * (D + 2) * sizeof(float);
    return r;
}

extern "C" size_t radar_chunk_attention_kvq_workspace_bytes(const radar_kvq_chunk_desc *d) {
    if (check_chunk(d) != RADAR_OK) return 0;
    return chunk_room(d->cache.D).bytes;
}

template <int D, int KW, bool FAR>
static hipError_t launch_chunk(const KcArgs &a, int64_t items, hipStream_t s) {
    constexpr int bytes = kc_lds_bytes<D, KW>();
    static std::atomic<uint64_t> configured{0};            // devices on which the kernel may have so much LDS (two threads may both say so)
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    const uint64_t bit = 1ull << (device & 63);
    if (device > 63 || !(configured.load(std::memory_order_relaxed) & bit)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void *>(&kvq_chunk_kernel<D, KW, FAR>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
        configured.fetch_or(bit, std::memory_order_relaxed);
    }
    return launch("kvq_chunk", kvq_chunk_kernel<D, KW, FAR>, dim3((unsigned)items), dim3(KW * kWave), bytes, s, a);
}

extern "C" radar_status radar_chunk_attention_kvq(const void *q, const void *cache, const int32_t *block_tables, const int32_t *ctx_lens,
                                                  const int32_t *row_starts, const int32_t *n_new, void *out, float *lse_out,
                                                  const radar_kvq_chunk_desc *d, void *workspace, size_t workspace_bytes, void *stream) {
    if (!q || !cache || !block_tables || !ctx_lens || !out || !workspace || (row_starts && n_new)) return RADAR_INVALID_ARG;
    const radar_status st = check_chunk(d);
    if (st != RADAR_OK) return st;
    if (!row_starts && d->N != (int64_t)d->B * d->T_max) return RADAR_INVALID_ARG;
    const int64_t blocks = chunk_blocks(d, row_starts != nullptr), Hkv = d->cache.Hkv;
    if (blocks * Hkv >= (1 << 22)) return RADAR_UNSUPPORTED_SHAPE;
    const KcRoom room = chunk_room(d->cache.D);
    if (workspace_bytes < room.bytes) return RADAR_WORKSPACE_TOO_SMALL;
    if (((uintptr_t)workspace & 255) != 0) return RADAR_INVALID_ARG;
    KcArgs a;
    a.q = static_cast<const __bf16 *>(q); a.cache = static_cast<const unsigned char *>(cache);
    a.tables = block_tables; a.ctx_lens = ctx_lens; a.row_starts = row_starts; a.n_new = n_new;
    a.out = static_cast<__bf16 *>(out); a.lse = lse_out;
    a.B = d->B; a.T = d->T_max; a.Hq = d->Hq; a.Hkv = (int)Hkv; a.G = a.Hq / a.Hkv; a.M = d->max_blocks; a.S = d->S_max; a.N = (int)d->N;
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
    const int64_t units = blocks * Hkv;
    const int kw = units < 512 ? 8 : units < 1024 ? 4 : units < 4096 ? 2 : 1;
    a.target = d->B <= kKcPlanned ? kKcTarget : 0;
    a.least = d->rows_per_split ? d->rows_per_split / 32 : 4 * kw;
    const int64_t items = units + a.target;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool far = (int64_t)a.n_blocks * a.block_bytes > UINT32_MAX;
    auto go = [&](auto near_kernel, auto far_kernel) { return far ? far_kernel(a, items, s) : near_kernel(a, items, s); };
    const hipError_t e = D == 128 ? (kw == 8   ? go(launch_chunk<128, 8, false>, launch_chunk<128, 8, true>)
                                     : kw == 4 ? go(launch_chunk<128, 4, false>, launch_chunk<128, 4, true>)
                                     : kw == 2 ? go(launch_chunk<128, 2, false>, launch_chunk<128, 2, true>)
                                               : go(launch_chunk<128, 1, false>, launch_chunk<128, 1, true>))
                                  : (kw == 8   ? go(launch_chunk<64, 8, false>, launch_chunk<64, 8, true>)
                                     : kw == 4 ? go(launch_chunk<64, 4, false>, launch_chunk<64, 4, true>)
                                     : kw == 2 ? go(launch_chunk<64, 2, false>, launch_chunk<64, 2, true>)
                                               : go(launch_chunk<64, 1, false>, launch_chunk<64, 1, true>));
    return e == hipSuccess ? RADAR_OK : RADAR_HIP_ERROR;
}
