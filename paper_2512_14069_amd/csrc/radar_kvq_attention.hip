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
#include <algorithm>

#include "radar_host.h"
#include "radar_kvq.h"

namespace radar {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kqLog2e = 1.4426950408889634f;
constexpr float kqLn2 = 0.6931471805599453f;

struct KqArgs {
    const __bf16 *q;
    const unsigned char *cache;
    const int32_t *tables, *parents, *ctx_lens, *n_nodes;
    __bf16 *out;
    float *lse;
    int B, T, Hq, Hkv, G, M, S, rbits, n_blocks;
    int64_t q_sb, q_st, q_sh, o_sb, o_st, o_sh;
    float scale_log2;
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

// The larger (the sum) over the four lanes that share a column: lane ^ 16, lane ^ 32.
__device__ __forceinline__ float kq_column_max(float v) {
    uint32_t u = __float_as_uint(v);
    const auto s = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
    u = __float_as_uint(v);
    const auto t = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
}
__device__ __forceinline__ float kq_column_sum(float v) {
    uint32_t u = __float_as_uint(v);
    const auto s = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    u = __float_as_uint(v);
    const auto t = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(t[0]) + __uint_as_float(t[1]);
}

// What a lane loads for a step of 32 keys: two keys' codes and scales of K (tile t: key 8 * (r/4) + 4t + r%4, r = lane % 16), eight keys' of V.
template <int D>
struct KqStep {
    uint32_t k[2][D / 32];
    uint32_t ks[2];
    uint32_t v[8];
    u32x2 vs;
    uint32_t there;                            // bit e: key 8 * (lane / 16) + e is there
};

template <int D>
__device__ __forceinline__ void kq_load(KqStep<D> &s, const KqArgs &a, const int32_t *table, int hk, int key0, int total) {
    using C = KvqChunk<D>;
    const int lane = lane_id(), r = lane & 15, grp = lane >> 4, R = 1 << a.rbits;
    auto chunk_of = [&](int key, bool *there) {
        const int blk = table[min(key, total - 1) >> a.rbits];
        *there = key < total && (uint32_t)blk < (uint32_t)a.n_blocks;
        return a.cache + ((size_t)((uint32_t)blk < (uint32_t)a.n_blocks ? blk : 0) * a.Hkv + hk) * C::bytes(R);
    };
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int key = key0 + 8 * (r >> 2) + 4 * t + (r & 3), row = key & (R - 1);
        bool there;
        const unsigned char *const c = chunk_of(key, &there);
        if constexpr (D == 128) {
            const u32x4 w = *reinterpret_cast<const u32x4 *>(c + C::k_row(row) + 16 * grp);
#pragma unroll
            for (int i = 0; i < 4; ++i) s.k[t][i] = w[i];
            s.ks[t] = c[C::k_scale(R, row, grp)];
        } else {
            const u32x2 w = *reinterpret_cast<const u32x2 *>(c + C::k_row(row) + 8 * grp);
            s.k[t][0] = w[0]; s.k[t][1] = w[1];
            s.ks[t] = c[C::k_scale(R, row, grp >> 1)];
        }
    }
    const int key = key0 + 8 * grp, row = key & (R - 1);
    bool there;
    const unsigned char *const c = chunk_of(key, &there);
    const int n = there ? min(total - key, 8) : 0;
    s.there = (1u << n) - 1;
    const u32x4 lo = *reinterpret_cast<const u32x4 *>(c + C::v_piece(R, row, D == 128 ? r : r >> 1));
    const u32x4 hi = *reinterpret_cast<const u32x4 *>(c + C::v_piece(R, row, D == 128 ? r : r >> 1) + 16);
    s.vs = *reinterpret_cast<const u32x2 *>(c + C::v_scale(R, row, D == 128 ? r >> 2 : r >> 3));
#pragma unroll
    for (int e = 0; e < 4; ++e) { s.v[e] = lo[e]; s.v[4 + e] = hi[e]; }
    if (n < 8) {                                                     // rows that are not there hold anything: zeros in V (K is masked)
#pragma unroll
        for (int e = 0; e < 8; ++e) s.v[e] = e < n ? s.v[e] : 0u;
        uint64_t both = (uint64_t)s.vs[1] << 32 | s.vs[0];
        both &= n > 0 ? ~0ull >> (64 - 8 * n) : 0ull;
        s.vs = u32x2{(uint32_t)both, (uint32_t)(both >> 32)};
    }
}

// A NaN block of V under a probability of zero would make NaN of queries that may not see it.  Only rows of the tree are hidden from anybody, so
// in a step that reaches them NaN blocks become zeros, and NaN is put where a query does see one.  A lane's outputs are d = D/4 * (lane / 16) ...,
// all of one block of 32.  allow: the lane's eight keys that its column sees.  All lanes call.
template <int D>
__device__ __forceinline__ bool kq_hide_nan(KqStep<D> &s, uint32_t allow) {
    const int lane = lane_id(), grp = lane >> 4;
    uint32_t bad = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (((s.vs[e >> 2] >> (8 * (e & 3))) & 255u) == kScaleNaN) {
            bad |= 1u << e;
            s.v[e] = 0;
            s.vs[e >> 2] &= ~(255u << (8 * (e & 3)));
        }
    if (__ballot(bad != 0) == 0ull) return false;
    const int holder = D == 128 ? 4 * grp : 8 * (grp >> 1);           // a lane that has the scales of this lane's outputs
    bool seen = false;
    for (int g = 0; g < 4; ++g) {
        const uint32_t b = (uint32_t)__shfl((int)bad, 16 * g + holder), see = (uint32_t)__shfl((int)allow, 16 * g + (lane & 15));
        seen |= (b & see) != 0;
    }
    return seen;
}

// One wavefront: 32 keys against 16 query columns.
template <int D>
__device__ __forceinline__ void kq_step(KqStep<D> &s, const bf16x8 (&qop)[D / 32], floatx4 (&oacc)[D / 16], float &m_run, float &l_run,
                                        uint64_t anc, int key0, int L, float scale_log2) {
    const int lane = lane_id(), r = lane & 15, grp = lane >> 4;
    floatx4 sacc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        sacc[t] = floatx4{0.f, 0.f, 0.f, 0.f};
        const float f = kvq_scale(s.ks[t]);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            uint32_t w[4];
            kvq_decode8(s.k[t][c], f, w);
            sacc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]}), qop[c], sacc[t], 0, 0, 0);
        }
    }
    // this lane's eight keys: 8 * grp + e, e = 4 * tile + register
    uint32_t allow = s.there;
    const int first = key0 + 8 * grp - L;                            // the first of them, counted from the tree's first row
    if (first + 8 > 0) {
        const uint32_t tree = first >= 64 ? 0u : (uint32_t)(first >= 0 ? anc >> first : anc << -first);
        allow &= first >= 0 ? tree : tree | ((1u << -first) - 1);
    }
    float x[8], mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        x[e] = (allow >> e) & 1u ? sacc[e >> 2][e & 3] * scale_log2 : -INFINITY;
        mx = fmaxf(mx, x[e]);
    }
    mx = kq_column_max(mx);
    const float m_new = fmaxf(m_run, mx), ref = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(m_run - ref);         // nothing yet: 0
    m_run = m_new;
    l_run *= alpha;
#pragma unroll
    for (int m = 0; m < D / 16; ++m) oacc[m] *= alpha;
    bf16x8 p;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float w = __builtin_amdgcn_exp2f(x[e] - ref);
        l_run += w;
        p[e] = (__bf16)w;
    }
    const bool nan = key0 + 32 > L && kq_hide_nan<D>(s, allow);
    // V^T operands: product m of lane (r, grp) is d = D/16 * r + m, keys 8 * grp + 0..7
    constexpr int NM = D / 16;
    uint32_t vop[NM][4];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const float f0 = kvq_scale((s.vs[e >> 2] >> (8 * (e & 3))) & 255u), f1 = kvq_scale((s.vs[(e + 1) >> 2] >> (8 * ((e + 1) & 3))) & 255u);
        const uint32_t w0 = D == 128 ? s.v[e] : s.v[e] >> (16 * (r & 1)), w1 = D == 128 ? s.v[e + 1] : s.v[e + 1] >> (16 * (r & 1));
        uint32_t a[4], b[4];
        kvq_decode8(w0, f0, a);
        kvq_decode8(w1, f1, b);
#pragma unroll
        for (int j = 0; j < NM / 2; ++j) {
            vop[2 * j][e >> 1] = __builtin_amdgcn_perm(b[j], a[j], 0x05040100u);
            vop[2 * j + 1][e >> 1] = __builtin_amdgcn_perm(b[j], a[j], 0x07060302u);
        }
    }
#pragma unroll
    for (int m = 0; m < NM; ++m)
        oacc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u32x4{vop[m][0], vop[m][1], vop[m][2], vop[m][3]}), p, oacc[m], 0, 0, 0);
    if (key0 + 32 > L)
#pragma unroll
        for (int m = 0; m < NM; ++m) oacc[m] = nan ? floatx4{NAN, NAN, NAN, NAN} : oacc[m];
}

constexpr int kKqThreads = 256;
constexpr int kKqWaves = kKqThreads / kWave;

template <int D>
__global__ __launch_bounds__(kKqThreads) void kvq_attn_kernel(KqArgs a) {
    constexpr int NM = D / 16;
    __shared__ float s_m[kKqWaves][16], s_l[kKqWaves][16];
    __shared__ float s_o[kKqWaves][16][D + 4];
    const int b = blockIdx.z, hk = blockIdx.y, cb = blockIdx.x, lane = lane_id(), w = wave_id(), r = lane & 15, grp = lane >> 4;
    const KqSeq s = kq_seq(a, b);
    const int col = cb * 16 + r, i = col / a.G, h = hk * a.G + col % a.G;
    const bool live = i < s.nn;
    bf16x8 qop[D / 32];                        // d = (D/4) * grp + 8 * c + 0..7
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
        u32x4 x = {0, 0, 0, 0};
        if (live) x = *reinterpret_cast<const u32x4 *>(a.q + (size_t)b * a.q_sb + (size_t)i * a.q_st + (size_t)h * a.q_sh + (D / 4) * grp + 8 * c);
        qop[c] = __builtin_bit_cast(bf16x8, x);
    }
    const uint64_t words = kq_ancestors(a.parents ? a.parents + (size_t)b * a.T : nullptr, s.nn);
    const int ii = min(i, RADAR_T_MAX - 1);
    uint64_t anc = (uint64_t)(uint32_t)__shfl((int)(uint32_t)words, ii) | (uint64_t)(uint32_t)__shfl((int)(uint32_t)(words >> 32), ii) << 32;
    if (!live) anc = 0;
    floatx4 oacc[NM];
#pragma unroll
    for (int m = 0; m < NM; ++m) oacc[m] = floatx4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;
    const int32_t *const table = a.tables + (size_t)b * a.M;
    if (cb * 16 < s.nn * a.G)
        for (int key0 = w * 32; key0 < s.total; key0 += kKqWaves * 32) {
            KqStep<D> st;
            kq_load<D>(st, a, table, hk, key0, s.total);
            kq_step<D>(st, qop, oacc, m_run, l_run, anc, key0, s.L, a.scale_log2);
        }
    const float l = kq_column_sum(l_run);
    if (grp == 0) { s_m[w][r] = m_run; s_l[w][r] = l; }
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) s_o[w][r][(D / 4) * grp + NM * e + m] = oacc[m][e];
    __syncthreads();
    // a lane: D/16 values of one column
    const int mc = threadIdx.x & 15, d0 = (threadIdx.x >> 4) * (D / 16), col2 = cb * 16 + mc, i2 = col2 / a.G, h2 = hk * a.G + col2 % a.G;
    if (i2 >= a.T) return;
    float M = -INFINITY, sum = 0.f, acc[D / 16];
    for (int v = 0; v < kKqWaves; ++v) M = fmaxf(M, s_m[v][mc]);
    const float ref = M == -INFINITY ? 0.f : M;
    for (int d = 0; d < D / 16; ++d) acc[d] = 0.f;
    for (int v = 0; v < kKqWaves; ++v) {
        const float f = __builtin_amdgcn_exp2f(s_m[v][mc] - ref);
        sum += s_l[v][mc] * f;
        for (int d = 0; d < D / 16; ++d) acc[d] += s_o[v][mc][d0 + d] * f;
    }
    const bool on = i2 < s.nn;
    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    __bf16 *const o = a.out + (size_t)b * a.o_sb + (size_t)i2 * a.o_st + (size_t)h2 * a.o_sh + d0;
    for (int d = 0; d < D / 16; ++d) o[d] = (__bf16)(on ? acc[d] * inv : 0.f);
    if (a.lse && d0 == 0) a.lse[((size_t)b * a.T + i2) * a.Hq + h2] = on ? (M + __builtin_amdgcn_logf(sum)) * kqLn2 : 0.f;
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
    return RADAR_OK;
}

extern "C" size_t radar_tree_attention_kvq_workspace_bytes(const radar_kvq_attn_desc *d) {
    if (check_kvq_attn(d) != RADAR_OK) return 0;
    return 256;
}

extern "C" radar_status radar_tree_attention_kvq(const void *q, const void *cache, const int32_t *block_tables, const int32_t *parents,
                                                 const int32_t *ctx_lens, const int32_t *n_nodes, void *out, float *lse_out,
                                                 const radar_kvq_attn_desc *d, void *workspace, size_t workspace_bytes, void *stream) {
    if (!q || !cache || !block_tables || !ctx_lens || !out || !workspace) return RADAR_INVALID_ARG;
    const radar_status st = check_kvq_attn(d);
    if (st != RADAR_OK) return st;
    if (workspace_bytes < 256) return RADAR_WORKSPACE_TOO_SMALL;
    if (((uintptr_t)workspace & 255) != 0) return RADAR_INVALID_ARG;
    KqArgs a;
    a.q = static_cast<const __bf16 *>(q); a.cache = static_cast<const unsigned char *>(cache);
    a.tables = block_tables; a.parents = parents; a.ctx_lens = ctx_lens; a.n_nodes = n_nodes;
    a.out = static_cast<__bf16 *>(out); a.lse = lse_out;
    a.B = d->B; a.T = d->T_max; a.Hq = d->Hq; a.Hkv = d->cache.Hkv; a.G = a.Hq / a.Hkv; a.M = d->max_blocks; a.S = d->S_max;
    a.rbits = kvq_log2(d->cache.block_rows); a.n_blocks = d->cache.n_blocks;
    const int64_t D = d->cache.D;
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
    const int64_t cols = (int64_t)a.T * a.G;
    const dim3 grid((unsigned)((cols + 15) / 16), (unsigned)a.Hkv, (unsigned)a.B);
    const hipError_t e = launch("kvq_attention", d->cache.D == 128 ? kvq_attn_kernel<128> : kvq_attn_kernel<64>, grid, dim3(kKqThreads), 0,
                                static_cast<hipStream_t>(stream), a);
    return e == hipSuccess ? RADAR_OK : RADAR_HIP_ERROR;
}
