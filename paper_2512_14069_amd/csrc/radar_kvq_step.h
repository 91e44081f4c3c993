// Attention over the paged 4-bit cache: one wavefront's step over 32 keys (gfx950), for trees (radar_kvq_attention.hip) and for chunks of new tokens
// (radar_kvq_chunk.hip).  Which keys a column sees is the caller's to say.
#pragma once

#include <type_traits>

#include "radar_kvq.h"

namespace radar {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kqLog2e = 1.4426950408889634f;
constexpr float kqLn2 = 0.6931471805599453f;

// Args, below: what a step has to know of the cache and the call, in a kernel's own arguments: rbits, n_blocks, block_bytes (of a block, all heads) and
// scale_log2.

typedef const __attribute__((address_space(1))) unsigned char *kq_bytes;      // global memory
__device__ __forceinline__ uint64_t kq_scalar(const void *p) {
    const uint64_t v = (uint64_t)(uintptr_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
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

// What a lane holds for a step of 32 keys: two keys' codes and scales of K (tile t: key 8 * (r/4) + 4t + r%4, r = lane % 16), eight keys' of V
// (8 * (lane / 16) + e).
template <int D>
struct KqK { uint32_t code[2][D / 32]; u32x2 scale; };     // (scales of the eight rows that the lane's two are among: word t, byte r % 4)
struct KqV { uint32_t code[8]; u32x2 scale; };

// The blocks of a step's first and second 16 keys (blocks are 16 rows or more): their numbers, the same in every lane.
struct KqIds { int a, b; };
template <typename Args>
__device__ __forceinline__ KqIds kq_ids(const Args &a, const int32_t *table, int key0, int total) {
    const int last = total - 1;
    return KqIds{uniform_word(table, min(key0, last) >> a.rbits), uniform_word(table, min(key0 + 16, last) >> a.rbits)};
}
template <typename Args>
__device__ __forceinline__ bool kq_there(const Args &a, int blk) { return (uint32_t)blk < (uint32_t)a.n_blocks; }

// Where the two halves' codes and scales begin: a row is D/2 bytes of codes further on, K's or V's, and D/32 bytes of scales.  All of it in
// scalar registers; a lane adds the place of its own rows, worked out once.  Two blocks of a layer of less than 4 GB are at most 32 bits apart
// (FAR: of any layer): a load then takes the lower of the two as its scalar base and an offset in one vector register.
struct KqBase { kq_bytes code, scale; uint64_t code_up, scale_up; bool second_up; };       // the lower one, how far up the other is, which it is
template <int D, typename Args>
__device__ __forceinline__ KqBase kq_base(const Args &a, kq_bytes base, KqIds id, int key0) {
    const int R = 1 << a.rbits, row_a = key0 & (R - 1), row_b = (key0 + 16) & (R - 1);
    const uint32_t ia = kq_there(a, id.a) ? (uint32_t)id.a : 0u, ib = kq_there(a, id.b) ? (uint32_t)id.b : 0u;
    KqBase s;
    s.second_up = ib >= ia;                                          // (of one block the second half's rows are the later ones)
    const uint32_t lo = s.second_up ? ia : ib, apart = s.second_up ? ib - ia : ia - ib;
    const int row = s.second_up ? row_a : row_b, rows = s.second_up ? row_b - row_a : row_a - row_b;
    const kq_bytes c = base + (uint64_t)lo * (uint64_t)a.block_bytes;
    const uint64_t up = (uint64_t)apart * (uint64_t)a.block_bytes;
    s.code = c + row * (D / 2);
    s.scale = c + R * D + row * (D / 32);
    s.code_up = up + (int64_t)(rows * (D / 2));
    s.scale_up = up + (int64_t)(rows * (D / 32));
    return s;
}
template <typename T, bool FAR>
__device__ __forceinline__ T kq_read(kq_bytes base, uint64_t up, bool is_up, uint32_t off) {
    if constexpr (FAR) return *reinterpret_cast<const __attribute__((address_space(1))) T *>(base + (is_up ? up : 0) + off);
    else return *reinterpret_cast<const __attribute__((address_space(1))) T *>(base + (uint32_t)((is_up ? (uint32_t)up : 0u) + off));
}

template <int D, bool FAR>
__device__ __forceinline__ void kq_load_k(KqK<D> &k, KqBase s, int lane) {
    using C = KvqChunk<D>;
    const int r = lane & 15, grp = lane >> 4, group = (r >> 2) & 1, blk = D == 128 ? grp : grp >> 1;
    const bool is_up = (r >= 8) == s.second_up;
    const uint32_t at = (uint32_t)(C::k_row(8 * group + (r & 3)) + (D / 8) * grp);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        if constexpr (D == 128) {
            const u32x4 x = kq_read<u32x4, FAR>(s.code + t * C::k_row(4), s.code_up, is_up, at);
#pragma unroll
            for (int i = 0; i < 4; ++i) k.code[t][i] = x[i];
        } else {
            const u32x2 x = kq_read<u32x2, FAR>(s.code + t * C::k_row(4), s.code_up, is_up, at);
            k.code[t][0] = x[0]; k.code[t][1] = x[1];
        }
    }
    k.scale = kq_read<u32x2, FAR>(s.scale, s.scale_up, is_up, (uint32_t)((group * C::kScales + blk) * 8));
}
template <int D, bool FAR, typename Args>
__device__ __forceinline__ void kq_load_v(KqV &v, const Args &a, KqBase s, int lane) {
    using C = KvqChunk<D>;
    const int r = lane & 15, grp = lane >> 4, piece = D == 128 ? r : r >> 1, blk = D == 128 ? r >> 2 : r >> 3;
    const bool is_up = (grp >= 2) == s.second_up;
    const kq_bytes code = s.code + ((D / 2) << a.rbits);
    const uint32_t at = (uint32_t)(((grp & 1) * C::kPieces + piece) * 32);
    const u32x4 lo = kq_read<u32x4, FAR>(code, s.code_up, is_up, at), hi = kq_read<u32x4, FAR>(code + 16, s.code_up, is_up, at);
    v.scale = kq_read<u32x2, FAR>(s.scale + ((D / 32) << a.rbits), s.scale_up, is_up, (uint32_t)(((grp & 1) * C::kScales + blk) * 8));
#pragma unroll
    for (int e = 0; e < 4; ++e) { v.code[e] = lo[e]; v.code[4 + e] = hi[e]; }
}

// Of the lane's eight V rows the first n are there; the others hold anything and become zeros (K's scores are masked).
__device__ __forceinline__ void kq_clear_v(KqV &s, int n) {
#pragma unroll
    for (int e = 0; e < 8; ++e) s.code[e] = e < n ? s.code[e] : 0u;
    uint64_t both = (uint64_t)s.scale[1] << 32 | s.scale[0];
    both &= n > 0 ? ~0ull >> (64 - 8 * n) : 0ull;
    s.scale = u32x2{(uint32_t)both, (uint32_t)(both >> 32)};
}

// A NaN block of V under a probability of zero would make NaN of queries that may not see it, and so would one whose scale is larger than any that is
// written: its larger codes are infinite.  Only rows from `hidden` on are hidden from anybody, so in a step that reaches them such blocks become zeros, and NaN is
// put where a query does see one.  A lane's outputs are d = D/4 * (lane / 16) ..., all of one block of 32.  Returns which of the step's 32 keys have
// such a block there; all lanes call.
template <int D>
__device__ __forceinline__ uint32_t kq_hide_nan(KqV &s, int grp) {
    uint32_t bad = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (((s.scale[e >> 2] >> (8 * (e & 3))) & 255u) > kScaleMost) {
            bad |= 1u << e;
            s.code[e] = 0;
            s.scale[e >> 2] &= ~(255u << (8 * (e & 3)));
        }
    if (__ballot(bad != 0) == 0ull) return 0;
    const int holder = D == 128 ? 4 * grp : 8 * (grp >> 1);           // a lane that has the scales of this lane's outputs
    uint32_t all = 0;
    for (int g = 0; g < 4; ++g) all |= (uint32_t)__shfl((int)bad, 16 * g + holder) << (8 * g);
    return all;
}

// A softmax's running reference.
constexpr float kKqMost = 2048.0f;             // what a lane's eight weights may add up to before the reference is moved
// Scores from 2^25 on (in log2 units) are far.  An exponent is fma(score, scale, -reference) with the reference rounded, and what was rounded off is
// up to half a step of 32 bits: 1 below 2^25, which is harmless as all of a column's weights have it alike, but 128 from 2^31 on, where all of them would
// be zero or infinite.  So the reference of a far column, and of one that has seen no key yet, waits in LDS as a score, and its weights are
// 2^((score - reference) scale); its register holds kKqNone, which sends every step there.
constexpr float kKqNone = 3.0e38f;
__device__ __forceinline__ bool kq_is_far(float negref) { return __builtin_amdgcn_ubfe(__float_as_uint(negref), 26, 5) >= 19; }      // exponent of 25 or more

// One wavefront, one step: scores of 32 keys, softmax against the running reference, outputs.  The loads of the wavefront's next step are
// asked for as soon as the registers of this one's are free: K's after the scores, V's at the end.
// From key `hidden` on there are keys that not all columns see; allow(column, key0 - hidden) has a bit for each of the 32 that the column sees.
template <int D, int NC, int AHEAD, typename QOp, typename NextK, typename Allow, typename Args>
__device__ __forceinline__ void kq_step(const KqK<D> &k, KqV &v, KqIds id, QOp qop, NextK next_k, floatx4 (&oacc)[D / 16][NC], float (&negref)[NC],
                                        float (&l_run)[NC], Allow allow, float *s_ref, const Args &a, int key0, int hidden, int total) {
    constexpr int NM = D / 16, CH = D / 32, COLS = 16 * NC;          // output tiles; steps of the scores' product; columns
    const int lane = lane_id(), r = lane & 15;
    floatx4 sacc[2][NC];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int n = 0; n < NC; ++n) sacc[t][n] = floatx4{0.f, 0.f, 0.f, 0.f};
    const uint32_t pick = 0x0c0c0cu | (uint32_t)(r & 3) << 24;       // that byte on top, zeros under it
    const float f[2] = {__uint_as_float(__builtin_amdgcn_perm(0u, k.scale[0], pick) >> 1), __uint_as_float(__builtin_amdgcn_perm(0u, k.scale[1], pick) >> 1)};
    // (the queries' operands come from LDS where there are many: asked for AHEAD of them ahead; the next codes are turned into
    // operands between the products of the ones before)
    constexpr int NQ = NC * CH;
    bf16x8 q[AHEAD];
#pragma unroll
    for (int x = 0; x < AHEAD; ++x) q[x] = qop(x % NC, x / NC);
    uint32_t w[2][2][4];
    kvq_decode8(k.code[0][0], f[0], w[0][0]);
    kvq_decode8(k.code[1][0], f[1], w[0][1]);
    if (NC > 2) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        if (c + 1 < CH) {
            kvq_decode8(k.code[0][c + 1], f[0], w[(c + 1) & 1][0]);
            kvq_decode8(k.code[1][c + 1], f[1], w[(c + 1) & 1][1]);
        }
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            const int x = c * NC + n;
            const bf16x8 cur = q[x % AHEAD];
            if (x + AHEAD < NQ) q[x % AHEAD] = qop((x + AHEAD) % NC, (x + AHEAD) / NC);
#pragma unroll
            for (int t = 0; t < 2; ++t)
                sacc[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u32x4{w[c & 1][t][0], w[c & 1][t][1], w[c & 1][t][2], w[c & 1][t][3]}), cur, sacc[t][n], 0, 0, 0);
        }
        if (NC > 2) {
#pragma unroll
            for (int n = 0; n < NC; ++n) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    if (c + 1 < CH) __builtin_amdgcn_sched_group_barrier(0x002, 1, 0);
                }
                if (c * NC + n + AHEAD < NQ) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    __builtin_amdgcn_sched_barrier(0);         // (the phases stay apart: run into each other they need twice the registers)
    next_k();
    __builtin_amdgcn_s_setprio(0);
    // this lane's eight keys: 8 * grp + e, e = 4 * tile + register
    uint32_t nan_keys = 0;
    const bool whole = key0 + 32 <= hidden && kq_there(a, id.a) && kq_there(a, id.b);      // nothing to mask
    if (!whole) {
        int lane2 = lane;
        asm volatile("" : "+v"(lane2));                              // (what only this needs is worked out here, and not kept in registers)
        const int r = lane2 & 15, grp = lane2 >> 4;
        const int n_there = kq_there(a, grp < 2 ? id.a : id.b) ? min(max(total - (key0 + 8 * grp), 0), 8) : 0;
        kq_clear_v(v, n_there);
        nan_keys = kq_hide_nan<D>(v, grp);
        const uint32_t there = (1u << n_there) - 1;
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            const uint32_t mine = (allow(n * 16 + r, key0 - hidden) >> (8 * grp)) & there;
#pragma unroll
            for (int e = 0; e < 8; ++e) sacc[e >> 2][n][e & 3] = (mine >> e) & 1u ? sacc[e >> 2][n][e & 3] : -INFINITY;
        }
    }
    bf16x8 p[NC];
#pragma unroll
    for (int n = 0; n < NC; ++n) {
        // The eight scores' exponentials against the running reference; p is the matrix cores' operand, the sum is of the unrounded ones, in fp32.
        auto weigh = [&](auto base, float shift) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[e >> 2][n][e & 3] - base, a.scale_log2, shift));
                sum = e == 0 ? w : sum + w;
                p[n][e] = (__bf16)w;
            }
            return sum;
        };
        float sum = weigh(std::integral_constant<int, 0>{}, negref[n]);
        // The reference is the columns' maximum at the time when some lane's sum last went past 2^11 (for a column without a key: at once).  Only then
        // do the four lanes of a column compare their maxima, and outputs and sums get rescaled: no step but a wavefront's first does it as a rule.
        // Weights of up to 2^11 instead of 1 lose nothing: they keep bf16's eight bits, and sums and outputs are fp32.
        if (__any(sum > kKqMost)) {
            float mx = sacc[0][n][0];
#pragma unroll
            for (int e = 1; e < 8; ++e) mx = fmaxf(mx, sacc[e >> 2][n][e & 3]);
            mx = kq_column_max(mx);
            int tid = threadIdx.x;
            asm volatile("" : "+v"(tid));                            // (the address is worked out here, and not kept in registers)
            float *const ref = s_ref + (tid >> 6) * COLS + n * 16 + (tid & 15);                  // (a column's four lanes agree)
            // a weight is 2^((score - base) scale + shift): shift 0 for a far column, base 0 for others
            const float old = *ref, old_neg = negref[n], old_base = kq_is_far(old_neg) ? old : 0.f, old_shift = kq_is_far(old_neg) ? 0.f : old_neg;
            mx = kq_is_far(old_neg) ? fmaxf(old, mx) : mx;
            const float neg = fminf(old_neg, -(mx * a.scale_log2)), base = kq_is_far(neg) ? mx : 0.f, shift = kq_is_far(neg) ? 0.f : neg;
            *ref = mx;
            negref[n] = kq_is_far(neg) ? kKqNone : neg;
            const float alpha = __builtin_amdgcn_exp2f(__builtin_fmaf(old_base - base, a.scale_log2, shift - old_shift));
            l_run[n] *= alpha;
#pragma unroll
            for (int m = 0; m < NM; ++m) oacc[m][n] *= alpha;
            sum = weigh(base, shift);
        }
        sum += l_run[n];
        asm volatile("" : "+v"(sum));                                // (added up here: left to the end of the step all of them stay in registers)
        l_run[n] = sum;
        __builtin_amdgcn_sched_barrier(0);
    }
    // Two wavefronts share a SIMD, and left alone do the same at the same time.  The one that has products goes first, the other one's softmax fills
    // the gaps (four sequences of 16384 rows, 64 heads: 142 us without, 133 with; taking turns between barriers 146).
    __builtin_amdgcn_s_setprio(1);
    // V^T operands: product m of lane (r, grp) is d = D/16 * r + m, keys 8 * grp + 0..7; a byte of the codes has two products' values
    float fv[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) fv[e] = kvq_scale((v.scale[e >> 2] >> (8 * (e & 3))) & 255u);
    if constexpr (D == 64) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v.code[e] >>= 16 * (r & 1);
    }
    u32x4 vop[2][2];
    auto decode = [&](auto byte, u32x4 (&to)[2]) {
        constexpr int J = decltype(byte)::value;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const uint32_t x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v.code[e], fv[e], J));
            const uint32_t y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v.code[e + 1], fv[e + 1], J));
            to[0][e >> 1] = __builtin_amdgcn_perm(y, x, 0x05040100u);
            to[1][e >> 1] = __builtin_amdgcn_perm(y, x, 0x07060302u);
        }
    };
    decode(std::integral_constant<int, 0>{}, vop[0]);
    if (NC > 2) __builtin_amdgcn_sched_barrier(0);
    auto outputs = [&](auto byte) {
        constexpr int J = decltype(byte)::value, LAST = NM / 2 - 1;
        if constexpr (J < LAST) decode(std::integral_constant<int, J + 1>{}, vop[(J + 1) & 1]);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int n = 0; n < NC; ++n)
                oacc[2 * J + x][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vop[J & 1][x]), p[n], oacc[2 * J + x][n], 0, 0, 0);
        if (NC > 2) {
#pragma unroll
            for (int x = 0; x < 2 * NC; ++x) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                if (J < LAST) __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    outputs(std::integral_constant<int, 0>{});
    outputs(std::integral_constant<int, 1>{});
    if constexpr (NM > 4) {
        outputs(std::integral_constant<int, 2>{});
        outputs(std::integral_constant<int, 3>{});
    }
    if (!whole && __ballot(nan_keys != 0) != 0ull) {
        int lane2 = lane;
        asm volatile("" : "+v"(lane2));
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            const bool sees = (nan_keys & allow(n * 16 + (lane2 & 15), key0 - hidden)) != 0;
#pragma unroll
            for (int m = 0; m < NM; ++m) oacc[m][n] = sees ? floatx4{NAN, NAN, NAN, NAN} : oacc[m][n];
        }
    }
}

}  // namespace radar
