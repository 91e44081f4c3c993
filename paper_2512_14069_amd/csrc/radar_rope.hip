// Rotary positions with one to four axes: rows of q and k turned (radar_rope), and on the way into the paged 4-bit cache (radar_kvq_append_rope), for gfx950.
//
// Pair j of a row is turned by t = position * inv_freq[j].  Angles are worked out in 64 bits: a position of 2^20 leaves fp32 four bits of
// a radian's fraction.  So is the turn itself, which costs nothing here (the vector units do as many products in 64 bits as in 32, and the bytes take
// longer) and leaves one rounding, to bf16 by way of fp32: k's codes are then the same whatever the order of the arithmetic.
//
// A workgroup has eight rows and some of the heads.  It finds out once which sequences its rows belong to and works out their sines and cosines (two a
// lane at D = 128), which lie in LDS until every lane has those of its eight pairs in registers; then a lane turns the same eight pairs of one head after the other.
//
// Many rows are bound by their bytes: 8360 rows of 40 heads, 171 MB, 35.4 us or 4.84 TB/s (16384 rows 5.3; a copy 5.1); into the cache 16384 rows of 32 heads on 8, 353 MB,
// 79.6 us or 4.44 TB/s, as codes are stored four bytes a lane.  Few rows are one launch: 60 rows 4.0 us, into the cache 4.8.
#include <algorithm>
#include <cmath>

#include "radar_host.h"
#include "radar_kvq.h"
#include "radar_rows.h"

namespace radar {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kRpThreads = 256, kRpRows = 8;
constexpr int kRpSequences = 1 << 30;          // most: a sequence and a wavefront's lanes behind it are counted in 32 bits
constexpr int64_t kRpGroups = 512;             // workgroups to aim for (960 rows of trees: 7.4 us with 512, 8.0 with 256, 9.1 with 1024)

struct RpArgs {
    const __bf16 *q, *k, *v;
    __bf16 *q_out, *k_out;
    unsigned char *cache;                      // null: k goes to k_out
    const float *inv_freq;
    const int32_t *positions, *ctx_lens, *row_starts, *n_new, *slots;
    int64_t N, total;                          // rows; slots of the cache
    int64_t q_sn, q_sh, kv_sn, kv_sh, qo_sn, qo_sh, ko_sn, ko_sh;
    int B, T, Hq, Hkv, D, pairs, axes, adjacent, rbits;
    int q_blocks, k_blocks, per_q, per_k, per_v;           // workgroups of eight rows' q and k; rounds of heads of a workgroup
    double scale;
    uint64_t axis[4];                          // two bits a pair
};

// Sine and cosine of an angle in radians: the nearest multiple of pi/2 is taken off in two parts (pi/2 to 107 bits, exact products by fma), and of what
// is left, at most pi/4, both are their Taylor sums to the 16th power (the next terms are below 2^-54).
__device__ __forceinline__ void rp_sin_cos(double t, double *sine, double *cosine) {
    const double n = rint(t * 0.63661977236758134308);     // 2 / pi
    double r = fma(-n, 1.57079632679489655800, t);
    r = fma(-n, 6.12323399573676603587e-17, r);
    const double z = r * r;
    double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;
    s = fma(s, z, 1.0 / 6227020800.0);
    s = fma(s, z, -1.0 / 39916800.0);
    s = fma(s, z, 1.0 / 362880.0);
    s = fma(s, z, -1.0 / 5040.0);
    s = fma(s, z, 1.0 / 120.0);
    s = fma(s, z, -1.0 / 6.0);
    s = fma(s * z, r, r);
    c = fma(c, z, -1.0 / 87178291200.0);
    c = fma(c, z, 1.0 / 479001600.0);
    c = fma(c, z, -1.0 / 3628800.0);
    c = fma(c, z, 1.0 / 40320.0);
    c = fma(c, z, -1.0 / 720.0);
    c = fma(c, z, 1.0 / 24.0);
    c = fma(c, z, -0.5);
    c = fma(c, z, 1.0);
    const double quarter = n - 4.0 * floor(n * 0.25);      // 0 ... 3
    const bool odd = quarter == 1.0 || quarter == 3.0;
    const double a = odd ? c : s, b = odd ? s : c;
    *sine = quarter >= 2.0 ? -a : a;
    *cosine = quarter == 1.0 || quarter == 2.0 ? -b : b;
}

// Values 2 i and 2 i + 1 of a word of bf16, and back: rounded to fp32, then to bf16, to the nearest.
__device__ __forceinline__ double rp_low(uint32_t w) { return (double)__uint_as_float(w << 16); }
__device__ __forceinline__ double rp_high(uint32_t w) { return (double)__uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t rp_pack(double lo, double hi) {
    float x = (float)lo, y = (float)hi;
    asm("" : "+v"(x), "+v"(y));                // (left alone, the two roundings become one, which takes eight instructions more)
    bf16x2 o;
    o[0] = (__bf16)x;
    o[1] = (__bf16)y;
    return __builtin_bit_cast(uint32_t, o);
}

// What a workgroup knows of its rows.
struct RpRow { int there, slot; };

// Which eight-value pieces a lane has of a row: those of its eight pairs, or two that are copied.
struct RpPieces { int a, b; bool turned; };
__device__ __forceinline__ RpPieces rp_pieces(const RpArgs &g, int p) {
    const int turning = g.pairs >> 3;
    RpPieces x;
    x.turned = p < turning;
    const bool halves = x.turned && !g.adjacent;
    x.a = halves ? p : 2 * p;
    x.b = halves ? p + turning : 2 * p + 1;
    return x;
}

__device__ __forceinline__ void rp_turn(u32x4 &a, u32x4 &b, const double (&c)[8], const double (&s)[8], bool adjacent) {
    if (adjacent) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const double x = rp_low(a[e]), y = rp_high(a[e]);
            a[e] = rp_pack(fma(x, c[e], -(y * s[e])), fma(x, s[e], y * c[e]));
            const double z = rp_low(b[e]), w = rp_high(b[e]);
            b[e] = rp_pack(fma(z, c[4 + e], -(w * s[4 + e])), fma(z, s[4 + e], w * c[4 + e]));
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const double x0 = rp_low(a[e]), x1 = rp_high(a[e]), y0 = rp_low(b[e]), y1 = rp_high(b[e]);
            a[e] = rp_pack(fma(x0, c[2 * e], -(y0 * s[2 * e])), fma(x1, c[2 * e + 1], -(y1 * s[2 * e + 1])));
            b[e] = rp_pack(fma(x0, s[2 * e], y0 * c[2 * e]), fma(x1, s[2 * e + 1], y1 * c[2 * e + 1]));
        }
    }
}

// Rows of more bytes than the L2s hold are read and stored past them: nobody finds them there later (8360 rows of 40 heads, cold: 36.0 us, 39.5 through them;
// 960 rows of 48 11.1, 11.0).
constexpr int64_t kRpStream = 64 << 20;
template <bool STREAM>
__device__ __forceinline__ u32x4 rp_load(const __bf16 *p) {
    const u32x4 *const at = reinterpret_cast<const u32x4 *>(p);
    if constexpr (STREAM) return __builtin_nontemporal_load(at);
    else return *at;
}
template <bool STREAM>
__device__ __forceinline__ void rp_store(__bf16 *p, u32x4 x) {
    u32x4 *const at = reinterpret_cast<u32x4 *>(p);
    if constexpr (STREAM) __builtin_nontemporal_store(x, at);
    else *at = x;
}

// Lane r < 8: the last sequence that starts at row n0 + r or before it, for rows that are `far`: no earlier one than seq; for others seq.  Eight lanes a row look at eight
// starts at a time, which leave a ninth: four rows, two of them 4000 idle sequences on, 4.7 us, 50000 on 5.3 (side by side 3.9; one sequence looked at after the other 332 and
// 8130).  All lanes call; any starts keep the result within [seq, B).
__device__ __forceinline__ int rp_behind(const RpArgs &g, int seq, bool far, int64_t n0) {
    const int lane = lane_id(), r = lane >> 3, k = lane & 7;
    int first = __shfl(seq, r), left = __shfl((int)far, r) != 0 ? g.B - first : 1;
    while (__ballot(left > 1) != 0) {
        const int step = (left + 8) / 9, at = (k + 1) * step;
        const uint64_t yes = __ballot(at < left && (int64_t)g.row_starts[first + min(at, left - 1)] <= n0 + r);
        const int on = __popcll(yes >> (8 * r) & 255) * step;
        first += on;
        left = min(step, left - on);
    }
    return __shfl(first, lane < kRpRows ? 8 * lane : lane);
}

// D0: the head's values, 0: any (g.D).  CACHE: k and v go into the cache.
template <int D0, bool CACHE, bool STREAM>
__global__ __launch_bounds__(kRpThreads) void rope_kernel(RpArgs g) {
    constexpr int kMostLanes = D0 ? D0 / 16 : 16;          // of a head's row
    __shared__ RpRow s_row[kRpRows];
    __shared__ int64_t s_pos[4][kRpRows];
    __shared__ __attribute__((aligned(16))) double2 s_cs[kRpRows * 8 * kMostLanes];
    __shared__ __attribute__((aligned(16))) u32x4 s_k[CACHE ? kRpThreads * 2 : 1];
    const int D = D0 ? D0 : g.D, LP = D / 16, tid = threadIdx.x, lane = lane_id();
    const int64_t n0 = (int64_t)blockIdx.x * kRpRows;
    const int y = blockIdx.y, role = y < g.q_blocks ? 0 : y < g.q_blocks + g.k_blocks ? 1 : 2;

    // ---- a lane's place, and its first values, which are asked for before anything is known of the rows (all N rows are memory of the tensors)
    const int per = kRpRows * LP, heads = kRpThreads / per;          // lanes of a head's eight rows; heads a round
    const int place = tid / per, rest = tid - place * per, row = rest / LP, p = rest - row * LP;
    const RpPieces at = rp_pieces(g, p);
    constexpr int V_LANES = CACHE ? kRpRows * D0 / 8 : 1, V_HEADS = kRpThreads / V_LANES;          // v: of a head's eight rows; heads a round
    const int l = tid % V_LANES, part = l / kWave * 8, row_in = l % kWave / 8, piece_in = part + l % 8;
    const bool is_v = CACHE && role == 2, is_q = role == 0;
    const int H = is_q ? g.Hq : g.Hkv, rounds = is_q ? g.per_q : is_v ? g.per_v : g.per_k, step = is_v ? V_HEADS : heads;
    const int h0 = (y - (is_q ? 0 : is_v ? g.q_blocks + g.k_blocks : g.q_blocks)) * rounds * step + (is_v ? tid / V_LANES : place);
    const int64_t n = min(n0 + (is_v ? row_in : row), g.N - 1), in_h = is_q ? g.q_sh : g.kv_sh;
    const __bf16 *const from = (is_q ? g.q : is_v ? g.v : g.k) + n * (is_q ? g.q_sn : g.kv_sn);
    u32x4 a, b;
    auto ask = [&](int h) {                                          // (past the heads: the last one once more)
        const __bf16 *const of = from + min(h, H - 1) * in_h;
        if (is_v) {
            a = rp_load<STREAM>(of + piece_in * 8);
        } else {
            a = rp_load<STREAM>(of + at.a * 8);
            b = rp_load<STREAM>(of + at.b * 8);
        }
    };
    ask(h0);

    // ---- the rows: sequence, number in it, whether it is there, positions, slots.  One wavefront finds them; what it loads is asked for as soon as an
    // address is known, whether the row is there or not.
    if (wave_id() == 0) {
        const int64_t mine = min(n0 + min(lane, kRpRows - 1), g.N - 1);
        int position[4] = {0, 0, 0, 0};
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (g.positions && x < g.axes) position[x] = g.positions[x * g.N + mine];
        int seq, i, ctx;
        bool there = n0 + lane < g.N;
        if (g.row_starts) {
            // up to 63 sequences at once, else the 63 from the first row's on; where a row lies behind them all, by a search
            const int base = g.B < kWave ? 0 : max(last_at_most(g.B, n0, [&](int x) { return (int64_t)g.row_starts[x]; }), 0);
            const int start = g.row_starts[min(base + lane, g.B)], context = g.ctx_lens ? g.ctx_lens[min(base + lane, g.B - 1)] : 0;
            int hit = 0;
#pragma unroll
            for (int r = 0; r < kRpRows; ++r) {
                const uint64_t begun = __ballot(base + lane < g.B && (int64_t)start <= n0 + r);
                if (r == lane && begun != 0) hit = 63 - __clzll((long long)begun);
            }
            seq = base + hit;
            int from = __shfl(start, hit), to = __shfl(start, min(hit + 1, kWave - 1));
            ctx = __shfl(context, hit);
            const bool far = hit == kWave - 1 && lane < kRpRows && there;
            if (__ballot(far) != 0) {
                seq = rp_behind(g, seq, far, n0);
                if (far) {
                    from = g.row_starts[seq];
                    to = g.row_starts[seq + 1];
                    ctx = g.ctx_lens ? g.ctx_lens[seq] : 0;
                }
            }
            there = there && mine >= from && mine < to && mine - from < g.T;
            i = there ? (int)mine - from : 0;
        } else {
            seq = (int)((uint32_t)mine / (uint32_t)g.T);
            i = (int)((uint32_t)mine - (uint32_t)seq * (uint32_t)g.T);
            ctx = g.ctx_lens ? g.ctx_lens[seq] : 0;
            there = there && (!g.n_new || i < g.n_new[seq]);
        }
        there = there && ctx >= 0;
        if (lane < kRpRows) {
            s_row[lane] = RpRow{there, CACHE ? g.slots[(size_t)seq * g.T + i] : -1};
#pragma unroll
            for (int x = 0; x < 4; ++x) s_pos[x][lane] = (int64_t)ctx + (g.positions ? position[x] : i);
        }
    }
    __syncthreads();

    if constexpr (CACHE) {
        if (is_v) {
            // ---- v: along the rows where they are read, down the eight rows where they are stored (they lie side by side in the cache)
            using C = KvqChunk<D0>;
            const int row_out = l % 8, piece_out = part + l % kWave / 8, turn = l % 8 * 8 + l % kWave / 8;
            const RpRow to = s_row[row_out];
            const bool stored = to.there && to.slot >= 0 && to.slot < g.total;
            const int R = 1 << g.rbits, slot_row = stored ? to.slot & (R - 1) : 0;
            unsigned char *const block = g.cache + (size_t)(stored ? to.slot >> g.rbits : 0) * g.Hkv * C::bytes(R);
            for (int x = 0; x < rounds; ++x) {
                const int h = h0 + x * V_HEADS;            // (the same in the whole wavefront)
                if (h >= g.Hkv) break;
                const uint32_t w0 = a[0], w1 = a[1], w2 = a[2], w3 = a[3];
                if (x + 1 < rounds) ask(h + V_HEADS);
                const KvqCodes c = kvq_encode8(w0, w1, w2, w3);
                const uint32_t code = (uint32_t)__shfl((int)c.code, turn), mark = (uint32_t)__shfl((int)c.mark, turn);
                if (!stored) continue;
                unsigned char *const chunk = block + (size_t)h * C::bytes(R);
                *reinterpret_cast<uint32_t *>(chunk + C::v_piece(R, slot_row, piece_out)) = code;
                if ((piece_out & 3) == 0) chunk[C::v_scale(R, slot_row, piece_out >> 2)] = (unsigned char)mark;
            }
            return;
        }
    }

    // ---- sines and cosines of eight rows
    for (int x = tid; x < kRpRows * g.pairs; x += kRpThreads) {
        const int row = x / g.pairs, j = x - row * g.pairs;
        const int axis = (int)(g.axis[j >> 5] >> (2 * (j & 31))) & 3;
        double s, c;
        rp_sin_cos((double)s_pos[axis][row] * (double)g.inv_freq[j], &s, &c);
        s_cs[(row * 8 + (j & 7)) * LP + (j >> 3)] = double2{c * g.scale, s * g.scale};
    }
    __syncthreads();
    double c[8], s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const double2 cs = s_cs[(row * 8 + e) * LP + (at.turned ? p : 0)];
        c[e] = cs.x;
        s[e] = cs.y;
    }
    const bool there = s_row[row].there != 0;

    if (!CACHE || is_q) {
        // ---- rows of q, or of k that go out as rows
        if (!there || place >= heads) return;
        const int64_t out_h = is_q ? g.qo_sh : g.ko_sh;
        __bf16 *const to = (is_q ? g.q_out : g.k_out) + n * (is_q ? g.qo_sn : g.ko_sn);
        for (int x = 0; x < rounds; ++x) {
            const int h = h0 + x * heads;
            if (h >= H) return;
            u32x4 o = a, z = b;
            if (x + 1 < rounds) ask(h + heads);
            if (at.turned) rp_turn(o, z, c, s, g.adjacent != 0);
            rp_store<STREAM>(to + h * out_h + at.a * 8, o);
            rp_store<STREAM>(to + h * out_h + at.b * 8, z);
        }
    } else if constexpr (CACHE) {
        // ---- k: turned into LDS, and from there along the rows into the cache
        using C = KvqChunk<D0>;
        constexpr int PIECES = D0 / 8;
        for (int x = 0; x < rounds; ++x) {
            const int first = h0 - place + x * heads;
            if (first >= g.Hkv) return;                    // (the same for the whole workgroup)
            u32x4 o = a, z = b;
            if (x + 1 < rounds) ask(first + place + heads);
            if (at.turned) rp_turn(o, z, c, s, g.adjacent != 0);
            if (x > 0) __syncthreads();
            s_k[(place * kRpRows + row) * PIECES + at.a] = o;
            s_k[(place * kRpRows + row) * PIECES + at.b] = z;
            __syncthreads();
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int i = tid + u * kRpThreads, piece = i % PIECES, r2 = i / PIECES % kRpRows, h2 = first + i / (PIECES * kRpRows);
                const u32x4 w = s_k[i];
                const uint32_t w0 = w[0], w1 = w[1], w2 = w[2], w3 = w[3];
                const KvqCodes e = kvq_encode8(w0, w1, w2, w3);
                const RpRow to = s_row[r2];
                if (!to.there || to.slot < 0 || to.slot >= g.total || h2 >= g.Hkv) continue;
                const int R = 1 << g.rbits, row2 = to.slot & (R - 1);
                unsigned char *const chunk = g.cache + ((size_t)(to.slot >> g.rbits) * g.Hkv + h2) * C::bytes(R);
                *reinterpret_cast<uint32_t *>(chunk + C::k_row(row2) + piece * 4) = e.code;
                if ((piece & 3) == 0) chunk[C::k_scale(R, row2, piece >> 2)] = (unsigned char)e.mark;
            }
        }
    }
}

}  // namespace radar

using namespace radar;

// What both calls check of a descriptor and their pointers, and the kernel's arguments but for the cache.
static radar_status rope_args(const void *q, const void *k, const void *v, void *q_out, void *k_out, const float *inv_freq, const int32_t *positions,
                              const int32_t *ctx_lens, const int32_t *row_starts, const int32_t *n_new, const radar_rope_desc *d, RpArgs *g) {
    if (!d || !inv_freq || (q != nullptr) != (q_out != nullptr)) return RADAR_INVALID_ARG;
    if (d->B < 1 || d->T_max < 1 || d->N < 0 || d->D < 1 || d->rotary_dim < 0 || d->axes < 1 || (row_starts && n_new)) return RADAR_INVALID_ARG;
    if (!row_starts && d->N != (int64_t)d->B * d->T_max) return RADAR_INVALID_ARG;
    if ((q && d->Hq < 1) || (k && d->Hkv < 1) || !std::isfinite(d->scale) || (d->interleaved != 0 && d->interleaved != 1)) return RADAR_INVALID_ARG;
    const int rotary = d->rotary_dim ? d->rotary_dim : d->D;
    if (rotary > d->D) return RADAR_INVALID_ARG;
    if (d->D % 16 != 0 || d->D > 256 || rotary % 16 != 0 || d->axes > 4 || d->N > INT32_MAX || d->Hq > 65535 || d->Hkv > 65535 || d->B > kRpSequences) return RADAR_UNSUPPORTED_SHAPE;
    g->pairs = rotary / 2;
    for (int j = 0; j < g->pairs; ++j) {
        if (d->pair_axis[j] >= d->axes) return RADAR_INVALID_ARG;
        g->axis[j >> 5] |= (uint64_t)d->pair_axis[j] << (2 * (j & 31));
    }
    g->q = static_cast<const __bf16 *>(q); g->k = static_cast<const __bf16 *>(k); g->v = static_cast<const __bf16 *>(v);
    g->q_out = static_cast<__bf16 *>(q_out); g->k_out = static_cast<__bf16 *>(k_out);
    g->inv_freq = inv_freq; g->positions = positions; g->ctx_lens = ctx_lens; g->row_starts = row_starts; g->n_new = n_new;
    g->N = d->N; g->B = d->B; g->T = d->T_max; g->Hq = q ? d->Hq : 0; g->Hkv = k ? d->Hkv : 0; g->D = d->D; g->axes = d->axes; g->adjacent = d->interleaved;
    g->scale = d->scale == 0.f ? 1.0 : (double)d->scale;
    const int64_t D = d->D;
    auto or_dense = [](int64_t s, int64_t dense) { return s ? s : dense; };
    g->q_sh = or_dense(d->q_stride_h, D); g->q_sn = or_dense(d->q_stride_n, D * d->Hq);
    g->kv_sh = or_dense(d->kv_stride_h, D); g->kv_sn = or_dense(d->kv_stride_n, D * d->Hkv);
    g->qo_sh = or_dense(d->q_out_stride_h, D); g->qo_sn = or_dense(d->q_out_stride_n, D * d->Hq);
    g->ko_sh = or_dense(d->k_out_stride_h, D); g->ko_sn = or_dense(d->k_out_stride_n, D * d->Hkv);
    // in place: the same rows
    if (q && q == q_out && (g->q_sh != g->qo_sh || g->q_sn != g->qo_sn)) return RADAR_INVALID_ARG;
    if (k && k == k_out && (g->kv_sh != g->ko_sh || g->kv_sn != g->ko_sn)) return RADAR_INVALID_ARG;
    const int64_t all[] = {g->q_sh, g->q_sn, g->kv_sh, g->kv_sn, g->qo_sh, g->qo_sn, g->ko_sh, g->ko_sn};
    for (int64_t s : all)
        if (s < 0 || (s & 7) != 0) return RADAR_INVALID_ARG;
    if ((((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_out | (uintptr_t)k_out) & 15) != 0) return RADAR_INVALID_ARG;
    return RADAR_OK;
}

static bool rope_streams(const RpArgs &g) { return g.N * g.D * 2 * (2 * g.Hq + 2 * g.Hkv) > kRpStream; }

// Heads are dealt to workgroups so that few rows still fill the chip; many rows keep all heads of their kind in one, which works out the angles once.
static radar_status launch_rope(const char *name, void (*kernel)(RpArgs), RpArgs &g, hipStream_t s) {
    const int64_t groups = (g.N + kRpRows - 1) / kRpRows;
    const int turned = kRpThreads / (kRpRows * (g.D / 16)), plain = kRpThreads / g.D;          // heads of a round: turned, and v's
    auto rounds = [](int H, int heads) { return heads > 0 ? (H + heads - 1) / heads : 0; };
    const int q = rounds(g.Hq, turned), k = rounds(g.Hkv, turned), v = g.cache ? rounds(g.Hkv, plain) : 0;
    const int most = (int)std::min<int64_t>(std::max<int64_t>(groups * (q + k + v) / kRpGroups, 1), 8);
    auto deal = [&](int n, int *per) { *per = std::min(most, std::max(n, 1)); return (n + *per - 1) / *per; };
    g.q_blocks = deal(q, &g.per_q);
    g.k_blocks = deal(k, &g.per_k);
    const int v_blocks = deal(v, &g.per_v);
    const int64_t blocks = g.q_blocks + g.k_blocks + v_blocks;
    if (blocks > 65535 || groups * blocks >= (1 << 24)) return RADAR_UNSUPPORTED_SHAPE;          // (a launch has less than 2^32 lanes)
    return launch(name, kernel, dim3((unsigned)groups, (unsigned)blocks), dim3(kRpThreads), 0, s, g) == hipSuccess ? RADAR_OK : RADAR_HIP_ERROR;
}

extern "C" radar_status radar_rope(const void *q, const void *k, void *q_out, void *k_out, const float *inv_freq, const int32_t *positions,
                                   const int32_t *ctx_lens, const int32_t *row_starts, const int32_t *n_new, const radar_rope_desc *d, void *stream) {
    if ((k != nullptr) != (k_out != nullptr) || (!q && !k)) return RADAR_INVALID_ARG;
    RpArgs g{};
    const radar_status st = rope_args(q, k, nullptr, q_out, k_out, inv_freq, positions, ctx_lens, row_starts, n_new, d, &g);
    if (st != RADAR_OK || g.N == 0) return st;
    const auto kernel = rope_streams(g) ? (g.D == 128 ? rope_kernel<128, false, true> : g.D == 64 ? rope_kernel<64, false, true> : rope_kernel<0, false, true>)
                                        : (g.D == 128 ? rope_kernel<128, false, false> : g.D == 64 ? rope_kernel<64, false, false> : rope_kernel<0, false, false>);
    return launch_rope("rope", kernel, g, static_cast<hipStream_t>(stream));
}

extern "C" radar_status radar_kvq_append_rope(const void *q, const void *k, const void *v, void *q_out, const float *inv_freq, const int32_t *positions,
                                              const int32_t *ctx_lens, const int32_t *row_starts, const int32_t *n_new, const int32_t *slots, void *cache,
                                              const radar_rope_desc *d, const radar_kvq_desc *c, void *stream) {
    if (!k || !v || !slots || !cache || !d) return RADAR_INVALID_ARG;
    radar_status st = kvq_check(c);
    if (st != RADAR_OK) return st;
    if (d->D != c->D || d->Hkv != c->Hkv || ((uintptr_t)cache & 15) != 0) return RADAR_INVALID_ARG;
    RpArgs g{};
    st = rope_args(q, k, v, q_out, nullptr, inv_freq, positions, ctx_lens, row_starts, n_new, d, &g);
    if (st != RADAR_OK || g.N == 0) return st;
    g.slots = slots; g.cache = static_cast<unsigned char *>(cache);
    g.total = (int64_t)c->n_blocks * c->block_rows; g.rbits = kvq_log2(c->block_rows);
    const auto kernel = rope_streams(g) ? (g.D == 128 ? rope_kernel<128, true, true> : rope_kernel<64, true, true>)
                                        : (g.D == 128 ? rope_kernel<128, true, false> : rope_kernel<64, true, false>);
    return launch_rope("kvq_append_rope", kernel, g, static_cast<hipStream_t>(stream));
}
