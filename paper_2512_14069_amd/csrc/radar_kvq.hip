// The paged key/value cache in 4 bits: block tables and slot maps, writing rows, reading them back, and moving
// the accepted path's rows into place (attention over it: radar_kvq_attention.hip).
#include <algorithm>

#include "radar_host.h"
#include "radar_kvq.h"

namespace radar {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ===================================================================== block tables and slot maps
// One workgroup: what every sequence gives back or takes is a prefix sum over the batch, and a batch's tables
// are a few kilobytes.  A lane works out one sequence's two numbers; the entries that move are counted through
// and dealt to the lanes one by one (a lane finds its sequence by bisection of the sums in LDS), so that a sequence
// that ends with hundreds of blocks takes as long as hundreds that give back one.  What bounds it is a chain of round trips (heights and lengths, the
// stack, the tables): 16 sequences 4.9 us, 1024 of which 64 have ended 6.8 and 4 for the slots.
constexpr int kBlThreads = 1024;
// Up to so many slots the same launch maps them (us, in it and in a launch of their own: 960 slots 4.2, 5.8; 3840 5.0, 6.4; 8192 6.7, 6.2; 16384 9.6, 6.3;
// 131072 51, 6.2).
constexpr int64_t kSlotsInline = 4096;

struct BlArgs {
    const int32_t *ctx_lens, *n_new;
    int32_t *tables;
    const int32_t *owned;
    int32_t *free_blocks;
    const int32_t *n_free;
    int32_t *owned_out, *n_free_out, *slots, *granted;
    int B, T, M, n_blocks, rbits;
    int map;                                // whether this launch writes the slots
};

struct BlSeq { int want, owned; bool fits; };

__device__ __forceinline__ int bl_new_rows(const BlArgs &a, int b) { return a.n_new ? min(max(a.n_new[b], 0), a.T) : a.T; }

__device__ __forceinline__ BlSeq bl_seq(const BlArgs &a, int b) {
    BlSeq s{0, 0, true};
    if (b >= a.B) return s;
    const int ctx = a.ctx_lens[b];
    s.owned = min(max(a.owned[b], 0), a.M);
    const int64_t w = ctx < 0 ? 0 : ((int64_t)ctx + bl_new_rows(a, b) + (1 << a.rbits) - 1) >> a.rbits;
    s.fits = w <= a.M;
    s.want = s.fits ? (int)w : s.owned;                            // refused: gives and takes nothing
    return s;
}

// Exclusive prefix sum over the workgroup's lanes, and their total.  All lanes call.
__device__ __forceinline__ uint32_t bl_scan(uint32_t v, uint32_t *waves, uint32_t *total) {
    const uint32_t incl = wave_scan_u32(v);
    if (lane_id() == kWave - 1) waves[wave_id()] = incl;
    __syncthreads();
    uint32_t before = 0, all = 0;
    for (int w = 0; w < kBlThreads / kWave; ++w) {
        if (w == wave_id()) before = all;
        all += waves[w];
    }
    __syncthreads();
    *total = all;
    return before + incl - v;
}

// The last of the chunk's sequences whose first item is at or before `item`, among those that have any.
__device__ __forceinline__ int bl_owner(const uint32_t *first, uint32_t item) {
    int lo = 0;
#pragma unroll
    for (int step = kBlThreads / 2; step > 0; step >>= 1)
        if (first[lo + step] <= item) lo += step;
    return lo;
}

__device__ __forceinline__ int bl_slot(const BlArgs &a, int b, int i, int ctx) {
    const int64_t pos = (int64_t)ctx + i;
    const int block = a.tables[(size_t)b * a.M + (pos >> a.rbits)];
    return (uint32_t)block < (uint32_t)a.n_blocks ? (block << a.rbits) + (int)(pos & ((1 << a.rbits) - 1)) : -1;
}

__global__ __launch_bounds__(kBlThreads) void kvq_blocks_kernel(BlArgs a) {
    __shared__ uint32_t first[kBlThreads];     // number of a sequence's first item that moves
    __shared__ int from[kBlThreads];           // its first table entry that moves
    __shared__ uint32_t waves[kBlThreads / kWave];
    const int tid = threadIdx.x;
    const int height = min(max(*a.n_free, 0), a.n_blocks);

    uint32_t given = 0;                        // by the chunks before
    for (int b0 = 0; b0 < a.B; b0 += kBlThreads) {
        const BlSeq s = bl_seq(a, b0 + tid);
        uint32_t total;
        first[tid] = bl_scan((uint32_t)max(s.owned - s.want, 0), waves, &total);
        from[tid] = s.want;
        __syncthreads();
        for (uint32_t t = tid; t < total; t += kBlThreads) {
            const int q = bl_owner(first, t);
            const int64_t to = (int64_t)height + given + t;       // (a stack that overflows has been given blocks twice)
            if (to < a.n_blocks) a.free_blocks[to] = a.tables[(size_t)(b0 + q) * a.M + from[q] + (t - first[q])];
        }
        given += total;
        __syncthreads();
    }
    const int64_t there = min((int64_t)height + given, (int64_t)a.n_blocks);

    int64_t asked = 0, taken = 0;              // by the chunks before; the same in every lane
    for (int b0 = 0; b0 < a.B; b0 += kBlThreads) {
        const int b = b0 + tid;
        const BlSeq s = bl_seq(a, b);
        const uint32_t need = (uint32_t)max(s.want - s.owned, 0);
        uint32_t total, got;
        const uint32_t before = bl_scan(need, waves, &total);
        const bool granted = s.fits && (need == 0 || asked + before + need <= there);
        // (what is granted is the first part of what is asked for: nothing behind a sequence that was refused for want of blocks)
        first[tid] = bl_scan(granted ? need : 0u, waves, &got);
        from[tid] = s.owned;
        __syncthreads();
        for (uint32_t t = tid; t < got; t += kBlThreads) {
            const int q = bl_owner(first, t);
            a.tables[(size_t)(b0 + q) * a.M + from[q] + (t - first[q])] = a.free_blocks[there - 1 - taken - t];
        }
        if (b < a.B) {
            a.owned_out[b] = granted ? s.want : s.owned;
            a.granted[b] = granted;
        }
        // A refused sequence's entries behind the owned ones go: they may name blocks that it gave back and others hold by now, and the
        // pass's later calls, which know of no refusal, would follow them to the rows that it asked for.
        for (uint64_t refused = __ballot(b < a.B && !granted); refused != 0; refused &= refused - 1) {
            const int src = __ffsll((unsigned long long)refused) - 1;
            int32_t *const table = a.tables + (size_t)(b0 + wave_id() * kWave + src) * a.M;
            for (int i = __shfl(s.owned, src) + lane_id(); i < a.M; i += kWave) table[i] = -1;
        }
        asked += total;
        taken += got;
        __syncthreads();
        if (a.map) {                           // this chunk's slots, from the entries just written
            from[tid] = granted && b < a.B && a.ctx_lens[b] >= 0 ? bl_new_rows(a, b) : 0;
            __syncthreads();
            const int items = min(kBlThreads, a.B - b0) * a.T;
            for (int t = tid; t < items; t += kBlThreads) {
                const int q = t / a.T, i = t - q * a.T;
                a.slots[(size_t)b0 * a.T + t] = i < from[q] ? bl_slot(a, b0 + q, i, a.ctx_lens[b0 + q]) : -1;
            }
            __syncthreads();
        }
    }
    if (tid == 0) *a.n_free_out = (int)(there - taken);
}

// The slots of many rows (a batch's prompts), after the tables are there.
__global__ __launch_bounds__(256) void kvq_slots_kernel(BlArgs a) {
    const int64_t items = (int64_t)a.B * a.T, step = (int64_t)gridDim.x * 256;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < items; t += step) {
        const int b = (int)(t / a.T), i = (int)(t - (int64_t)b * a.T), ctx = a.ctx_lens[b];
        a.slots[t] = a.granted[b] && ctx >= 0 && i < bl_new_rows(a, b) ? bl_slot(a, b, i, ctx) : -1;
    }
}

// ===================================================================== rows into the cache and out of it
// Eight rows of the input and one head take 2 * D lanes: the first half of them K, the other V, a lane eight values (16
// bytes of bf16, 4 of codes).  All go along the rows where they touch values, and so do lanes of K at the codes, which lie in one piece; there lanes
// of V go down the eight rows, whose codes of the same eight values lie side by side: where the rows follow each other in the cache (prompts, trees)
// all store and load whole lines.  A word and a scale change lanes between the two orders.
constexpr int kRwThreads = 256, kRwGroups = 2048, kRwLayers = 4;

struct RwArgs {
    const __bf16 *k, *v;                       // append: rows in;
    __bf16 *k_out, *v_out;                     // read: rows out, [layers][N][Hkv][D]
    const int32_t *slots;
    unsigned char *cache;
    int64_t N, stride_n, stride_h, layer_stride, total;   // total: slots of the cache
    int rbits, Hkv, layers, per;               // read: layers, and those of a workgroup
};

template <int D>
struct RwLane {                                // which eight values a lane has
    int64_t n;                                 // row of the input
    int h, row8, piece;
    bool is_v;
};
// down: a wavefront's lanes of V go down the rows, as the codes lie; otherwise along them, as the values do.
template <int D>
__device__ __forceinline__ RwLane<D> rw_lane(int Hkv, bool down) {
    constexpr int P = D / 8, HALF = 8 * P;     // lanes of K, of V
    const uint32_t unit = blockIdx.x * (kRwThreads / (2 * HALF)) + threadIdx.x / (2 * HALF), group = unit / (uint32_t)Hkv;      // (of a grid of less than 2^24)
    const int l = threadIdx.x % (2 * HALF), l2 = l % HALF;
    RwLane<D> r;
    r.is_v = l >= HALF;
    r.row8 = !r.is_v ? l2 / P : down ? l2 % 8 : l2 % 64 / 8;
    r.piece = !r.is_v ? l2 % P : l2 / 64 * 8 + (down ? l2 % 64 / 8 : l2 % 8);
    r.h = (int)(unit - group * (uint32_t)Hkv);
    r.n = (int64_t)group * 8 + r.row8;
    return r;
}
// What the lane has that is this one's counterpart in the other order (K: itself).
__device__ __forceinline__ uint32_t rw_turned(bool is_v, uint32_t x) {
    const int l = lane_id();
    return (uint32_t)__shfl((int)x, is_v ? l % 8 * 8 + l / 8 : l);
}

template <int D>
__global__ __launch_bounds__(kRwThreads) void kvq_append_kernel(RwArgs a) {
    using C = KvqChunk<D>;
    const RwLane<D> in = rw_lane<D>(a.Hkv, false), r = rw_lane<D>(a.Hkv, true);
    const int64_t n = min(in.n, a.N - 1);      // (lanes past the end go along: the maximum is taken over whole wavefronts)
    const int slot = a.slots[min(r.n, a.N - 1)];
    const u32x4 x = *reinterpret_cast<const u32x4 *>((in.is_v ? a.v : a.k) + n * a.stride_n + in.h * a.stride_h + in.piece * 8);
    const uint32_t x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];      // (a bit cast of a vector's element would take its first)
    const KvqCodes c = kvq_encode8(x0, x1, x2, x3);
    const uint32_t code = rw_turned(in.is_v, c.code), mark = rw_turned(in.is_v, c.mark);
    if (r.n >= a.N || slot < 0 || slot >= a.total) return;
    const int R = 1 << a.rbits, row = slot & (R - 1);
    unsigned char *const chunk = a.cache + ((size_t)(slot >> a.rbits) * a.Hkv + r.h) * C::bytes(R);
    *reinterpret_cast<uint32_t *>(chunk + (r.is_v ? C::v_piece(R, row, r.piece) : C::k_row(row) + r.piece * 4)) = code;
    if ((r.piece & 3) == 0) chunk[r.is_v ? C::v_scale(R, row, r.piece >> 2) : C::k_scale(R, row, r.piece >> 2)] = (unsigned char)mark;
}

// A workgroup reads its rows in `per` layers, U at a time: where a row is in a layer is worked out once (80 layers of 576 rows of 8 heads, 188 MB of
// outputs: 53 us with four layers, 66 with one; 8191 rows of one layer 9.2).  The outputs are stored past the caches: kept there they push out what the
// next kernel needs (a commit after such a read 44 us, 61 with ordinary stores), and the 8191 rows take 10.3 us.
template <int D, int U>
__global__ __launch_bounds__(kRwThreads) void kvq_read_kernel(RwArgs a) {
    using C = KvqChunk<D>;
    const RwLane<D> r = rw_lane<D>(a.Hkv, true), out = rw_lane<D>(a.Hkv, false);
    const int slot = a.slots[min(r.n, a.N - 1)], first = blockIdx.y * a.per, last = min(first + a.per, a.layers) - 1;
    const bool there = slot >= 0 && slot < a.total;
    const int R = 1 << a.rbits, row = there ? slot & (R - 1) : 0;
    const unsigned char *const chunk = a.cache + ((size_t)(there ? slot >> a.rbits : 0) * a.Hkv + r.h) * C::bytes(R);
    const unsigned char *const code = chunk + (r.is_v ? C::v_piece(R, row, r.piece) : C::k_row(row) + r.piece * 4);
    const unsigned char *const scale = chunk + (r.is_v ? C::v_scale(R, row, r.piece >> 2) : C::k_scale(R, row, r.piece >> 2));
    __bf16 *const to = (r.is_v ? a.v_out : a.k_out) + ((size_t)out.n * a.Hkv + r.h) * D + out.piece * 8;
    const size_t out_stride = (size_t)a.N * a.Hkv * D;
    for (int l0 = first; l0 <= last; l0 += U) {
        uint32_t w[U], byte[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const size_t at = (size_t)min(l0 + u, last) * a.layer_stride;
            w[u] = there ? *reinterpret_cast<const uint32_t *>(code + at) : 0u;
            byte[u] = there ? scale[at] : 0u;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (l0 + u > last) break;
            uint32_t o[4];
            kvq_decode8(rw_turned(r.is_v, w[u]), kvq_scale(rw_turned(r.is_v, byte[u])), o);
            if (out.n < a.N) __builtin_nontemporal_store(u32x4{o[0], o[1], o[2], o[3]}, reinterpret_cast<u32x4 *>(to + (size_t)(l0 + u) * out_stride));
        }
    }
}

// ===================================================================== the accepted path's rows into place
// Rows move as they are: D/4 words of codes, a word a lane, and the scales' bytes.  A wavefront finds out once where its lanes' words of one
// sequence's rows come from and go to (length, path, table: a chain of round trips), and then moves them in `per` pairs of layer and head: four at a
// time for the usual path of at most eight rows, one at a time for longer ones.  All of a pair's rows are read before its first is written, so any
// path is right.  64 sequences in 80 layers of 8 heads: 44 us (a pair a wavefront, words dealt along the rows: 64); one sequence in 32 layers 4.3.
constexpr int kCmThreads = 256, kCmWaves = 4096, kCmQuick = 8;

struct CmArgs {
    unsigned char *cache;
    const int32_t *tables, *ctx_lens, *accept_len, *accept_path;
    int32_t *new_ctx;
    int64_t layer_stride;
    int M, P, rbits, Hkv, units, n_blocks, per;        // units: layers * Hkv; per: of a wavefront
};

template <int D>
__global__ __launch_bounds__(kCmThreads) void kvq_commit_kernel(CmArgs a) {
    using C = KvqChunk<D>;
    constexpr int W = D / 4, PER = kWave / W;   // words of codes of a row, K and V; rows that a wavefront's load covers
    constexpr int S = 2 * (D / 32);             // scale bytes of a row
    const int b = blockIdx.y, first = (blockIdx.x * (kCmThreads / kWave) + wave_id()) * a.per, last = min(first + a.per, a.units) - 1, lane = lane_id();
    const int ctx = a.ctx_lens[b];
    const int n = ctx < 0 ? 0 : min(max(a.accept_len[b], 0), a.P - 1);
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.new_ctx) a.new_ctx[b] = ctx < 0 ? ctx : (int)min((int64_t)ctx + n + 1, (int64_t)INT32_MAX);
    if (n == 0 || first > last) return;
    const int R = 1 << a.rbits;
    const int64_t rows = (int64_t)a.M << a.rbits;
    auto base_of = [&](int unit) {
        const int layer = unit / a.Hkv, h = unit - layer * a.Hkv;
        return a.cache + (size_t)layer * a.layer_stride + (size_t)h * C::bytes(R);
    };

    // Lane s knows where row s goes from and to: its block's bytes from a layer's first, and the row in it; from < 0: it stays.
    int64_t from = -1, to = -1;
    int from_row = 0, to_row = 0;
    if (lane >= 1 && lane <= n) {
        const int p = a.accept_path[(size_t)b * a.P + lane];
        const int64_t src = (int64_t)ctx + p, dst = (int64_t)ctx + lane;
        if (p >= 0 && p < RADAR_T_MAX && p != lane && src < rows && dst < rows) {
            const int bs = a.tables[(size_t)b * a.M + (src >> a.rbits)], bd = a.tables[(size_t)b * a.M + (dst >> a.rbits)];
            if ((uint32_t)bs < (uint32_t)a.n_blocks && (uint32_t)bd < (uint32_t)a.n_blocks) {
                from = (int64_t)bs * a.Hkv * C::bytes(R); from_row = (int)(src & (R - 1));
                to = (int64_t)bd * a.Hkv * C::bytes(R); to_row = (int)(dst & (R - 1));
            }
        }
    }
    auto at64 = [](int64_t v, int s) {
        return (int64_t)((uint64_t)(uint32_t)__shfl((int)(uint32_t)v, s) | (uint64_t)(uint32_t)__shfl((int)(uint32_t)((uint64_t)v >> 32), s) << 32);
    };
    const int wi = lane % W;                    // this lane's word of a row: K's first, then V's eights
    auto code_at = [&](int row) { return wi < W / 2 ? C::k_row(row) + wi * 4 : C::v_piece(R, row, wi - W / 2); };
    const int si = lane % S;
    auto scale_at = [&](int row) { return si < S / 2 ? C::k_scale(R, row, si) : C::v_scale(R, row, si - S / 2); };

    if (n <= kCmQuick) {
        // Words and rows a load: K's along its rows, V's and the scales down the rows, whose words of the same values are neighbours in the cache.
        constexpr int KL = D / 64, ITEMS = 2 * KL, U = 4;
        static_assert(kCmQuick * D / 8 == KL * kWave && kCmQuick * S <= kWave);
        int64_t src[ITEMS + 1], dst[ITEMS + 1];                      // of this lane's words and its scale, < 0: there is none
#pragma unroll
        for (int i = 0; i <= ITEMS; ++i) {
            const int row = i < KL ? (i * kWave + lane) / (D / 8) : lane % 8;
            const bool mine = i < ITEMS || lane / 8 < S;
            src[i] = at64(from, 1 + row); dst[i] = at64(to, 1 + row);              // (lanes behind the path know of no row)
            const int fr = __shfl(from_row, 1 + row), tr = __shfl(to_row, 1 + row);
            auto in_chunk = [&](int r) {
                if (i < KL) return C::k_row(r) + lane % (D / 8) * 4;
                if (i < ITEMS) return C::v_piece(R, r, (i - KL) * 8 + lane / 8);
                return lane / 8 < S / 2 ? C::k_scale(R, r, lane / 8) : C::v_scale(R, r, lane / 8 - S / 2);
            };
            if (!mine) src[i] = -1;
            if (src[i] >= 0) { src[i] += in_chunk(fr); dst[i] += in_chunk(tr); }
        }
        for (int u0 = first; u0 <= last; u0 += U) {
            uint32_t word[U][ITEMS];
            unsigned char scale[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const unsigned char *const base = base_of(min(u0 + u, last));
#pragma unroll
                for (int i = 0; i < ITEMS; ++i) word[u][i] = src[i] >= 0 ? *reinterpret_cast<const uint32_t *>(base + src[i]) : 0u;
                scale[u] = src[ITEMS] >= 0 ? base[src[ITEMS]] : (unsigned char)0;
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // every row has been read
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u0 + u > last) break;
                unsigned char *const base = base_of(u0 + u);
#pragma unroll
                for (int i = 0; i < ITEMS; ++i)
                    if (src[i] >= 0) *reinterpret_cast<uint32_t *>(base + dst[i]) = word[u][i];
                if (src[ITEMS] >= 0) base[dst[ITEMS]] = scale[u];
            }
        }
        return;
    }

    constexpr int ITEMS = RADAR_T_MAX / PER, BYTES = RADAR_T_MAX * S / kWave;
    for (int unit = first; unit <= last; ++unit) {
        unsigned char *const base = base_of(unit);
        int m = n;
        asm volatile("" : "+v"(m));            // (in each pass anew: what comes of comparing it would be kept for the loop, in more scalars than there are)
        m = __builtin_amdgcn_readfirstlane(m);
        uint32_t word[ITEMS];
        unsigned char scale[BYTES];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            word[i] = 0;
            if (1 + i * PER <= m) {             // the same in every lane
                const int s = min(1 + i * PER + lane / W, kWave - 1);
                const int64_t f = at64(from, s);
                const int row = __shfl(from_row, s);
                if (f >= 0) word[i] = *reinterpret_cast<const uint32_t *>(base + f + code_at(row));
            }
        }
#pragma unroll
        for (int i = 0; i < BYTES; ++i) {
            scale[i] = 0;
            if (1 + i * (kWave / S) <= m) {
                const int s = min(1 + i * (kWave / S) + lane / S, kWave - 1);
                const int64_t f = at64(from, s);
                const int row = __shfl(from_row, s);
                if (f >= 0) scale[i] = base[f + scale_at(row)];
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // every row has been read
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (1 + i * PER <= m) {
                const int s = 1 + i * PER + lane / W;
                const int64_t t = at64(to, min(s, kWave - 1));
                const int row = __shfl(to_row, min(s, kWave - 1));
                if (s <= m && t >= 0) *reinterpret_cast<uint32_t *>(base + t + code_at(row)) = word[i];
            }
        }
#pragma unroll
        for (int i = 0; i < BYTES; ++i) {
            if (1 + i * (kWave / S) <= m) {
                const int s = 1 + i * (kWave / S) + lane / S;
                const int64_t t = at64(to, min(s, kWave - 1));
                const int row = __shfl(to_row, min(s, kWave - 1));
                if (s <= m && t >= 0) base[t + scale_at(row)] = scale[i];
            }
        }
    }
}

}  // namespace radar

using namespace radar;

extern "C" size_t radar_kvq_block_bytes(int32_t block_rows, int32_t D) {
    radar_kvq_desc d{};
    d.n_blocks = d.Hkv = 1;
    d.block_rows = block_rows;
    d.D = D;
    return kvq_check(&d) == RADAR_OK ? (size_t)block_rows * (D + D / 16) : 0;
}

extern "C" radar_status radar_kvq_blocks(const int32_t *ctx_lens, const int32_t *n_new, int32_t *block_tables, const int32_t *owned,
                                         int32_t *free_blocks, const int32_t *n_free, int32_t *owned_out, int32_t *n_free_out, int32_t *slots,
                                         int32_t *granted, const radar_kvq_blocks_desc *d, void *stream) {
    if (!ctx_lens || !block_tables || !owned || !free_blocks || !n_free || !owned_out || !n_free_out || !slots || !granted || !d) return RADAR_INVALID_ARG;
    if (d->B < 1 || d->T_max < 1 || d->max_blocks < 1 || d->n_blocks < 1) return RADAR_INVALID_ARG;
    radar_kvq_desc c{};
    c.n_blocks = d->n_blocks; c.block_rows = d->block_rows; c.Hkv = 1; c.D = 64;
    const radar_status st = kvq_check(&c);
    if (st != RADAR_OK) return st;
    // what all sequences ask for or give back is counted in 32 bits
    if ((int64_t)d->B * d->max_blocks > INT32_MAX || (int64_t)d->B * d->T_max > INT32_MAX) return RADAR_UNSUPPORTED_SHAPE;
    BlArgs a{ctx_lens, n_new, block_tables, owned, free_blocks, n_free, owned_out, n_free_out, slots, granted,
             d->B, d->T_max, d->max_blocks, d->n_blocks, kvq_log2(d->block_rows), 0};
    a.map = (int64_t)d->B * d->T_max <= kSlotsInline;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = launch("kvq_blocks", kvq_blocks_kernel, dim3(1), dim3(kBlThreads), 0, s, a);
    if (e == hipSuccess && !a.map) {
        const int64_t groups = ((int64_t)d->B * d->T_max + 255) / 256;
        e = launch("kvq_slots", kvq_slots_kernel, dim3((unsigned)std::min<int64_t>(groups, 2048)), dim3(256), 0, s, a);
    }
    return e == hipSuccess ? RADAR_OK : RADAR_HIP_ERROR;
}

// What append and read share: arguments and grid.
static radar_status rw_args(const void *k, const void *v, const int32_t *slots, const void *cache, int64_t N, const radar_kvq_desc *d, RwArgs *a, int64_t *groups) {
    if (!k || !v || !slots || !cache || N < 0) return RADAR_INVALID_ARG;
    const radar_status st = kvq_check(d);
    if (st != RADAR_OK) return st;
    if ((((uintptr_t)k | (uintptr_t)v | (uintptr_t)cache) & 15) != 0) return RADAR_INVALID_ARG;
    a->slots = slots; a->N = N; a->total = (int64_t)d->n_blocks * d->block_rows;
    a->cache = static_cast<unsigned char *>(const_cast<void *>(cache));
    a->rbits = kvq_log2(d->block_rows); a->Hkv = d->Hkv;
    const int units = kRwThreads / (2 * d->D);
    if (N > (int64_t)INT32_MAX) return RADAR_UNSUPPORTED_SHAPE;
    *groups = ((N + 7) / 8 * d->Hkv + units - 1) / units;
    return *groups < (1 << 24) ? RADAR_OK : RADAR_UNSUPPORTED_SHAPE;               // (a launch has less than 2^32 lanes)
}

extern "C" radar_status radar_kvq_append(const void *k, const void *v, const int32_t *slots, void *cache, int64_t N, int64_t stride_n, int64_t stride_h,
                                         const radar_kvq_desc *d, void *stream) {
    RwArgs a{};
    int64_t groups;
    const radar_status st = rw_args(k, v, slots, cache, N, d, &a, &groups);
    if (st != RADAR_OK) return st;
    a.k = static_cast<const __bf16 *>(k); a.v = static_cast<const __bf16 *>(v);
    a.stride_h = stride_h ? stride_h : d->D;
    a.stride_n = stride_n ? stride_n : (int64_t)d->D * d->Hkv;
    if (a.stride_n < 0 || a.stride_h < 0 || ((a.stride_n | a.stride_h) & 7) != 0) return RADAR_INVALID_ARG;
    if (N == 0) return RADAR_OK;
    const hipError_t e = launch("kvq_append", d->D == 128 ? kvq_append_kernel<128> : kvq_append_kernel<64>, dim3((unsigned)groups), dim3(kRwThreads), 0,
                                static_cast<hipStream_t>(stream), a);
    return e == hipSuccess ? RADAR_OK : RADAR_HIP_ERROR;
}

// Bytes between layers, or -1 where the descriptor's are not possible.
static int64_t layer_bytes(const radar_kvq_desc *d) {
    const int64_t dense = (int64_t)d->n_blocks * d->Hkv * d->block_rows * (d->D + d->D / 16);
    if (d->layers < 1 || d->layer_stride < 0 || (d->layer_stride & 15) != 0) return -1;
    if (d->layer_stride != 0 && d->layers > 1 && d->layer_stride < dense) return -1;       // layers would share memory
    return d->layer_stride ? d->layer_stride : dense;
}

extern "C" radar_status radar_kvq_read(const void *cache, const int32_t *slots, void *k, void *v, int64_t N, const radar_kvq_desc *d, void *stream) {
    RwArgs a{};
    int64_t groups;
    const radar_status st = rw_args(k, v, slots, cache, N, d, &a, &groups);
    if (st != RADAR_OK) return st;
    a.k_out = static_cast<__bf16 *>(k); a.v_out = static_cast<__bf16 *>(v);
    a.layer_stride = layer_bytes(d);
    if (a.layer_stride < 0) return RADAR_INVALID_ARG;
    if (d->layers > 65535) return RADAR_UNSUPPORTED_SHAPE;
    if (N == 0) return RADAR_OK;
    // layers a workgroup: up to four, as long as eight workgroups a CU are left
    a.layers = d->layers;
    a.per = (int)std::min<int64_t>({std::max<int64_t>(groups * d->layers / kRwGroups, 1), kRwLayers, d->layers});
    const auto kernel = d->D == 128 ? (a.per > 1 ? kvq_read_kernel<128, 4> : kvq_read_kernel<128, 1>) : a.per > 1 ? kvq_read_kernel<64, 4> : kvq_read_kernel<64, 1>;
    const hipError_t e = launch("kvq_read", kernel, dim3((unsigned)groups, (unsigned)((d->layers + a.per - 1) / a.per)),
                                dim3(kRwThreads), 0, static_cast<hipStream_t>(stream), a);
    return e == hipSuccess ? RADAR_OK : RADAR_HIP_ERROR;
}

extern "C" radar_status radar_kvq_commit(void *cache, const int32_t *block_tables, int32_t max_blocks, const int32_t *ctx_lens, const int32_t *accept_len,
                                         const int32_t *accept_path, int32_t path_len, int32_t B, int32_t *new_ctx_lens, const radar_kvq_desc *d,
                                         void *stream) {
    if (!cache || !block_tables || !ctx_lens || !accept_len || !accept_path || new_ctx_lens == ctx_lens) return RADAR_INVALID_ARG;
    if (max_blocks < 1 || path_len < 1 || B < 1 || ((uintptr_t)cache & 15) != 0) return RADAR_INVALID_ARG;
    const radar_status st = kvq_check(d);
    if (st != RADAR_OK) return st;
    if (path_len > RADAR_T_MAX || B > 65535) return RADAR_UNSUPPORTED_SHAPE;
    CmArgs a{static_cast<unsigned char *>(cache), block_tables, ctx_lens, accept_len, accept_path, new_ctx_lens, layer_bytes(d),
             max_blocks, path_len, kvq_log2(d->block_rows), d->Hkv, 0, d->n_blocks, 0};
    if (a.layer_stride < 0) return RADAR_INVALID_ARG;
    if ((int64_t)d->layers * d->Hkv >= (1 << 24)) return RADAR_UNSUPPORTED_SHAPE;
    a.units = d->layers * d->Hkv;
    // pairs a wavefront: as many as leave 16 wavefronts a CU
    a.per = (int)std::min<int64_t>(std::max<int64_t>((int64_t)a.units * B / kCmWaves, 1), 16);
    const int per_group = kCmThreads / kWave * a.per;
    const dim3 grid((unsigned)((a.units + per_group - 1) / per_group), (unsigned)B);
    const hipError_t e = launch("kvq_commit", d->D == 128 ? kvq_commit_kernel<128> : kvq_commit_kernel<64>, grid, dim3(kCmThreads), 0,
                                static_cast<hipStream_t>(stream), a);
    return e == hipSuccess ? RADAR_OK : RADAR_HIP_ERROR;
}
