// The paged 4-bit cache's layout, for the kernels that write it, move its rows and attend over it (gfx950).
#pragma once

#include "radar_device.h"

namespace radar {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t kScaleMost = 252, kScaleNaN = 255;      // largest scale byte of finite values, and that of a block that held an infinity or NaN

// Sections of a chunk (one KV head's rows of one block), in bytes from its start.  R rows, head dimension D.
template <int D>
struct KvqChunk {
    static constexpr int kRow = D / 2, kPieces = D / 8, kScales = D / 32;     // bytes of a row's codes; eights of a row; scales of a row
    __host__ __device__ static constexpr int bytes(int R) { return R * (D + D / 16); }
    __device__ static int k_row(int row) { return row * kRow; }
    __device__ static int v_piece(int R, int row, int piece) { return R * kRow + (((row >> 3) * kPieces + piece) * 8 + (row & 7)) * 4; }
    __device__ static int k_scale(int R, int row, int blk) { return R * D + ((row >> 3) * kScales + blk) * 8 + (row & 7); }
    __device__ static int v_scale(int R, int row, int blk) { return R * (D + D / 32) + ((row >> 3) * kScales + blk) * 8 + (row & 7); }
};

__device__ __forceinline__ float kvq_scale(uint32_t byte) { return __uint_as_float(byte << 23); }   // 255: infinity, which the conversions below take for NaN

// Eight codes of a row (the nibbles of w, lowest first) as bf16, exactly: two to a word.
__device__ __forceinline__ void kvq_decode8(uint32_t w, float scale, uint32_t (&out)[4]) {
    out[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
    out[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
    out[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
    out[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
}

// Which limits of radar_kvq_desc a call's descriptor breaks (host).
inline radar_status kvq_check(const radar_kvq_desc *d) {
    if (!d || d->n_blocks < 1 || d->Hkv < 1 || d->block_rows < 1) return RADAR_INVALID_ARG;
    if ((d->D != 64 && d->D != 128) || (d->block_rows != 16 && d->block_rows != 32 && d->block_rows != 64 && d->block_rows != 128) || d->Hkv > 65535 ||
        (int64_t)d->n_blocks * d->block_rows > INT32_MAX)
        return RADAR_UNSUPPORTED_SHAPE;
    return RADAR_OK;
}
inline int kvq_log2(int rows) { return rows == 16 ? 4 : rows == 32 ? 5 : rows == 64 ? 6 : 7; }

}  // namespace radar
