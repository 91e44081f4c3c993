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

// Eight values of a row as codes (the nibbles of the result, lowest first) and the scale byte of the 32 that they are among, which four neighbouring
// lanes have between them: all four call.  The largest magnitude is found on the bit patterns (larger than 0x7f7f: not a number or infinite).
// amax = (1 + m/128) 2^(E-127): the scale's exponent is E - 127 - 2, or one more from 1.75 on, where 6 would be too little by more than half a step.
struct KvqCodes { uint32_t code, mark; };
__device__ __forceinline__ KvqCodes kvq_encode8(uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3) {
    auto two = [](uint32_t x) { return max(x & 0x7fffu, (x >> 16) & 0x7fffu); };
    uint32_t top = max(max(two(x0), two(x1)), max(two(x2), two(x3)));
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    const bool sound = top < 0x7f80u;
    const uint32_t byte = (uint32_t)min(max((int)(top >> 7) - 2 + ((top & 127u) >= 96u ? 1 : 0), 1), (int)kScaleMost);
    const float scale = kvq_scale(byte);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x0), scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x1), scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x2), scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x3), scale, 3);
    return KvqCodes{sound ? w : 0u, sound ? byte : kScaleNaN};
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
