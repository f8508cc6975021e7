// The 4-bit cache format on the device.  The d values of a (position, kv head) are blocks of 32 that share a power of
// two 2^e; a value is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (codes 0 .. 7, the sign above them) times it.  A cache is
// [num_blocks][kv heads] blocks of (d/2 + d/32) * block_size bytes:
//   codes    [block_size][d/2]     channel 2i in the low half of byte i, 2i + 1 in the high half
//   scales   [d/32][block_size]    e + 127
// gfx950 turns two codes and a power of two into two bfloat16 in one instruction, exactly (every code times 2^e has
// at most two significant bits), and rounds two floats to codes in one.
#pragma once
#include "ra_device.h"

namespace ra {

template <int D>
struct Fp4 {
    static constexpr int ROW = D / 2;             // code bytes of a position
    static constexpr int GROUPS = D / 32;         // scales of a position
    __host__ __device__ static constexpr int64_t block_bytes(int block_size_log2) {
        return (int64_t)(ROW + GROUPS) << block_size_log2;
    }
};

// 2^e as the conversions below want it, from the scale byte (they read the exponent bits alone).
__device__ __forceinline__ float fp4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// The two values of byte BYTE of `codes` as bfloat16 bits, the even channel in the low half.
template <int BYTE>
__device__ __forceinline__ uint32_t fp4_pair(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, BYTE));
}
// The 8 values of a word.
__device__ __forceinline__ u32x4 fp4_octet(uint32_t codes, float scale) {
    return u32x4{fp4_pair<0>(codes, scale), fp4_pair<1>(codes, scale), fp4_pair<2>(codes, scale), fp4_pair<3>(codes, scale)};
}

// The scale byte of a block whose largest magnitude has the bfloat16 bits `top`: e = floor(log2 a) - 2, and one more from
// 1.75 * 2^floor(log2 a) on, so that no value is off by more than half a step of its place on the grid.  Infinities and NaN
// end up at the largest e, where the largest value, 6 * 2^125, is still finite.
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t top) {
    const int b = (int)(top >> 7) + ((top & 0x7fu) >= 0x60u ? 1 : 0) - 2;
    return (uint32_t)(b < 0 ? 0 : b > 252 ? 252 : b);
}
// 8 bfloat16 to a word of codes (round to nearest even code, saturating; a NaN counts as an infinity).
__device__ __forceinline__ uint32_t fp4_encode(const u32x4 x, float scale) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, bf16_lo(x[0]), bf16_hi(x[0]), scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, bf16_lo(x[1]), bf16_hi(x[1]), scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, bf16_lo(x[2]), bf16_hi(x[2]), scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, bf16_lo(x[3]), bf16_hi(x[3]), scale, 3);
    return w;
}

}  // namespace ra
