// Rows in 8 bits: e4m3 values with a power-of-two scale for each block of 128 of them.
//
// A row of d values is d bytes and, in another array, a byte per block: 2^(byte - 127), 255 for NaN (the e8m0 format).  A row
// has 4 ceil(d / 512) scale bytes, so that four consecutive blocks' scales are one aligned word; bytes past the last
// block are 127.  The scale of a block is the smallest power of two 2^e, e >= -126, with which its largest magnitude is at most
// 448 (e = 0 for a block of zeros).  A power of two rather than amax / 448: e4m3 is a floating-point format, so a block
// loses no precision by lying up to a factor of two below 448, and every use of a scale -- here, in the products -- is exact.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sv_device.h"

namespace sv {

// the value of a scale byte
__device__ __forceinline__ float scale_value(uint32_t byte) {
    return byte == 255u ? __builtin_nanf("") : __uint_as_float(byte ? byte << 23 : 0x00400000u);
}

// The scale byte of a block from its largest magnitude's bits (of non-negative floats, infinities and NaN above all others), and
// what its values are multiplied by: 2^-e.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
    if (amax_bits >= 0x7F800000u) return 255u;                       // an infinity or a NaN: the whole block is NaN
    if (amax_bits == 0u) return 127u;
    const int e = (int)(amax_bits >> 23) - 127 - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);      // 448 = 1.75 * 2^8
    return (uint32_t)(max(e, -126) + 127);
}
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }   // byte 1 .. 247

// largest bits of the 16 lanes of a DPP row, in every lane
__device__ __forceinline__ uint32_t row16_max_u32(uint32_t x) {
    x = umax32(x, dpp_u32<DPP_QUAD_1032>(x));
    x = umax32(x, dpp_u32<DPP_QUAD_2301>(x));
    x = umax32(x, dpp_u32<DPP_ROW_HALF_MIRROR>(x));
    return umax32(x, dpp_u32<DPP_ROW_MIRROR>(x));
}

// Eight consecutive values of a block per lane, 16 lanes a block: the eight in 8 bits (round to nearest even), and the
// scale byte.  Lanes past the row's end come with zeros.  All lanes must be active.
__device__ __forceinline__ uint2 quantize_8(const float (&v)[8], uint32_t* byte_out) {
    uint32_t most = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = umax32(most, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    const uint32_t byte = scale_byte(row16_max_u32(most));
    *byte_out = byte;
    if (byte == 255u) return uint2{0x7F7F7F7Fu, 0x7F7F7F7Fu};
    const float f = inverse_scale(byte);
    uint2 q;
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * f, v[1] * f, 0, false);
    q.x = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2] * f, v[3] * f, w, true);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * f, v[5] * f, 0, false);
    q.y = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[6] * f, v[7] * f, w, true);
    return q;
}

// the four scale bytes of the wavefront's 512 values as one word (lanes 0, 16, 32, 48 of `byte`)
__device__ __forceinline__ uint32_t scale_word(uint32_t byte) {
    return (uint32_t)__builtin_amdgcn_readlane((int)byte, 0) | (uint32_t)__builtin_amdgcn_readlane((int)byte, 16) << 8 |
           (uint32_t)__builtin_amdgcn_readlane((int)byte, 32) << 16 | (uint32_t)__builtin_amdgcn_readlane((int)byte, 48) << 24;
}

// eight stored values (16 bytes of bfloat16, 32 of float32), widened
template <int DT>
struct Eight {
    u32x4 w[DT == DT_BF16 ? 1 : 2];
    __device__ __forceinline__ void load(const char* p) {
        w[0] = *reinterpret_cast<const u32x4*>(p);
        if constexpr (DT == DT_F32) w[1] = *reinterpret_cast<const u32x4*>(p + 16);
    }
    __device__ __forceinline__ void store(char* p) const {
        *reinterpret_cast<u32x4*>(p) = w[0];
        if constexpr (DT == DT_F32) *reinterpret_cast<u32x4*>(p + 16) = w[1];
    }
    __device__ __forceinline__ void clear() {
        w[0] = zero16();
        if constexpr (DT == DT_F32) w[1] = zero16();
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (DT == DT_BF16) v[i] = __uint_as_float(i & 1 ? w[0][i / 2] & 0xFFFF0000u : w[0][i / 2] << 16);
            else v[i] = __uint_as_float(w[i / 4][i % 4]);
        }
    }
    // rounded to the storage type; v becomes what is stored
    __device__ __forceinline__ void put(float (&v)[8]) {
        if constexpr (DT == DT_BF16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[0][i] = (uint32_t)f32_to_bf16_any(v[2 * i]) | (uint32_t)f32_to_bf16_any(v[2 * i + 1]) << 16;
            }
            get(v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i / 4][i % 4] = __float_as_uint(v[i]);
        }
    }
    // round to nearest even; infinities and NaN stay what they are
    static __device__ __forceinline__ uint16_t f32_to_bf16_any(float x) {
        return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
    }
};

}  // namespace sv
