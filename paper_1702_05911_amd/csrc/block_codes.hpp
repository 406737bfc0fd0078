// Codes and scales of 8-bit blocks, eight values a lane (block_quantize.hip, rms_norm.hip).
#pragma once
#include "encoder.hpp"

namespace pqt {
namespace {

constexpr int kBlock = PQT_BLOCK;
constexpr int kLanesOfBlock = kBlock / 8;

// exponent byte of the smallest 2^e, e >= -126, with m <= 448 * 2^e (448 = 1.75 * 2^8), of the bits of m >= 0
__device__ __forceinline__ uint32_t scale_byte(uint32_t m) {
    const int e = (int)(m >> 23) - 8 + ((m & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)max(e, 1);
}
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }   // 2^-e: byte is 1 .. 247

// magnitude bits; those of infinities and NaN are at least kNotFinite
constexpr uint32_t kNotFinite = 0x7f800000u;
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t finite_magnitude(float v) { return magnitude(v) < kNotFinite ? magnitude(v) : 0u; }

// e4m3 numbers of eight floats under a scale, to nearest even; `all_finite`: the same for the wavefront, so that what NaN costs is
// paid only where there is one
__device__ __forceinline__ uint2 eight_codes(const float (&v)[8], float inv, bool all_finite) {
    int lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, 0, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, lo, true);
    int hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * inv, v[5] * inv, 0, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * inv, v[7] * inv, hi, true);
    if (!all_finite) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (magnitude(v[j]) >= kNotFinite) {
                int& word = j < 4 ? lo : hi;
                word = (int)(((uint32_t)word & ~(0xffu << (8 * (j & 3)))) | (0x7fu << (8 * (j & 3))));
            }
    }
    return uint2{(uint32_t)lo, (uint32_t)hi};
}

__device__ __forceinline__ uint32_t max_of_16(uint32_t v) {
    v = max(v, dpp_take<0xB1, 0xf>(v, v));
    v = max(v, dpp_take<0x4E, 0xf>(v, v));
    v = max(v, dpp_take<0x141, 0xf>(v, v));
    return max(v, dpp_take<0x140, 0xf>(v, v));
}

}  // namespace
}  // namespace pqt
