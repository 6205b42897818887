// Rows in 8 bits: e4m3 codes, and for each 128 elements of a row one power of two (e8m0), the least that leaves no element beyond 448.
#pragma once

#include "sp_elem.h"

namespace sp {

constexpr int kQ8Block = 128;
constexpr float kQ8Most = 448.f;       // 1.75 * 2^8, the largest e4m3 value
constexpr uint32_t kQ8NaN = 255;       // a block that holds an infinity or NaN
inline int64_t q8_blocks(int64_t c) { return (c + kQ8Block - 1) / kQ8Block; }
inline int64_t q8_scales(int64_t c) { return (q8_blocks(c) + 3) / 4 * 4; }  // bytes of a row of scales

// The code of a block's scale from its largest size (as it is, NaN for NaN): the exponent e of 2^e, + 127, with top <= 448 * 2^e.
__device__ __forceinline__ uint32_t q8_scale(float top) {
    const uint32_t b = __float_as_uint(top);
    if (b >= 0x7f800000u) return kQ8NaN;
    if (b == 0) return 127;
    // top = 1.m * 2^(b >> 23): 448 = 1.75 * 2^8.  Tops below 2^-118 (subnormal ones too) have the least scale, 2^-127.
    const int e = (int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u);
    return e < 0 ? 0u : (uint32_t)e;
}
// 1 / scale as a factor: 2^(127 - code) is beyond fp32 for code 0 only, which two factors make.
__device__ __forceinline__ float q8_times(float v, uint32_t code) { return ldexpf(v, 127 - (int)code); }

// Four elements, divided by their block's scale, as codes; to nearest even.
__device__ __forceinline__ uint32_t q8_codes(float a, float b, float c, float d, uint32_t code) {
    if (code == kQ8NaN) return 0;  // whatever they are, the scale makes NaN of them
    int r = 0;
    r = __builtin_amdgcn_cvt_pk_fp8_f32(q8_times(a, code), q8_times(b, code), r, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(q8_times(c, code), q8_times(d, code), r, true);
    return (uint32_t)r;
}

// The largest size of values in LANES neighbouring lanes.  NaN counts as the largest: sizes are compared as whole numbers.
template <int LANES>
__device__ __forceinline__ float q8_top(float v) {
    struct Most {
        static __device__ __forceinline__ float of(float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); }
    };
    return lanes_reduce<LANES, Most>(v);
}
__device__ __forceinline__ float q8_size(float v) { return __uint_as_float(__float_as_uint(v) & 0x7fffffffu); }
__device__ __forceinline__ float q8_larger(float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); }

}  // namespace sp
