// The 8-bit key/value cache: layout, scales and conversions shared by the kernels that write, read and thin it out.
//   K codes [B, Hkv, cap, D]             one byte (e4m3) per channel
//   V codes [B, Hkv, cap / 32, D, 32]    channel-major inside each block of 32 rows: the product P V wants the keys of a channel side by side, and
//                                        a thread of mma.sync then finds its eight of them in one 8-byte load
//   scales  [B, Hkv, cap / 32] fp32      a power of two per 32 rows and head, one for K and one for V: value = code * scale
// The scale is the smallest power of two s >= 2^-100 with 448 s >= the block's largest finite magnitude.  A power of two costs a floating code nothing (its relative precision
// is the same at every scale) and makes code = round(x / s) exact arithmetic: every implementation finds the same codes, and moving a row to another scale
// rounds only what falls below the smallest normal code.
#pragma once

#include <cuda_fp16.h>

#include "dm_internal.h"

namespace dm {
namespace kv8 {

constexpr int BLK = DM_KV8_BLOCK;                  // rows of the cache that share a scale

struct Cache {
    uint8_t *k, *v;
    float *ks, *vs;
    int cap;                                       // rows, a multiple of BLK
};

#ifdef __CUDACC__
// exponent field of the scale for a largest magnitude `amax` (finite, >= 0): 2^(e-8) where the mantissa is at most 1.75, else 2^(e-7)
__device__ __forceinline__ float scale_of(float amax) {
    const int bits = __float_as_int(amax);
    const int e = (bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
    return __int_as_float(max(e, 127 - 100) << 23);
}
__device__ __forceinline__ float inverse_pow2(float s) { return __int_as_float((254 << 23) - __float_as_int(s)); }   // 1 / s of a power of two in [2^-126, 2^126]
// two codes from two values that are multiples of the scale already (|x| <= 448 where finite); NaN and infinities become the NaN code
__device__ __forceinline__ uint32_t encode2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    uint32_t c = r;
    if (!(fabsf(lo) <= 3.0e38f)) c = (c & 0xff00u) | 0x7fu;
    if (!(fabsf(hi) <= 3.0e38f)) c = (c & 0x00ffu) | 0x7f00u;
    return c;
}
__device__ __forceinline__ uint32_t f16x2_of(uint32_t two_codes) {         // the low 16 bits: two e4m3 -> two f16, exact
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two_codes));
    return r;
}
__device__ __forceinline__ float2 decode2(uint32_t two_codes) {
    const uint32_t h = f16x2_of(two_codes);
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}
#endif

}  // namespace kv8
}  // namespace dm
