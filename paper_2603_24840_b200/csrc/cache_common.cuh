// The paged 8-bit cache: layout, its scales, conversions.  Shared by the append and the attention that reads it.
#pragma once
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include "arrol_internal.h"

namespace {

constexpr int CACHE_MAX_D = 128;
constexpr float E4M3_MOST = 448.0f;
constexpr int CACHE_LEAST_EXPONENT = -100;        // of a scale

// Exponent e of the least power of two with amax 2^-e <= 448 = 0.875 x 2^9, not below the least one; amax finite, not negative.
__device__ __forceinline__ int cache_exponent(float amax) {
    const uint32_t u = __float_as_uint(amax);
    if (u < 0x00800000u) return CACHE_LEAST_EXPONENT;                  // zero and subnormals
    // amax = m 2^x, m in [1, 2): 448 = 1.75 x 2^8
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x007FFFFFu) > 0x00600000u ? 1 : 0);
    return e < CACHE_LEAST_EXPONENT ? CACHE_LEAST_EXPONENT : e;
}
__device__ __forceinline__ float cache_power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }       // 2^e, normal
// The larger of the maximum and |x|, leaving out what is not finite (x - x is then NaN, which fmaxf passes over).
__device__ __forceinline__ float finite_max(float most, float x) { return fmaxf(most, fabsf(x) + (x - x)); }
// Two numbers rounded to e4m3, nearest even, NaN stays NaN; an infinity would become 448.
__device__ __forceinline__ uint16_t e4m3_pair_finite(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
// the same with infinities to NaN
__device__ __forceinline__ uint16_t e4m3_pair(float lo, float hi) { return e4m3_pair_finite(lo + (lo - lo), hi + (hi - hi)); }
__device__ __forceinline__ uint32_t e4m3_pair_to_half(uint16_t c) {                                              // exact
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(c));
    return r;
}
__device__ __forceinline__ float2 e4m3_pair_to_float(uint16_t c) {
    const uint32_t h = e4m3_pair_to_half(c);
    float2 f;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(f.x), "=f"(f.y) : "r"(h));
    return f;
}

// Tokens of sequence i; none where its length is not one that its table row can hold.
__device__ __forceinline__ int cache_tokens(const int32_t* lengths, int i, int table_pages, int page, bool& bad) {
    const int n = lengths[i];
    if (n < 0 || n > (int64_t)table_pages * page) { bad = true; return 0; }
    return n;
}

inline int cache_check(const arrol_cache& c) {
    if (c.pages < 0 || c.page < 1 || c.Hkv < 1 || c.D < 1) return ARROL_ERR_INVALID_ARG;
    if ((c.page != 16 && c.page != 32 && c.page != 64 && c.page != 128) || c.D % 16 || c.D > CACHE_MAX_D || c.Hkv > 65536) return ARROL_ERR_UNSUPPORTED;
    if (c.pages == 0) return ARROL_OK;
    const int64_t bytes = (int64_t)c.Hkv * c.page * c.D;
    auto pages_ok = [&](const void* p, int64_t stride) { return p && arrol_aligned(p, 16) && stride % 16 == 0 && stride >= bytes && stride < ((int64_t)1 << 32); };
    auto scales_ok = [&](const void* p, int64_t stride) { return p && arrol_aligned(p, 4) && stride >= c.Hkv && stride < ((int64_t)1 << 32); };
    return pages_ok(c.k_cache, c.k_page_stride) && pages_ok(c.v_cache, c.v_page_stride) && scales_ok(c.k_scale, c.k_scale_stride) && scales_ok(c.v_scale, c.v_scale_stride)
               ? ARROL_OK : ARROL_ERR_INVALID_ARG;
}
inline bool cache_rows_ok(const void* p, int64_t stride, int heads, int D) {
    return p && arrol_aligned(p, 16) && stride % 8 == 0 && stride >= (int64_t)heads * D && stride < ((int64_t)1 << 38);
}

}  // namespace
