// Heads held in 4 bits: codes (sign, two bits of exponent, one of mantissa) times a scale of six significant bits per head.
// What a code stands for has at most two significant bits, so code times scale is exactly a bf16 number.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include "pec_paged.h"

namespace pec {

// Device view of such a cache: PagedCache's strides are those of the codes, in bytes.
struct Q4Cache {
    uint8_t *k, *v;
    uint16_t *ks, *vs;                       // bf16 bits
    PagedCache c;
    int64_t ks_sp, ks_st, ks_sh, vs_sp, vs_st, vs_sh;
    int32_t Hkv;
};
// Host checks of the cache and the batch; fills `out`.
int resolve_q4_cache(const char *who, const pec_q4_cache &a, const int32_t *status, Q4Cache &out);

namespace q4 {

constexpr int kHeadBytes = kHeadDim / 2;
constexpr uint16_t kNaN = 0x7fff;

// The smallest number of six significant bits with 6 s >= most, between 2^-100 and 1.3125 * 2^125.  The products 6 s are exact.
// `most` may have been rounded to odd: 6 s has bits to spare.
__device__ __forceinline__ float scale_of(float most)
{
    constexpr uint32_t step = 1u << 18;      // of 23 bits after the first, five stay
    uint32_t b = __float_as_uint(most * (0x1.555552p-3f)) & ~(step - 1);               // at most two numbers short
    if (6.f * __uint_as_float(b) < most) b += step;
    if (6.f * __uint_as_float(b) < most) b += step;
    return fminf(fmaxf(__uint_as_float(b), 0x1p-100f), 1.3125f * 0x1p125f);
}

// Two numbers in units of the scale to a byte of codes, ties to the even code; magnitudes over 6 become 6.
__device__ __forceinline__ uint32_t encode2(float lo, float hi)
{
    uint32_t r;
    asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %2, %1;\n\tmov.b32 %0, {t, 0, 0, 0};\n\t}" : "=r"(r) : "f"(lo), "f"(hi));
    return r;
}

// Eight codes to bf16, times the scale (twice the same bf16 in `s2`): r[i] = channels 2 i, 2 i + 1.
// A nibble's bits put at those of a bf16's sign, the low two of its exponent and the first of its mantissa make its value times
// 2^-126, 0.5 being a subnormal of it; both factors are exact.
__device__ __forceinline__ void decode8(uint32_t w, __nv_bfloat162 s2, uint32_t (&r)[4])
{
    const uint32_t w4 = w << 4;
    const __nv_bfloat162 up = __halves2bfloat162(__ushort_as_bfloat16(0x7e80), __ushort_as_bfloat16(0x7e80));      // 2^126
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // bytes 1 and 3: byte i of w << 4 (the even channel on top) and of w (the odd one)
        const uint32_t x = __byte_perm(w, w4, (uint32_t)(i << 12) | (uint32_t)((4 + i) << 4));
        const uint32_t t = (x & 0x80008000u) | ((x >> 6) & 0x01c001c0u);
        const __nv_bfloat162 y = __hmul2(__hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&t), up), s2);
        r[i] = *reinterpret_cast<const uint32_t *>(&y);
    }
}
// The same to fp16, times a scale that fp16 holds.
__device__ __forceinline__ void decode8_f16(uint32_t w, __half2 s2, uint32_t (&r)[4])
{
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 y = __hmul2(*reinterpret_cast<const __half2 *>(&r[i]), s2);
        r[i] = *reinterpret_cast<const uint32_t *>(&y);
    }
}
__device__ __forceinline__ __nv_bfloat162 twice(uint16_t s) { return __halves2bfloat162(__ushort_as_bfloat16(s), __ushort_as_bfloat16(s)); }

}  // namespace q4
}  // namespace pec
