// PTX wrappers of the paged attention kernels, beside those of pec_sm100.cuh.
#pragma once
#include "pec_sm100.cuh"

namespace pec {
namespace sm100 {

// idesc_bf16_f32 for fp16 A/B.
__host__ __device__ constexpr uint32_t idesc_f16_f32(int m, int n, int a_mn_major, int b_mn_major) { return idesc_bf16_f32(m, n, a_mn_major, b_mn_major) & ~(1u << 7 | 1u << 10); }
// For kind::f8f6f4 (8 bits and fewer) with fp32 accumulation; formats: 0 e4m3, 1 e5m2, 5 e2m1 (in shared memory 16 codes in the first 8 of
// every 16 bytes).
constexpr int kE4M3 = 0, kE5M2 = 1, kE2M1 = 5;
__host__ __device__ constexpr uint32_t idesc_f8f6f4_f32(int m, int n, int a_format, int b_format, int a_mn_major, int b_mn_major)
{
    return (1u << 4)                      // D format: f32
         | ((uint32_t)a_format << 7)
         | ((uint32_t)b_format << 10)
         | ((uint32_t)a_mn_major << 15)
         | ((uint32_t)b_mn_major << 16)
         | ((uint32_t)(n >> 3) << 17)
         | ((uint32_t)(m >> 4) << 24);
}

// 16 consecutive columns of this warp's 32 TMEM lanes, and back.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};\n\t"
        "tcgen05.wait::st.sync.aligned;"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

}  // namespace sm100
}  // namespace pec
