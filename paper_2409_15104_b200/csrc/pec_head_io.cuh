// A head of 128 channels held by 16 lanes, for the kernels that go over heads one by one: lane l has channels 4 l .. 4 l + 3 and
// their rotary partners 64 on.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

namespace pec {
namespace heads {

// Four channels of a head as they lie in memory.
template <class E> struct Quad;
template <> struct Quad<__nv_bfloat16> {
    typedef uint2 Raw;
    static __device__ __forceinline__ void unpack(const Raw &u, float (&x)[4])
    {
        x[0] = __uint_as_float(u.x << 16); x[1] = __uint_as_float(u.x & 0xffff0000u);
        x[2] = __uint_as_float(u.y << 16); x[3] = __uint_as_float(u.y & 0xffff0000u);
    }
    static __device__ __forceinline__ Raw pack(const float (&x)[4])
    {
        const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
        return make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
    }
};
template <> struct Quad<float> {
    typedef float4 Raw;
    static __device__ __forceinline__ void unpack(const Raw &u, float (&x)[4]) { x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w; }
    static __device__ __forceinline__ Raw pack(const float (&x)[4]) { return make_float4(x[0], x[1], x[2], x[3]); }
};
template <class E> struct Head { typename Quad<E>::Raw lo, hi; };    // a lane's eight channels
template <class E>
__device__ __forceinline__ Head<E> load_head(const E *head, int l)
{
    typedef typename Quad<E>::Raw Raw;
    Head<E> u;
    u.lo = *reinterpret_cast<const Raw *>(head + 4 * l);
    u.hi = *reinterpret_cast<const Raw *>(head + 64 + 4 * l);
    return u;
}
template <class E>
__device__ __forceinline__ void store_head(E *head, int l, const Head<E> &u)
{
    typedef typename Quad<E>::Raw Raw;
    *reinterpret_cast<Raw *>(head + 4 * l) = u.lo;
    *reinterpret_cast<Raw *>(head + 64 + 4 * l) = u.hi;
}

}  // namespace heads
}  // namespace pec
