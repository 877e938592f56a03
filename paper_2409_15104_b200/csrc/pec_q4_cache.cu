// A paged K/V cache held in 4 bits: new keys (normalised and rotated on the way) and values into it (pec_kv_append_q4), and what it
// holds back into packed tensors (pec_kv_read_q4).
//
//     s = least number of six significant bits with 6 s >= max |z|,   code = nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 to |z| / s,
//     z = the head's channels; for keys after norm and rotation (see pec_heads.cu), which are worked out in fp64
//
// Both are bound by memory, a head of bf16 being 256 bytes on one side and 66 on the other: 131072 rows of 8 + 8 heads are read in 116 us
// where memory takes 103.  Appending has some 150 instructions and three dependent loads (the request, the page, the angles) for each four
// heads and does not reach that: 7302 tokens with norm and rotation, and 8901 read, 34 us (23 and 10 by themselves) where memory takes 13
// (all of it in fp64 took 49).
//
// Which code is the nearest is decided exactly (but for normalised or rotated channels within 2^-41 of a border, where fp64 ends).  bf16
// channels that are quantised as they are: x / s is either a border between two codes or 2^-11 away from it (x has 8 bits, s 6, a border 3),
// while the product with the reciprocal is off by 2^-19: put on a grid of 2^-14 it is a border where x / s is one, and on its side
// elsewhere.  Everything else is worked out in fp32 with a bound of its error.  Where the least and the largest number within the bound have
// different codes (one of 200 usual heads has such a channel), the channel goes through fp64, where they would have different scales the
// head: z times 1 / s, rounded to 41 bits for the same reason (an fp32 x is 2^-25 away from a border at least), then to fp32 with the last
// bit set where anything was cut off, so that nothing becomes a border that is none.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <type_traits>
#include "pec_head_io.cuh"
#include "pec_host.h"
#include "pec_internal.h"
#include "pec_q4.cuh"

namespace pec {
namespace q4 {
using heads::Quad;

constexpr int kThreads = 64, kWarps = kThreads / 32;
constexpr int kLanes = 8, kHeads = 32 / kLanes;      // appending: lanes of a head, heads of a warp at once
constexpr int kRows = 4, kPair = 2;          // reading: heads of a half warp in flight, for as many tokens

// To fp32 towards zero, the last bit set where bits were cut off: compares with any number of fewer bits as z does.
__device__ __forceinline__ float to_odd(double z)
{
    const uint32_t f = __float_as_uint(__double2float_rz(z));
    return __uint_as_float(f | ((__double2loint(z) & 0x1fffffff) != 0 ? 1u : 0u));
}

// Over the lanes of a head.
__device__ __forceinline__ float head_max(float x)
{
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
    return x;
}
// The same, NaN if any is.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float head_max_nan(float x)
{
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) x = max_nan(x, __shfl_xor_sync(0xffffffffu, x, d));
    return x;
}
__device__ __forceinline__ float rcp(float x)      // to 2^-23 of itself
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Lane l of a head has its channels 8 l .. 8 l + 7 and their rotary partners 64 on.
template <class E> struct Share { typename Quad<E>::Raw x[4]; };
template <class E>
__device__ __forceinline__ Share<E> load_share(const E *head, int l)
{
    Share<E> u;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const E *at = head + 64 * k + 8 * l;
        if constexpr (sizeof(E) == 2) {
            const uint4 v = *reinterpret_cast<const uint4 *>(at);
            u.x[2 * k] = make_uint2(v.x, v.y); u.x[2 * k + 1] = make_uint2(v.z, v.w);
        } else {
            u.x[2 * k] = reinterpret_cast<const float4 *>(at)[0]; u.x[2 * k + 1] = reinterpret_cast<const float4 *>(at)[1];
        }
    }
    return u;
}
template <class E>
__device__ __forceinline__ void unpack(const Share<E> &u, float (&x)[16])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) Quad<E>::unpack(u.x[k], *reinterpret_cast<float (*)[4]>(x + 4 * k));
}

// A lane's codes, eight in each half of the head, and the head's scale (bits).
struct Coded { uint32_t lo, hi; uint16_t scale; };
__device__ __forceinline__ uint32_t encode8(const float *y)
{
    return encode2(y[0], y[1]) | encode2(y[2], y[3]) << 8 | encode2(y[4], y[5]) << 16 | encode2(y[6], y[7]) << 24;
}
__device__ __forceinline__ uint16_t bits_of(float s) { return (uint16_t)(__float_as_uint(s) >> 16); }

// bf16 channels as they are.
__device__ __forceinline__ Coded quantise(const Share<__nv_bfloat16> &u)
{
    constexpr float kGrid = 0x1.8p9f;                      // its neighbours are 2^-14 away
    float x[16], most = 0.f;
    unpack(u, x);
#pragma unroll
    for (int i = 0; i < 16; ++i) most = max_nan(most, fabsf(x[i]));
    most = head_max_nan(most);
    const float s = scale_of(most), f = rcp(s);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = fmaf(x[i], f, kGrid) - kGrid;
    return {encode8(x), encode8(x + 8), most < INFINITY ? bits_of(s) : kNaN};
}

// What happens to a head first: norm (weight, or NULL), rotation by the angles of a position (table, or NULL; see pec_rope_table).
struct Change { bool norm; float eps; const void *w; const float *table; int64_t n_pos; int32_t pos; };
template <class E>
__device__ __forceinline__ void weights(const Change &g, int l, float (&w)[16])
{
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = 1.f;
    if (g.w) unpack(load_share(static_cast<const E *>(g.w), l), w);
}
// Cosine and sine of a pair at pos = 64 a + b, by the addition theorem, in R.
template <class R>
__device__ __forceinline__ void turned(float kc, float ks, float fc, float fs, R &c, R &t)
{
    c = (R)kc * (R)fc - (R)ks * (R)fs;
    t = (R)ks * (R)fc + (R)kc * (R)fs;
}

// In fp64, for what is seldom and so in few registers: pair by pair from memory.  `head` is the lane's (NULL: none).
template <class E>
struct Exact {
    const E *head;
    const Change &g;
    int l;
    double r;

    static __device__ __forceinline__ double channel(const void *x, int i)
    {
        if constexpr (sizeof(E) == 2) return __uint_as_float((uint32_t)static_cast<const uint16_t *>(x)[i] << 16);
        else return static_cast<const float *>(x)[i];
    }
    // By a converged warp.
    __device__ __forceinline__ Exact(const E *head_, const Change &g_, int l_) : head(head_), g(g_), l(l_), r(1.0)
    {
        if (!g.norm) return;
        double ss = 0.0;
        if (head) {
            float x[16];
            unpack(load_share(head, l), x);
#pragma unroll
            for (int i = 0; i < 16; ++i) ss = fma((double)x[i], (double)x[i], ss);
        }
#pragma unroll
        for (int d = kLanes / 2; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
        r = rsqrt(ss * (1.0 / kHeadDim) + (double)g.eps);
    }
    __device__ __forceinline__ void pair(int k, double (&z)[2]) const
    {
        if (!head) { z[0] = z[1] = 0.0; return; }
        double a = channel(head, k), b = channel(head, 64 + k), c, t;
        if (g.w) { a *= channel(g.w, k); b *= channel(g.w, 64 + k); }              // (exact: 48 bits)
        if (g.table) {
            const float *coarse = g.table + 2 * 4096 + (int64_t)(g.pos >> 6) * 64 + k, *fine = g.table + (g.pos & 63) + 64 * k;
            turned(coarse[0], coarse[(g.n_pos + 63) / 64 * 64], fine[0], fine[4096], c, t);
            const double lo = a;
            a = fma(lo, c, -b * t);
            b = fma(b, c, lo * t);
        }
        z[0] = r * a; z[1] = r * b;
    }
    static __device__ __forceinline__ uint32_t code(double z, double r_s)
    {
        return encode2(to_odd(__longlong_as_double((__double_as_longlong(z * r_s) + 0x800) & ~0xfffll)), 0.f) & 15u;
    }
    // A head, by a converged warp.
    __device__ __forceinline__ Coded all() const
    {
        float most = 0.f;
        bool bad = false;
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
            double z[2];
            pair(8 * l + i, z);
            most = fmaxf(most, fmaxf(fabsf(to_odd(z[0])), fabsf(to_odd(z[1]))));
            bad = bad || !(fabs(z[0]) < INFINITY) || !(fabs(z[1]) < INFINITY);
        }
        most = head_max(bad ? INFINITY : most);
        const float s = scale_of(most);
        const double r_s = 1.0 / (double)s;
        Coded c = {0u, 0u, most < INFINITY ? bits_of(s) : kNaN};
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
            double z[2];
            pair(8 * l + i, z);
            c.lo |= code(z[0], r_s) << 4 * i;
            c.hi |= code(z[1], r_s) << 4 * i;
        }
        return c;
    }
    // A lane's channels whose codes have a bit set in `doubt`.
    __device__ __forceinline__ void some(Coded &c, uint32_t (&doubt)[2]) const
    {
        const double r_s = 1.0 / (double)__uint_as_float((uint32_t)c.scale << 16);
#pragma unroll 1
        while (doubt[0] | doubt[1]) {
            const int i = (__ffs(doubt[0] ? doubt[0] : doubt[1]) - 1) >> 2;
            const uint32_t nibble = 15u << 4 * i;
            double z[2];
            pair(8 * l + i, z);
            if (doubt[0] & nibble) c.lo = (c.lo & ~nibble) | code(z[0], r_s) << 4 * i;
            if (doubt[1] & nibble) c.hi = (c.hi & ~nibble) | code(z[1], r_s) << 4 * i;
            doubt[0] &= ~nibble; doubt[1] &= ~nibble;
        }
    }
};

// The linear map of a lane's pairs (see pec_heads.cu) up to the norm's factor: z_lo = lo * lc - hi * hs, z_hi = hi * hc + lo * ls.
struct Map { float lc[8], hs[8], hc[8], ls[8]; };
template <class E>
__device__ __forceinline__ void make_map(Map &m, const Change &g, int l)
{
    float w[16], c[8], t[8];
    weights<E>(g, l, w);
    if (g.table) {
        const int64_t na = (g.n_pos + 63) / 64;
        const float *coarse = g.table + 2 * 4096 + (int64_t)(g.pos >> 6) * 64 + 8 * l, *fine = g.table + (g.pos & 63) + 512 * l;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float4 kc = __ldg(reinterpret_cast<const float4 *>(coarse) + k), ks = __ldg(reinterpret_cast<const float4 *>(coarse + na * 64) + k);
            const float cc[4] = {kc.x, kc.y, kc.z, kc.w}, cs[4] = {ks.x, ks.y, ks.z, ks.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) turned(cc[i], cs[i], __ldg(fine + (4 * k + i) * 64), __ldg(fine + 4096 + (4 * k + i) * 64), c[4 * k + i], t[4 * k + i]);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (!g.table) { c[i] = 1.f; t[i] = 0.f; }
        m.lc[i] = w[i] * c[i]; m.ls[i] = w[i] * t[i]; m.hc[i] = w[8 + i] * c[i]; m.hs[i] = w[8 + i] * t[i];
    }
}

// In fp32; false where that does not decide the scale, bits of `doubt` set where it does not decide a code.  With M the head's largest |z|, a pair has |w lo|, |w hi| <= sqrt(2) M (a rotation keeps
// their norm), so |lo lc| + |hi hs| <= 2 M.  In units of 2^-24: lc and its like are off by 3 of the pair's norm (the addition theorem) and
// by a rounding, the products and the sum round once each: z is off by (2 * 3 + 2 * 3) M at most.  The norm's factor is off by 15 (21 roundings
// of positive numbers in the mean of the squares, of which the root makes half, and rsqrtf's 4), the reciprocal of s by 2, their product
// and the last sum by one each: y = z / s <= 6 is off by 6 * (12 + 19) = 186, less than kOff.
template <class E, bool kTurn>
__device__ __forceinline__ bool quantise(const Share<E> &u, bool norm, float eps, const Map &m, Coded &out, uint32_t (&doubt)[2])
{
    constexpr float kOff = 0x1p-16f;
    float x[16], r = 1.f;
    unpack(u, x);
    bool ok = true;
    if (norm) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
        for (int d = kLanes / 2; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
        const float mean = fmaf(ss, 1.f / kHeadDim, eps);
        ok = mean > 0x1p-90f && mean < 0x1p90f;            // (squares that underflow are nothing to it)
        r = rsqrtf(mean);
    }
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float lo = x[i], hi = x[8 + i];
        x[i] = kTurn ? fmaf(lo, m.lc[i], -(hi * m.hs[i])) : lo * m.lc[i];
        x[8 + i] = kTurn ? fmaf(hi, m.hc[i], lo * m.ls[i]) : hi * m.hc[i];
        most = max_nan(most, max_nan(fabsf(x[i]), fabsf(x[8 + i])));
    }
    most = head_max_nan(most);
    ok = ok && most > 0x1p-60f && most < 0x1p60f;
    most *= r;
    const float s = scale_of(most * (1.f + 0x1p-18f)), before = __uint_as_float(__float_as_uint(s) - (1u << 18));      // the number before s
    ok = ok && 6.f * before < most * (1.f - 0x1p-18f);
    const float f = r * rcp(s);
    float y[8];
    uint32_t codes[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = fmaf(x[8 * k + i], f, -kOff);
        const uint32_t less = encode8(y);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = fmaf(x[8 * k + i], f, kOff);
        const uint32_t more = encode8(y), some = (less | less >> 1 | less >> 2) & 0x11111111u;
        doubt[k] = (less ^ more) & (0x77777777u | some << 3);                          // (not of the sign of a 0)
        codes[k] = less;
    }
    out = {codes[0], codes[1], bits_of(s)};
    return ok;
}

struct Append {
    const void *k, *v;
    int64_t k_st, k_sh, v_st, v_sh;                                 // elements
    Q4Cache q;
    const void *kw;
    int32_t norm;
    float eps;
    const float *table;                                             // (see pec_rope_table), or NULL
    int64_t n_pos;
    int32_t *status;
};

// A warp = a token and a part of its key heads, or (blockIdx.y from `parts` on) of its value heads; a lane has kDeep of them in flight.
template <class E, bool kTurn, int kDeep>
__global__ void __launch_bounds__(kThreads)
kv_append_q4_kernel(const Append p, const int parts, const int per)
{
    const PagedCache &pc = p.q.c;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane % kLanes, group = lane / kLanes;
    const int32_t t = blockIdx.x * kWarps + warp;
    const bool is_k = (int)blockIdx.y < parts;
    const int h0 = ((int)blockIdx.y - (is_k ? 0 : parts)) * per, h1 = min(h0 + per, p.q.Hkv);
    const int64_t s_in = is_k ? p.k_sh : p.v_sh;
    const E *const src = static_cast<const E *>(is_k ? p.k : p.v) + t * (is_k ? p.k_st : p.v_st) + (h0 + group) * s_in;
    const int mine = t < pc.T ? (h1 - h0 - group + kHeads - 1) / kHeads : 0;         // heads of this lane
    Share<E> u[kDeep] = {};
    auto fetch = [&](int n) {
#pragma unroll
        for (int i = 0; i < kDeep; ++i)
            if (n + i < mine) u[i] = load_share(src + (n + i) * kHeads * s_in, l);
    };
    fetch(0);
    int32_t b, start, end, kv;
    int64_t pos = -1, page = 0, slot = 0;
    if (t < pc.T && find_request(pc, t, p.status, b, start, end, kv)) {
        pos = (int64_t)kv - end + t;
        const int64_t nth = pos / pc.page_size;
        slot = pos - nth * pc.page_size;
        if (pos >= 0 && nth < pc.max_pages && (!kTurn || pos < p.n_pos)) {
            page = pc.table[b * pc.table_stride + nth];             // looked at after the angles
        } else {
            if (lane == 0) raise_status(p.status, PEC_ERR_BAD_INDEX);
            pos = -1;
        }
    }
    const bool turn = is_k && kTurn, math = sizeof(E) == 4 || (is_k && (p.norm || kTurn));   // uniform over the block
    if (pos < 0) return;
    const Change change = {is_k && p.norm, p.eps, is_k && p.norm ? p.kw : nullptr, turn ? p.table : nullptr, p.n_pos, (int32_t)pos};
    Map m;
    if (math) make_map<E>(m, change, l);
    if (page < 0 || page >= pc.num_pages) {
        if (lane == 0) raise_status(p.status, PEC_ERR_BAD_INDEX);
        return;
    }
    const int64_t s_codes = is_k ? pc.k_sh : pc.v_sh, s_scale = is_k ? p.q.ks_sh : p.q.vs_sh;
    uint8_t *codes = (is_k ? p.q.k : p.q.v) + page * (is_k ? pc.k_sp : pc.v_sp) + slot * (is_k ? pc.k_st : pc.v_st) + (h0 + group) * s_codes;
    uint16_t *scale = (is_k ? p.q.ks : p.q.vs) + page * (is_k ? p.q.ks_sp : p.q.vs_sp) + slot * (is_k ? p.q.ks_st : p.q.vs_st) + (h0 + group) * s_scale;
    auto store = [&](const Coded &c, int n) {
        if (n >= mine) return;
        uint8_t *to = codes + n * kHeads * s_codes;
        *reinterpret_cast<uint32_t *>(to + 4 * l) = c.scale == kNaN ? 0u : c.lo;
        *reinterpret_cast<uint32_t *>(to + 32 + 4 * l) = c.scale == kNaN ? 0u : c.hi;
        if (l == 0) scale[n * kHeads * s_scale] = c.scale;
    };
    const int most = (h1 - h0 + kHeads - 1) / kHeads;                // the same for all lanes: shuffles stay converged
    for (int n = 0; n < most; n += kDeep) {
        if (n) fetch(n);
        Coded c[kDeep];
        uint32_t doubt[kDeep][2];
        uint32_t whole = 0;
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            if (math) {
                const bool ok = turn ? quantise<E, true>(u[i], change.norm, p.eps, m, c[i], doubt[i]) : quantise<E, false>(u[i], change.norm, p.eps, m, c[i], doubt[i]);
                if (!ok && n + i < mine) whole |= 1u << i;
                if (!ok || n + i >= mine) doubt[i][0] = doubt[i][1] = 0u;
            } else if constexpr (sizeof(E) == 2) {
                c[i] = quantise(u[i]);
            }
            store(c[i], n + i);
        }
        if (!math) continue;
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            if (__builtin_expect(!__any_sync(0xffffffffu, doubt[i][0] | doubt[i][1]), 1)) continue;
            const Exact<E> exact(n + i < mine ? src + (n + i) * kHeads * s_in : nullptr, change, l);
            exact.some(c[i], doubt[i]);
            store(c[i], n + i);
        }
#pragma unroll 1
        for (uint32_t left = __reduce_or_sync(0xffffffffu, whole); __builtin_expect(left != 0, 0); left &= left - 1) {
            const int i = __ffs(left) - 1;
            const Exact<E> exact(n + i < mine ? src + (n + i) * kHeads * s_in : nullptr, change, l);
            const Coded again = exact.all();
            store(again, whole >> i & 1u ? n + i : mine);
        }
    }
}

struct Read {
    Q4Cache q;
    void *k, *v;
    int64_t k_st, k_sh, v_st, v_sh;                                 // elements
    int32_t *status;
};

// Warp: `tokens` rows in turn, whose pages are looked up at once; blockIdx.y = a part of the key heads, or (from `parts` on) of the value
// heads.  A half warp takes a head, a lane eight channels of it: 64 contiguous bytes in, 256 or 512 out.
template <class E>
__global__ void __launch_bounds__(kThreads)
kv_read_q4_kernel(const Read p, const int parts, const int per, const int tokens)
{
    const PagedCache &pc = p.q.c;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane & 15, half = lane >> 4;
    const int64_t t0 = ((int64_t)blockIdx.x * kWarps + warp) * tokens;
    const bool is_k = (int)blockIdx.y < parts;
    const int h0 = ((int)blockIdx.y - (is_k ? 0 : parts)) * per, h1 = min(h0 + per, p.q.Hkv);
    const int64_t s_codes = is_k ? pc.k_sh : pc.v_sh, s_scale = is_k ? p.q.ks_sh : p.q.vs_sh, s_out = is_k ? p.k_sh : p.v_sh;
    const uint8_t *pool = (is_k ? p.q.k : p.q.v) + 4 * l;
    const uint16_t *scales = is_k ? p.q.ks : p.q.vs;
    E *rows = static_cast<E *>(is_k ? p.k : p.v) + 8 * l;
    const int64_t s_row = is_k ? p.k_st : p.v_st;
    for (int64_t t = t0; t < t0 + tokens && t < pc.T;) {
        int32_t b, start, end, kv;
        if (!find_request(pc, (int32_t)t, p.status, b, start, end, kv)) { ++t; continue; }
        // The rows from t on that are of the same request (the last row by itself: its search is the one that looks at all offsets).
        const int n = t == pc.T - 1 ? 1 : (int)(min(min((int64_t)end, t0 + tokens), (int64_t)pc.T - 1) - t);
        int64_t page = -1, slot = 0;
        if (lane < n) {
            const int64_t pos = (int64_t)kv - end + t + lane, nth = pos / pc.page_size;
            slot = pos - nth * pc.page_size;
            if (pos >= 0 && nth < pc.max_pages) page = pc.table[b * pc.table_stride + nth];
            if (page < 0 || page >= pc.num_pages) {
                raise_status(p.status, PEC_ERR_BAD_INDEX);
                page = -1;
            }
        }
        const int64_t codes_at = page * (is_k ? pc.k_sp : pc.v_sp) + slot * (is_k ? pc.k_st : pc.v_st);
        const int64_t scale_at = page * (is_k ? p.q.ks_sp : p.q.vs_sp) + slot * (is_k ? p.q.ks_st : p.q.vs_st);
        for (int i0 = 0; i0 < n; i0 += kPair) {
            for (int h = h0 + half; h < h1 + half; h += 2 * kRows) {       // (both halves as often)
                uint32_t w[kPair][kRows];
                uint16_t s[kPair][kRows];
                bool good[kPair];
#pragma unroll
                for (int j = 0; j < kPair; ++j) {
                    const int from = min(i0 + j, 31);
                    good[j] = __shfl_sync(0xffffffffu, page, from) >= 0 && i0 + j < n;
                    const uint8_t *codes = pool + __shfl_sync(0xffffffffu, codes_at, from);
                    const uint16_t *scale = scales + __shfl_sync(0xffffffffu, scale_at, from);
#pragma unroll
                    for (int i = 0; i < kRows; ++i) {
                        if (!good[j] || h + 2 * i >= h1) continue;
                        w[j][i] = __ldg(reinterpret_cast<const uint32_t *>(codes + (h + 2 * i) * s_codes));
                        s[j][i] = __ldg(scale + (h + 2 * i) * s_scale);
                    }
                }
#pragma unroll
                for (int j = 0; j < kPair; ++j) {
                    E *out = rows + (t + i0 + j) * s_row;
#pragma unroll
                    for (int i = 0; i < kRows; ++i) {
                        if (!good[j] || h + 2 * i >= h1) continue;
                        uint32_t r[4];
                        decode8(w[j][i], twice(s[j][i]), r);
                        E *to = out + (h + 2 * i) * s_out;
                        if constexpr (sizeof(E) == 2) {
                            *reinterpret_cast<uint4 *>(to) = make_uint4(r[0], r[1], r[2], r[3]);
                        } else {
                            *reinterpret_cast<uint4 *>(to) = make_uint4(r[0] << 16, r[0] & 0xffff0000u, r[1] << 16, r[1] & 0xffff0000u);
                            *reinterpret_cast<uint4 *>(to + 4) = make_uint4(r[2] << 16, r[2] & 0xffff0000u, r[3] << 16, r[3] & 0xffff0000u);
                        }
                    }
                }
            }
        }
        t += n;
    }
}

// Heads of a warp.  (T new tokens of H key heads; limits by T * 2 H, 148 SMs with 32 warps.)
// Appending.  Four where there are too few warps to fill the SMs, and where a token has no more: with norm and rotation, one request, 1024
// tokens of 8 heads 7.8 us with 4 and 7.9 with 8, 2048 10.8 and 9.2; 16384 of 4 heads 36.8, and 43.9 in the form for more (two in flight).
// 32, which share a token's angles, where there are warps enough even so: 1024 of 16 heads 9.4 with 8 and 9.8 with 32, 2048 13.5 and 11.9;
// 1024 of 32 heads 13.4 and 13.7, 2048 25.3 and 19.8; 512 of 64 heads 13.2 and 14.3, 1024 25.3 and 19.9.
inline int append_heads(int64_t T, int64_t H)
{
    const int64_t all = T * 2 * H;
    return H <= 4 || all < (int64_t)148 * 32 * 4 ? 4 : all < (int64_t)148 * 32 * 12 ? 8 : 32;
}
// Reading (head-major and token-major pages alike, but where two figures are given).  To bf16: 256 tokens of 8 heads 3.0 us with 4 and 2.9 with 8,
// 1024 4.0 and 3.4, 8192 13.7 and 10.9; 16384 of 16 heads 32.0 with 8 and 31.7 with 32, 65536 115.8 and 111.1; 8192 of 32 heads 31.9 and 33.2,
// 16384 59.4 and 59.3; 16384 of 64 heads 116.0 and 111.6.  To fp32, whose rows are twice as long: 8192 of 8 heads 21.0 / 19.3 with 8 and
// 19.5 / 20.3 with 4, 16384 36.0 / 32.6 and 31.0 / 30.9, 65536 120.0 / 112.7 and 105.8 / 104.0.
inline int read_heads(int64_t T, int64_t H, bool f32)
{
    const int64_t all = T * 2 * H;
    return f32 ? (all < (int64_t)148 * 32 * 40 ? 8 : 4) : all < (int64_t)148 * 32 * 256 ? 8 : 32;
}
// Rows of a reading warp in turn: more of them in flight, where that leaves warps enough.  One by one, by twos, by fours: 2048 rows of 8 + 8
// heads 4.4, 4.9 and 5.1 us, 4096 8.2, 6.7 and 7.3, 8192 14.5, 11.6 and 10.9, 65536 93.5, 64.5 and 59.7; of 1 + 1 heads 2048 3.8, 4.1 and 4.5,
// 4096 6.1, 5.1 and 5.0, 8192 10.2, 7.7 and 6.6.  With 32 heads a warp 16384 of 64 + 64 heads 136, 112 and 118; with eight of fp32, 2048 of
// 8 + 8 heads 6.8, 7.5 and 7.7, 8192 19.3, 23.2 and 21.8.
inline int tokens_per_warp(int64_t T, int parts, int64_t heads, bool f32)
{
    const int64_t warps = T * 2 * parts;
    if (warps < (int64_t)148 * 40 || (f32 && heads > 4)) return 1;
    return warps < (int64_t)148 * 80 || heads > 8 ? 2 : 4;
}

}  // namespace q4

static bool aligned(const void *p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Strides of [T, H, 128] tensors of channels: at least a head, whole 16-byte vectors.
static int check_rows(const char *who, const int64_t (&s)[4], int64_t esz)
{
    for (const int64_t x : s) {
        if (x < kHeadDim) { set_error("%s: strides must be >= D", who); return PEC_ERR_INVALID_ARG; }
        if ((x * esz) % 16 != 0) { set_error("%s: strides must be multiples of 16 bytes", who); return PEC_ERR_ALIGNMENT; }
    }
    return PEC_OK;
}

int resolve_q4_cache(const char *who, const pec_q4_cache &a, const int32_t *status, Q4Cache &out)
{
    if (!a.k_pages || !a.v_pages || !a.k_scales || !a.v_scales || !a.block_table || !a.cu_q || !a.kv_lens || !status) {
        set_error("%s: k_pages, v_pages, k_scales, v_scales, block_table, cu_q, kv_lens and status must be non-NULL", who);
        return PEC_ERR_INVALID_ARG;
    }
    if (a.D != kHeadDim) { set_error("%s: D=%d unsupported (only 128)", who, a.D); return PEC_ERR_UNSUPPORTED; }
    out.c = {a.k_pages_stride_p, a.k_pages_stride_t, a.k_pages_stride_h, a.v_pages_stride_p, a.v_pages_stride_t, a.v_pages_stride_h,
             a.block_table, a.table_stride, a.max_pages, a.page_size, a.num_pages, a.cu_q, a.kv_lens, a.B, (int32_t)a.T};
    const int rc = check_batch(who, out.c, a.T, a.Hkv);
    if (rc != PEC_OK) return rc;
    for (const int64_t s : {out.c.k_sp, out.c.k_st, out.c.k_sh, out.c.v_sp, out.c.v_st, out.c.v_sh}) {
        if (s < q4::kHeadBytes) { set_error("%s: strides of the pages must be >= D / 2 bytes", who); return PEC_ERR_INVALID_ARG; }
        if (s % 32 != 0) { set_error("%s: strides of the pages must be multiples of 32 bytes", who); return PEC_ERR_ALIGNMENT; }
    }
    for (const int64_t s : {a.k_scales_stride_p, a.k_scales_stride_t, a.k_scales_stride_h, a.v_scales_stride_p, a.v_scales_stride_t, a.v_scales_stride_h})
        if (s < 1) { set_error("%s: strides of the scales must be >= 1", who); return PEC_ERR_INVALID_ARG; }
    if (!aligned(a.k_pages, 32) || !aligned(a.v_pages, 32) || !aligned(a.k_scales, 2) || !aligned(a.v_scales, 2)) {
        set_error("%s: k_pages and v_pages must be 32-byte aligned (scales 2-byte)", who);
        return PEC_ERR_ALIGNMENT;
    }
    if (!aligned(a.block_table, 4) || !aligned(a.cu_q, 4) || !aligned(a.kv_lens, 4) || !aligned(status, 4)) {
        set_error("%s: block_table, cu_q, kv_lens and status must be 4-byte aligned", who);
        return PEC_ERR_ALIGNMENT;
    }
    out.k = static_cast<uint8_t *>(a.k_pages); out.v = static_cast<uint8_t *>(a.v_pages);
    out.ks = static_cast<uint16_t *>(a.k_scales); out.vs = static_cast<uint16_t *>(a.v_scales);
    out.ks_sp = a.k_scales_stride_p; out.ks_st = a.k_scales_stride_t; out.ks_sh = a.k_scales_stride_h;
    out.vs_sp = a.v_scales_stride_p; out.vs_st = a.v_scales_stride_t; out.vs_sh = a.v_scales_stride_h;
    out.Hkv = a.Hkv;
    return PEC_OK;
}

}  // namespace pec

using namespace pec;

extern "C" int pec_kv_append_q4(const pec_kv_append_q4_args *a, void *cuda_stream)
{
    const char *who = "pec_kv_append_q4";
    if (!a) { set_error("%s: args is NULL", who); return PEC_ERR_INVALID_ARG; }
    if (!a->k || !a->v) { set_error("%s: k and v must be non-NULL", who); return PEC_ERR_INVALID_ARG; }
    if (a->dtype != PEC_BF16 && a->dtype != PEC_F32) { set_error("%s: unknown dtype %d", who, a->dtype); return PEC_ERR_UNSUPPORTED; }
    q4::Append p;
    int rc = resolve_q4_cache(who, a->cache, a->status, p.q);
    if (rc != PEC_OK) return rc;
    rc = check_norm_rope(who, a->norm, a->eps, a->rope_table, a->n_pos);
    if (rc != PEC_OK) return rc;
    const int64_t esz = a->dtype == PEC_BF16 ? 2 : 4;
    const int64_t s[4] = {a->k_stride_t, a->k_stride_h, a->v_stride_t, a->v_stride_h};
    rc = check_rows(who, s, esz);
    if (rc != PEC_OK) return rc;
    if (!aligned(a->k, 16) || !aligned(a->v, 16) || !aligned(a->k_weight, 16)) { set_error("%s: k, v and the weight must be 16-byte aligned", who); return PEC_ERR_ALIGNMENT; }
    const int64_t T = a->cache.T;
    if (T == 0) return PEC_OK;
    p.k = a->k; p.v = a->v; p.k_st = s[0]; p.k_sh = s[1]; p.v_st = s[2]; p.v_sh = s[3];
    p.kw = a->k_weight; p.norm = a->norm; p.eps = a->eps; p.table = a->rope_table; p.n_pos = a->n_pos; p.status = a->status;
    const int per = q4::append_heads(T, p.q.Hkv), parts = (p.q.Hkv + per - 1) / per;
    const dim3 grid((unsigned)((T + q4::kWarps - 1) / q4::kWarps), (unsigned)(2 * parts));
    const bool turn = p.table != nullptr;
    const auto pick = [&](auto deep) {
        constexpr int kDeep = decltype(deep)::value;
        return esz == 2 ? (turn ? q4::kv_append_q4_kernel<__nv_bfloat16, true, kDeep> : q4::kv_append_q4_kernel<__nv_bfloat16, false, kDeep>)
                        : (turn ? q4::kv_append_q4_kernel<float, true, kDeep> : q4::kv_append_q4_kernel<float, false, kDeep>);
    };
    const auto kernel = per > q4::kHeads ? pick(std::integral_constant<int, 2>{}) : pick(std::integral_constant<int, 1>{});
    kernel<<<grid, q4::kThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(p, parts, per);
    const cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess) { set_error("%s: launch failed: %s", who, cudaGetErrorString(err)); return PEC_ERR_CUDA; }
    return PEC_OK;
}

extern "C" int pec_kv_read_q4(const pec_kv_read_q4_args *a, void *cuda_stream)
{
    const char *who = "pec_kv_read_q4";
    if (!a) { set_error("%s: args is NULL", who); return PEC_ERR_INVALID_ARG; }
    if (!a->k_out || !a->v_out) { set_error("%s: k_out and v_out must be non-NULL", who); return PEC_ERR_INVALID_ARG; }
    if (a->dtype != PEC_BF16 && a->dtype != PEC_F32) { set_error("%s: unknown dtype %d", who, a->dtype); return PEC_ERR_UNSUPPORTED; }
    q4::Read p;
    int rc = resolve_q4_cache(who, a->cache, a->status, p.q);
    if (rc != PEC_OK) return rc;
    const int64_t esz = a->dtype == PEC_BF16 ? 2 : 4;
    const int64_t s[4] = {a->k_out_stride_t, a->k_out_stride_h, a->v_out_stride_t, a->v_out_stride_h};
    rc = check_rows(who, s, esz);
    if (rc != PEC_OK) return rc;
    if (!aligned(a->k_out, 16) || !aligned(a->v_out, 16)) { set_error("%s: k_out and v_out must be 16-byte aligned", who); return PEC_ERR_ALIGNMENT; }
    const int64_t T = a->cache.T;
    if (T == 0) return PEC_OK;
    p.k = a->k_out; p.v = a->v_out; p.k_st = s[0]; p.k_sh = s[1]; p.v_st = s[2]; p.v_sh = s[3]; p.status = a->status;
    const int per = q4::read_heads(T, p.q.Hkv, esz == 4), parts = (p.q.Hkv + per - 1) / per;
    const int tokens = q4::tokens_per_warp(T, parts, per < p.q.Hkv ? per : p.q.Hkv, esz == 4);
    const dim3 grid((unsigned)((T + q4::kWarps * tokens - 1) / (q4::kWarps * tokens)), (unsigned)(2 * parts));
    const auto kernel = esz == 2 ? q4::kv_read_q4_kernel<__nv_bfloat16> : q4::kv_read_q4_kernel<float>;
    kernel<<<grid, q4::kThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(p, parts, per, tokens);
    const cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess) { set_error("%s: launch failed: %s", who, cudaGetErrorString(err)); return PEC_ERR_CUDA; }
    return PEC_OK;
}
