// Per-head steps between the QKV GEMM and the attention: RMS norm of every query and key head with the rotary encoding in
// the same pass (pec_qk_norm_rope), and the same for new keys on their way into a paged cache, the values beside them
// (pec_kv_append).
//
//     y = x / sqrt(mean(x^2) + eps) * w                         (norm)
//     z[i] = y[i] cos a - y[i + 64] sin a,   z[i + 64] = y[i + 64] cos a + y[i] sin a,   a = p theta^(-2 i / 128)
//
// Bound by memory: every element is read once and written once, rounded once at the end (sums and products in fp32).  A
// head is held by 16 lanes, each with channels 4 l .. 4 l + 3 and their partners 64 on, so that the rotation needs nothing from
// another lane and the sum of squares four shuffles.  With r = 1 / sqrt(..) both steps are one linear map of the pair,
//     z[i] = r (x[i] (w[i] cos) - x[i + 64] (w[i + 64] sin)),   z[i + 64] = r (x[i + 64] (w[i + 64] cos) + x[i] (w[i] sin)),
// whose coefficients depend on the token only and stay in registers while a warp walks the token's heads (two at a time, one per
// half warp, kRows pairs of loads in flight).
// A block takes eight tokens, a warp each.  Its threads work out the tokens' cosines and sines together, with neighbouring lanes
// on neighbouring tokens: the fine part of pec_rope_table's table is stored channel-major, and a token looked up by itself
// touches 128 lines of it for 4 bytes each, more than all the data of eight heads.
// (8192 tokens of 64 + 8 bf16 heads, 302 MB: a block per token with angles per lane and partners by shuffle 132 us; a warp per 16
// heads that looked its angles up itself 83 us, half of the LSU wavefronts spent on the table.)
#include <cmath>
#include <cstdio>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include "pec_host.h"
#include "pec_internal.h"
#include "pec_paged.h"

namespace pec {
namespace heads {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kRows = 4;                     // heads of a half warp in flight

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

struct Turn { const float *table; int64_t n_pos; };            // table of pec_rope_table, or NULL: no rotation
constexpr int kFine = 64 * 64;
constexpr int kLdAngle = 68;                                    // padded row: eight tokens x four channels without bank conflicts
struct Angles { float cos[kWarps][kLdAngle], sin[kWarps][kLdAngle]; int32_t pos[kWarps]; };

// Cosines and sines of the block's tokens (position < 0: none) at p = 64 a + b by the addition theorem (see pec_rope_table).
__device__ __forceinline__ void angles(const Turn &t, Angles &a)
{
    const int tok = threadIdx.x & 7;
    const int32_t p = a.pos[tok];
    if (p < 0) return;
    const int64_t na = (t.n_pos + 63) / 64;
    const float *coarse = t.table + 2 * kFine + (int64_t)(p >> 6) * 64, *fine = t.table + (p & 63);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int i = (threadIdx.x >> 3) + 32 * j;
        const float cc = __ldg(coarse + i), cs = __ldg(coarse + na * 64 + i), fc = __ldg(fine + i * 64), fs = __ldg(fine + kFine + i * 64);
        a.cos[tok][i] = cc * fc - cs * fs;
        a.sin[tok][i] = cs * fc + cc * fs;
    }
}

// The linear map of a lane's four pairs: z_lo = lo * lc - hi * hs, z_hi = hi * hc + lo * ls.
struct Map { float2 lc[2], hs[2], hc[2], ls[2]; };
template <class E>
__device__ __forceinline__ void make_map(Map &m, const void *w, const float *cos, const float *sin, int l)
{
    float wl[4] = {1.f, 1.f, 1.f, 1.f}, wh[4] = {1.f, 1.f, 1.f, 1.f};
    if (w) {
        const Head<E> u = load_head(static_cast<const E *>(w), l);
        Quad<E>::unpack(u.lo, wl);
        Quad<E>::unpack(u.hi, wh);
    }
    float4 c = make_float4(1.f, 1.f, 1.f, 1.f), s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (cos) {
        c = *reinterpret_cast<const float4 *>(cos + 4 * l);
        s = *reinterpret_cast<const float4 *>(sin + 4 * l);
    }
    m.lc[0] = make_float2(wl[0] * c.x, wl[1] * c.y); m.lc[1] = make_float2(wl[2] * c.z, wl[3] * c.w);
    m.ls[0] = make_float2(wl[0] * s.x, wl[1] * s.y); m.ls[1] = make_float2(wl[2] * s.z, wl[3] * s.w);
    m.hc[0] = make_float2(wh[0] * c.x, wh[1] * c.y); m.hc[1] = make_float2(wh[2] * c.z, wh[3] * c.w);
    m.hs[0] = make_float2(-wh[0] * s.x, -wh[1] * s.y); m.hs[1] = make_float2(-wh[2] * s.z, -wh[3] * s.w);
}

// Norm and rotation of one head held by a half warp.  Without a rotation a pair's channels do not meet: 0 times a partner that is not
// finite would be NaN.  (kTurn is the kernels' parameter because a choice here takes ten registers more and a block less per SM.)
template <class E, bool kTurn>
__device__ __forceinline__ void head_math(Head<E> &u, bool norm, float eps, const Map &m)
{
    float a[4], b[4];
    Quad<E>::unpack(u.lo, a);
    Quad<E>::unpack(u.hi, b);
    float2 lo[2] = {make_float2(a[0], a[1]), make_float2(a[2], a[3])}, hi[2] = {make_float2(b[0], b[1]), make_float2(b[2], b[3])};
    if (norm) {
        float2 sq = __fmul2_rn(lo[0], lo[0]);
        sq = __ffma2_rn(lo[1], lo[1], sq);
        sq = __ffma2_rn(hi[0], hi[0], sq);
        sq = __ffma2_rn(hi[1], hi[1], sq);
        float ss = sq.x + sq.y;
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
        const float r = rsqrtf(fmaf(ss, 1.f / kHeadDim, eps));
        const float2 r2 = make_float2(r, r);
#pragma unroll
        for (int i = 0; i < 2; ++i) { lo[i] = __fmul2_rn(lo[i], r2); hi[i] = __fmul2_rn(hi[i], r2); }
    }
    float zl[4], zh[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float2 x = kTurn ? __ffma2_rn(lo[i], m.lc[i], __fmul2_rn(hi[i], m.hs[i])) : __fmul2_rn(lo[i], m.lc[i]);
        const float2 y = kTurn ? __ffma2_rn(hi[i], m.hc[i], __fmul2_rn(lo[i], m.ls[i])) : __fmul2_rn(hi[i], m.hc[i]);
        zl[2 * i] = x.x; zl[2 * i + 1] = x.y; zh[2 * i] = y.x; zh[2 * i + 1] = y.y;
    }
    u.lo = Quad<E>::pack(zl);
    u.hi = Quad<E>::pack(zh);
}

struct NormRope {
    const void *q, *k;
    void *qo, *ko;
    int64_t q_st, q_sh, k_st, k_sh, qo_st, qo_sh, ko_st, ko_sh;     // elements
    int32_t T, Hq, Hkv;
    const void *qw, *kw;
    int32_t norm;
    float eps;
    Turn turn;
    const int32_t *positions;
    int64_t pos0;
    int32_t *status;
};

// Block: eight tokens; blockIdx.y = a part of `per` query heads, or (from q_parts on) of key heads.
template <class E, bool kTurn>
__global__ void __launch_bounds__(kThreads)
norm_rope_kernel(const NormRope p, const int q_parts, const int per)
{
    __shared__ __align__(16) Angles sh;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane & 15, half = lane >> 4;
    const int32_t t = blockIdx.x * kWarps + warp;
    const bool is_q = (int)blockIdx.y < q_parts;
    const int h0 = ((int)blockIdx.y - (is_q ? 0 : q_parts)) * per, h1 = min(h0 + per, is_q ? p.Hq : p.Hkv);
    const int64_t sh_in = is_q ? p.q_sh : p.k_sh, sh_out = is_q ? p.qo_sh : p.ko_sh;
    const E *src = static_cast<const E *>(is_q ? p.q : p.k) + t * (is_q ? p.q_st : p.k_st) + (h0 + half) * sh_in;
    E *dst = static_cast<E *>(is_q ? p.qo : p.ko) + t * (is_q ? p.qo_st : p.ko_st) + (h0 + half) * sh_out;

    // Loads and stores run over the half warp's heads h0 + half, + 2, ...; `src` and `dst` are at the next one.
    int left = t < p.T ? (h1 - h0 - half + 1) / 2 : 0;              // heads not yet loaded
    auto fetch = [&](Head<E> (&u)[kRows]) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (i < left) u[i] = load_head(src, l);
            src += 2 * sh_in;
        }
        left -= kRows;
    };
    Head<E> u[kRows] = {};
    int todo = left;
    fetch(u);
    // A negative position marks a padding row; one past the table is reported.
    int64_t pos = -1;
    if (t < p.T) pos = p.positions ? (int64_t)p.positions[t] : p.pos0 + t;
    if (kTurn && pos >= p.turn.n_pos) {
        if (lane == 0) raise_status(p.status, PEC_ERR_BAD_INDEX);
        pos = -1;
    }
    if (kTurn) {
        if (lane == 0) sh.pos[warp] = (int32_t)pos;
        __syncthreads();
        angles(p.turn, sh);
        __syncthreads();
    }
    if (pos < 0) return;
    Map m;
    make_map<E>(m, p.norm ? (is_q ? p.qw : p.kw) : nullptr, kTurn ? sh.cos[warp] : nullptr, sh.sin[warp], l);
    const int rounds = ((h1 - h0 + 1) / 2 + kRows - 1) / kRows;     // the same for both halves: shuffles stay converged
    for (int r = 0; r < rounds; ++r) {
        if (r) fetch(u);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            head_math<E, kTurn>(u[i], p.norm != 0, p.eps, m);
            if (i < todo) store_head(dst, l, u[i]);
            dst += 2 * sh_out;
        }
        todo -= kRows;
    }
}

struct Append {
    const void *k, *v;
    int64_t k_st, k_sh, v_st, v_sh;                                 // elements
    void *k_pages, *v_pages;
    PagedCache c;
    int32_t Hkv;
    const void *kw;
    int32_t norm;
    float eps;
    Turn turn;
    int32_t *status;
};

// As above; blockIdx.y = a part of the key heads, or (from `parts` on) of the value heads, which are copied.
template <class E, bool kTurn>
__global__ void __launch_bounds__(kThreads)
kv_append_kernel(const Append p, const int parts, const int per)
{
    __shared__ __align__(16) Angles sh;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane & 15, half = lane >> 4;
    const int32_t t = blockIdx.x * kWarps + warp;
    const bool is_k = (int)blockIdx.y < parts;
    const int h0 = ((int)blockIdx.y - (is_k ? 0 : parts)) * per, h1 = min(h0 + per, p.Hkv);
    const int64_t s_in = is_k ? p.k_sh : p.v_sh, s_out = is_k ? p.c.k_sh : p.c.v_sh;
    const E *src = static_cast<const E *>(is_k ? p.k : p.v) + t * (is_k ? p.k_st : p.v_st) + (h0 + half) * s_in;

    int left = t < p.c.T ? (h1 - h0 - half + 1) / 2 : 0;
    auto fetch = [&](Head<E> (&u)[kRows]) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (i < left) u[i] = load_head(src, l);
            src += 2 * s_in;
        }
        left -= kRows;
    };
    Head<E> u[kRows] = {};
    int todo = left;
    fetch(u);
    int32_t b, start, end, kv;
    int64_t pos = -1, page = 0, slot = 0;
    if (t < p.c.T && find_request(p.c, t, p.status, b, start, end, kv)) {
        pos = (int64_t)kv - end + t;
        const int64_t nth = pos / p.c.page_size;
        slot = pos - nth * p.c.page_size;
        if (pos >= 0 && nth < p.c.max_pages && (!kTurn || pos < p.turn.n_pos)) {
            page = p.c.table[b * p.c.table_stride + nth];           // looked at when the angles are done
        } else {
            if (lane == 0) raise_status(p.status, PEC_ERR_BAD_INDEX);
            pos = -1;
        }
    }
    const bool turn = is_k && kTurn, math = is_k && (p.norm || kTurn);   // uniform over the block
    if (turn) {
        if (lane == 0) sh.pos[warp] = (int32_t)pos;
        __syncthreads();
        angles(p.turn, sh);
        __syncthreads();
    }
    if (pos < 0) return;
    if (page < 0 || page >= p.c.num_pages) {
        if (lane == 0) raise_status(p.status, PEC_ERR_BAD_INDEX);
        return;
    }
    Map m;
    make_map<E>(m, math && p.norm ? p.kw : nullptr, turn ? sh.cos[warp] : nullptr, sh.sin[warp], l);
    E *dst = static_cast<E *>(is_k ? p.k_pages : p.v_pages) + page * (is_k ? p.c.k_sp : p.c.v_sp) + slot * (is_k ? p.c.k_st : p.c.v_st) +
             (h0 + half) * s_out;
    const int rounds = ((h1 - h0 + 1) / 2 + kRows - 1) / kRows;
    for (int r = 0; r < rounds; ++r) {
        if (r) fetch(u);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (math) head_math<E, kTurn>(u[i], p.norm != 0, p.eps, m);
            if (i < todo) store_head(dst, l, u[i]);
            dst += 2 * s_out;
        }
        todo -= kRows;
    }
}

// Heads of a part: as many as a warp loads at once (8) where the call is too small to fill the GPU otherwise (a warp of each of 148 SMs'
// 32 and 32 heads), four times that where it is not, so that the angles are worked out for more heads.  Both sides (parts of 8 / 32)
// at T * H = 20000, 75000, 150000, 300000, 600000: norm of 72 heads 5.0 / 7.3, 12.6 / 12.8, 21.0 / 17.5, 35.3 / 30.8, 64.9 / 55.1 us, of 40
// heads 4.9 / 7.5, 13.0 / 13.2, 21.8 / 18.6, 38.6 / 33.1, 71.4 / 61.2; append of 32 heads 4.8 / 7.6, 9.4 / 9.2, 17.8 / 14.5, 31.8 / 26.8,
// 62.5 / 54.2, of 8 heads (one part either way) the same.  Ten heads would gain at every size: 6.8 / 6.2 to 118 / 98.6.
inline int heads_per_part(int64_t T, int64_t H) { return T * H < (int64_t)148 * 32 * 32 ? 2 * kRows : 8 * kRows; }

}  // namespace heads

static inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Row strides of [T, H, 128] tensors: at least a head, whole 16-byte vectors.
static int check_strides(const char *who, const int64_t *s, int n, int64_t esz)
{
    for (int i = 0; i < n; ++i) {
        if (s[i] < kHeadDim) { set_error("%s: strides must be >= D", who); return PEC_ERR_INVALID_ARG; }
        if ((s[i] * esz) % 16 != 0) { set_error("%s: strides must be multiples of 16 bytes", who); return PEC_ERR_ALIGNMENT; }
    }
    return PEC_OK;
}

static int check_norm_rope(const char *who, int32_t norm, float eps, const float *table, int64_t n_pos)
{
    if (norm != 0 && norm != 1) { set_error("%s: norm must be 0 or 1", who); return PEC_ERR_INVALID_ARG; }
    if (norm && !(eps > 0.f && std::isfinite(eps))) { set_error("%s: eps must be finite and > 0", who); return PEC_ERR_INVALID_ARG; }
    if (table && (n_pos < 1 || n_pos >= ((int64_t)1 << 31))) { set_error("%s: the rotary table needs 1 <= n_pos < 2^31", who); return PEC_ERR_INVALID_ARG; }
    if (!aligned16(table)) { set_error("%s: the rotary table must be 16-byte aligned", who); return PEC_ERR_ALIGNMENT; }
    return PEC_OK;
}

int check_paged_cache(const char *who, const void *k_pages, const void *v_pages, const PagedCache &c, int64_t T, int32_t Hkv,
                      int32_t D, int32_t dtype, const int32_t *status)
{
    if (!k_pages || !v_pages || !c.table || !c.cu_q || !c.kv_lens || !status) {
        set_error("%s: k_pages, v_pages, block_table, cu_q, kv_lens and status must be non-NULL", who);
        return PEC_ERR_INVALID_ARG;
    }
    if (D != kHeadDim) { set_error("%s: D=%d unsupported (only 128)", who, D); return PEC_ERR_UNSUPPORTED; }
    if (dtype != PEC_BF16 && dtype != PEC_F32) { set_error("%s: unknown dtype %d", who, dtype); return PEC_ERR_UNSUPPORTED; }
    if (Hkv < 1 || Hkv > 65535) { set_error("%s: need 1 <= Hkv <= 65535 (got %d)", who, Hkv); return PEC_ERR_INVALID_ARG; }
    if (c.B < 1 || T < 0) { set_error("%s: need B >= 1 and T >= 0", who); return PEC_ERR_INVALID_ARG; }
    if (c.B > (1 << 20) || T > ((int64_t)1 << 30)) { set_error("%s: more than 2^20 requests or 2^30 tokens unsupported", who); return PEC_ERR_UNSUPPORTED; }
    if (c.page_size < 8 || c.page_size % 8 != 0 || c.page_size > (1 << 16)) {
        set_error("%s: page_size must be a multiple of 8, at most 65536 (got %d)", who, c.page_size);
        return PEC_ERR_UNSUPPORTED;
    }
    if (c.num_pages < 1 || c.num_pages >= ((int64_t)1 << 31)) { set_error("%s: need 1 <= num_pages < 2^31", who); return PEC_ERR_INVALID_ARG; }
    if (c.max_pages < 1 || (c.B > 1 && c.table_stride < c.max_pages)) {
        set_error("%s: need max_pages >= 1 and table_stride >= max_pages", who);
        return PEC_ERR_INVALID_ARG;
    }
    if ((int64_t)c.max_pages * c.page_size > ((int64_t)1 << 30)) { set_error("%s: more than 2^30 tokens of one request unsupported", who); return PEC_ERR_UNSUPPORTED; }
    const int64_t esz = dtype == PEC_BF16 ? 2 : 4, s[6] = {c.k_sp, c.k_st, c.k_sh, c.v_sp, c.v_st, c.v_sh};
    const int rc = check_strides(who, s, 6, esz);
    if (rc != PEC_OK) return rc;
    if (!aligned16(k_pages) || !aligned16(v_pages)) { set_error("%s: k_pages and v_pages must be 16-byte aligned", who); return PEC_ERR_ALIGNMENT; }
    if ((reinterpret_cast<uintptr_t>(c.table) | reinterpret_cast<uintptr_t>(c.cu_q) | reinterpret_cast<uintptr_t>(c.kv_lens) |
         reinterpret_cast<uintptr_t>(status)) & 3u) {
        set_error("%s: block_table, cu_q, kv_lens and status must be 4-byte aligned", who);
        return PEC_ERR_ALIGNMENT;
    }
    return PEC_OK;
}

}  // namespace pec

using namespace pec;

extern "C" int pec_qk_norm_rope(const pec_norm_rope_args *a, void *cuda_stream)
{
    const char *who = "pec_qk_norm_rope";
    if (!a) { set_error("%s: args is NULL", who); return PEC_ERR_INVALID_ARG; }
    if (a->T < 0 || a->Hq < 0 || a->Hkv < 0 || a->Hq + (int64_t)a->Hkv < 1) { set_error("%s: need T, Hq, Hkv >= 0 and at least one head", who); return PEC_ERR_INVALID_ARG; }
    if ((a->Hq > 0 && (!a->q || !a->q_out)) || (a->Hkv > 0 && (!a->k || !a->k_out))) { set_error("%s: q, q_out (k, k_out) must be non-NULL where there are such heads", who); return PEC_ERR_INVALID_ARG; }
    if (a->D != kHeadDim) { set_error("%s: D=%d unsupported (only 128)", who, a->D); return PEC_ERR_UNSUPPORTED; }
    if (a->dtype != PEC_BF16 && a->dtype != PEC_F32) { set_error("%s: unknown dtype %d", who, a->dtype); return PEC_ERR_UNSUPPORTED; }
    if (a->T > ((int64_t)1 << 30) || a->Hq > 65535 || a->Hkv > 65535) { set_error("%s: more than 2^30 tokens or 65535 heads unsupported", who); return PEC_ERR_UNSUPPORTED; }
    int rc = check_norm_rope(who, a->norm, a->eps, a->rope_table, a->n_pos);
    if (rc != PEC_OK) return rc;
    if (!a->status) { set_error("%s: the status word must be non-NULL", who); return PEC_ERR_INVALID_ARG; }
    if (!a->positions && (a->pos0 < 0 || (a->rope_table && a->pos0 > a->n_pos - a->T))) {
        set_error("%s: positions pos0 .. pos0 + T - 1 must lie inside the table", who);
        return PEC_ERR_INVALID_ARG;
    }
    const int64_t esz = a->dtype == PEC_BF16 ? 2 : 4;
    const int64_t sq[4] = {a->q_stride_t, a->q_stride_h, a->q_out_stride_t, a->q_out_stride_h};
    const int64_t sk[4] = {a->k_stride_t, a->k_stride_h, a->k_out_stride_t, a->k_out_stride_h};
    if (a->Hq > 0 && (rc = check_strides(who, sq, 4, esz)) != PEC_OK) return rc;
    if (a->Hkv > 0 && (rc = check_strides(who, sk, 4, esz)) != PEC_OK) return rc;
    if ((a->Hq > 0 && (!aligned16(a->q) || !aligned16(a->q_out))) || (a->Hkv > 0 && (!aligned16(a->k) || !aligned16(a->k_out))) ||
        !aligned16(a->q_weight) || !aligned16(a->k_weight) ||
        ((reinterpret_cast<uintptr_t>(a->positions) | reinterpret_cast<uintptr_t>(a->status)) & 3u)) {
        set_error("%s: tensors and weights must be 16-byte aligned (positions, status 4-byte)", who);
        return PEC_ERR_ALIGNMENT;
    }
    if ((a->Hq > 0 && a->q == a->q_out && (sq[0] != sq[2] || sq[1] != sq[3])) ||
        (a->Hkv > 0 && a->k == a->k_out && (sk[0] != sk[2] || sk[1] != sk[3]))) {
        set_error("%s: in place means the same strides", who);
        return PEC_ERR_INVALID_ARG;
    }
    if (a->T == 0) return PEC_OK;
    heads::NormRope p;
    p.q = a->q; p.k = a->k; p.qo = a->q_out; p.ko = a->k_out;
    p.q_st = sq[0]; p.q_sh = sq[1]; p.qo_st = sq[2]; p.qo_sh = sq[3];
    p.k_st = sk[0]; p.k_sh = sk[1]; p.ko_st = sk[2]; p.ko_sh = sk[3];
    p.T = (int32_t)a->T; p.Hq = a->Hq; p.Hkv = a->Hkv;
    p.qw = a->q_weight; p.kw = a->k_weight; p.norm = a->norm; p.eps = a->eps;
    p.turn = {a->rope_table, a->n_pos};
    p.positions = a->positions; p.pos0 = a->rope_table ? a->pos0 : 0; p.status = a->status;      // (no position matters without a table)
    const int per = heads::heads_per_part(p.T, p.Hq + p.Hkv), q_parts = (p.Hq + per - 1) / per;
    const dim3 grid((unsigned)((p.T + heads::kWarps - 1) / heads::kWarps), (unsigned)(q_parts + (p.Hkv + per - 1) / per));
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const bool turn = p.turn.table != nullptr;
    const auto kernel = esz == 2 ? (turn ? heads::norm_rope_kernel<__nv_bfloat16, true> : heads::norm_rope_kernel<__nv_bfloat16, false>)
                                 : (turn ? heads::norm_rope_kernel<float, true> : heads::norm_rope_kernel<float, false>);
    kernel<<<grid, heads::kThreads, 0, stream>>>(p, q_parts, per);
    const cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess) { set_error("%s: launch failed: %s", who, cudaGetErrorString(err)); return PEC_ERR_CUDA; }
    return PEC_OK;
}

extern "C" int pec_kv_append(const pec_kv_append_args *a, void *cuda_stream)
{
    const char *who = "pec_kv_append";
    if (!a) { set_error("%s: args is NULL", who); return PEC_ERR_INVALID_ARG; }
    if (!a->k || !a->v) { set_error("%s: k and v must be non-NULL", who); return PEC_ERR_INVALID_ARG; }
    heads::Append p;
    p.c = {a->k_pages_stride_p, a->k_pages_stride_t, a->k_pages_stride_h, a->v_pages_stride_p, a->v_pages_stride_t, a->v_pages_stride_h,
           a->block_table, a->table_stride, a->max_pages, a->page_size, a->num_pages, a->cu_q, a->kv_lens, a->B, (int32_t)a->T};
    int rc = check_paged_cache(who, a->k_pages, a->v_pages, p.c, a->T, a->Hkv, a->D, a->dtype, a->status);
    if (rc != PEC_OK) return rc;
    rc = check_norm_rope(who, a->norm, a->eps, a->rope_table, a->n_pos);
    if (rc != PEC_OK) return rc;
    const int64_t esz = a->dtype == PEC_BF16 ? 2 : 4;
    const int64_t s[4] = {a->k_stride_t, a->k_stride_h, a->v_stride_t, a->v_stride_h};
    rc = check_strides(who, s, 4, esz);
    if (rc != PEC_OK) return rc;
    if (!aligned16(a->k) || !aligned16(a->v) || !aligned16(a->k_weight)) { set_error("%s: k, v and the weight must be 16-byte aligned", who); return PEC_ERR_ALIGNMENT; }
    if (a->T == 0) return PEC_OK;
    p.k = a->k; p.v = a->v; p.k_st = s[0]; p.k_sh = s[1]; p.v_st = s[2]; p.v_sh = s[3];
    p.k_pages = a->k_pages; p.v_pages = a->v_pages; p.Hkv = a->Hkv;
    p.kw = a->k_weight; p.norm = a->norm; p.eps = a->eps; p.turn = {a->rope_table, a->n_pos}; p.status = a->status;
    const int per = heads::heads_per_part(a->T, 2 * (int64_t)a->Hkv), parts = (a->Hkv + per - 1) / per;
    const dim3 grid((unsigned)((a->T + heads::kWarps - 1) / heads::kWarps), (unsigned)(2 * parts));
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const bool turn = p.turn.table != nullptr;
    const auto kernel = esz == 2 ? (turn ? heads::kv_append_kernel<__nv_bfloat16, true> : heads::kv_append_kernel<__nv_bfloat16, false>)
                                 : (turn ? heads::kv_append_kernel<float, true> : heads::kv_append_kernel<float, false>);
    kernel<<<grid, heads::kThreads, 0, stream>>>(p, parts, per);
    const cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess) { set_error("%s: launch failed: %s", who, cudaGetErrorString(err)); return PEC_ERR_CUDA; }
    return PEC_OK;
}
