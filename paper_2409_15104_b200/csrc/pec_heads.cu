// Per-head steps between the QKV GEMM and the attention: RMS norm of every query and key head with the rotary encoding in
// the same pass (pec_qk_norm_rope), and the same for new keys on their way into a paged cache, the values beside them
// (pec_kv_append).
//
//     y = x / sqrt(mean(x^2) + eps) * w                         (norm)
//     z[i] = y[i] cos a - y[i + 64] sin a,   z[i + 64] = y[i + 64] cos a + y[i] sin a,   a = p theta^(-2 i / 128)
//
// Bound by memory: every element is read once and written once, rounded once at the end (sums and products in fp32).  A
// head is held by 16 lanes, each with channels 4 l .. 4 l + 3 and their partners 64 on, so that the rotation needs nothing from
// another lane and the sum of squares four shuffles.  The angle depends on the token only: a warp takes some heads of one
// token (two at a time, one per half warp, the loads of kRows pairs in flight), and its lanes work out the cosines and sines of
// their four channels once, from the two-level table of pec_rope_table.  Nothing goes through shared memory.
// (Measured on 8192 tokens of 64 + 8 bf16 heads, 302 MB: a block per token with the angles in shared memory and the partners by
// shuffle took 132 us.)
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

// Cosines and sines of channels 4 l .. 4 l + 3 at position p = 64 a + b by the addition theorem (see pec_rope_table).
__device__ __forceinline__ void angles(const Turn &t, int32_t p, int l, float (&c)[4], float (&s)[4])
{
    const int64_t na = (t.n_pos + 63) / 64;
    const int b = p & 63;
    const float *coarse = t.table + 2 * kFine + (int64_t)(p >> 6) * 64 + 4 * l, *fine = t.table + 4 * l * 64 + b;
    const float4 c4 = __ldg(reinterpret_cast<const float4 *>(coarse)), s4 = __ldg(reinterpret_cast<const float4 *>(coarse + na * 64));
    const float cc[4] = {c4.x, c4.y, c4.z, c4.w}, cs[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float fc = __ldg(fine + i * 64), fs = __ldg(fine + kFine + i * 64);
        c[i] = cc[i] * fc - cs[i] * fs;
        s[i] = cs[i] * fc + cc[i] * fs;
    }
}

// Norm and rotation of one head held by a half warp.
template <class E>
__device__ __forceinline__ void head_math(Head<E> &u, bool norm, const float (&wl)[4], const float (&wh)[4], float eps,
                                          bool turn, const float (&c)[4], const float (&s)[4])
{
    float lo[4], hi[4];
    Quad<E>::unpack(u.lo, lo);
    Quad<E>::unpack(u.hi, hi);
    if (norm) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) { ss = fmaf(lo[i], lo[i], ss); ss = fmaf(hi[i], hi[i], ss); }
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
        const float r = rsqrtf(ss * (1.f / kHeadDim) + eps);
#pragma unroll
        for (int i = 0; i < 4; ++i) { lo[i] = lo[i] * r * wl[i]; hi[i] = hi[i] * r * wh[i]; }
    }
    if (turn) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = lo[i], b = hi[i];
            lo[i] = fmaf(a, c[i], -b * s[i]);
            hi[i] = fmaf(b, c[i], a * s[i]);
        }
    }
    u.lo = Quad<E>::pack(lo);
    u.hi = Quad<E>::pack(hi);
}

template <class E>
__device__ __forceinline__ void load_weight(const void *w, int l, float (&lo)[4], float (&hi)[4])
{
    if (w) {
        const Head<E> u = load_head(static_cast<const E *>(w), l);
        Quad<E>::unpack(u.lo, lo);
        Quad<E>::unpack(u.hi, hi);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) lo[i] = hi[i] = 1.f;
    }
}

struct NormRope {
    const void *q, *k;
    void *qo, *ko;
    int64_t q_st, q_sh, k_st, k_sh, qo_st, qo_sh, ko_st, ko_sh;     // elements
    int32_t T, Hq, H;                                               // H = query and key heads
    const void *qw, *kw;
    int32_t norm;
    float eps;
    Turn turn;
    const int32_t *positions;
    int64_t pos0;
    int32_t *status;
};

// Warp: heads [h0, h0 + per) of one token.
template <class E>
__global__ void __launch_bounds__(kThreads)
norm_rope_kernel(const NormRope p, const int parts, const int per)
{
    const int lane = threadIdx.x & 31, l = lane & 15, half = lane >> 4;
    const int64_t unit = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    const int32_t t = (int32_t)(unit / parts);
    if (t >= p.T) return;
    const int h0 = (int)(unit - (int64_t)t * parts) * per, h1 = min(h0 + per, p.H);

    auto fetch = [&](int base, Head<E> (&u)[kRows]) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int h = base + half + 2 * i;
            if (h < h1)
                u[i] = load_head(h < p.Hq ? static_cast<const E *>(p.q) + t * p.q_st + h * p.q_sh
                                          : static_cast<const E *>(p.k) + t * p.k_st + (h - p.Hq) * p.k_sh, l);
        }
    };
    Head<E> u[kRows] = {};
    fetch(h0, u);
    // A negative position marks a padding row; one past the table is reported.
    const int64_t pos = p.positions ? (int64_t)p.positions[t] : p.pos0 + t;
    if (pos < 0) return;
    if (p.turn.table && pos >= p.turn.n_pos) {
        if (lane == 0) raise_status(p.status, PEC_ERR_BAD_INDEX);
        return;
    }
    float c[4] = {}, s[4] = {}, ql[4], qh[4], kl[4], kh[4];
    if (p.turn.table) angles(p.turn, (int32_t)pos, l, c, s);
    load_weight<E>(p.norm && h0 < p.Hq ? p.qw : nullptr, l, ql, qh);
    load_weight<E>(p.norm && h1 > p.Hq ? p.kw : nullptr, l, kl, kh);
    for (int base = h0; base < h1; base += 2 * kRows) {
        if (base != h0) fetch(base, u);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int h = base + half + 2 * i;
            const bool is_q = h < p.Hq;
            float wl[4], wh[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) { wl[x] = is_q ? ql[x] : kl[x]; wh[x] = is_q ? qh[x] : kh[x]; }
            head_math<E>(u[i], p.norm != 0, wl, wh, p.eps, p.turn.table != nullptr, c, s);
            if (h < h1)
                store_head(is_q ? static_cast<E *>(p.qo) + t * p.qo_st + h * p.qo_sh
                                : static_cast<E *>(p.ko) + t * p.ko_st + (h - p.Hq) * p.ko_sh, l, u[i]);
        }
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

// As above over a token's key heads and then its value heads.
template <class E>
__global__ void __launch_bounds__(kThreads)
kv_append_kernel(const Append p, const int parts, const int per)
{
    const int lane = threadIdx.x & 31, l = lane & 15, half = lane >> 4;
    const int64_t unit = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    const int32_t t = (int32_t)(unit / parts);
    if (t >= p.c.T) return;
    const int H = 2 * p.Hkv, h0 = (int)(unit - (int64_t)t * parts) * per, h1 = min(h0 + per, H);

    auto fetch = [&](int base, Head<E> (&u)[kRows]) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int h = base + half + 2 * i;
            if (h < h1)
                u[i] = load_head(h < p.Hkv ? static_cast<const E *>(p.k) + t * p.k_st + h * p.k_sh
                                           : static_cast<const E *>(p.v) + t * p.v_st + (h - p.Hkv) * p.v_sh, l);
        }
    };
    Head<E> u[kRows] = {};
    fetch(h0, u);
    float wl[4], wh[4], c[4] = {}, s[4] = {};
    const bool math = h0 < p.Hkv && (p.norm || p.turn.table);      // values alone, or keys as they are: a copy
    load_weight<E>(math && p.norm ? p.kw : nullptr, l, wl, wh);
    int32_t b, end;
    if (!find_request(p.c, t, p.status, b, end)) return;
    const int64_t pos = (int64_t)p.c.kv_lens[b] - end + t, nth = pos / p.c.page_size;
    bool ok = pos >= 0 && nth < p.c.max_pages && (!p.turn.table || pos < p.turn.n_pos);
    int64_t page = -1;
    if (ok) {
        page = p.c.table[b * p.c.table_stride + nth];
        ok = page >= 0 && page < p.c.num_pages;
    }
    if (!ok) {
        if (lane == 0) raise_status(p.status, PEC_ERR_BAD_INDEX);
        return;
    }
    if (math && p.turn.table) angles(p.turn, (int32_t)pos, l, c, s);
    const int64_t slot = pos - nth * p.c.page_size;
    E *k_slot = static_cast<E *>(p.k_pages) + page * p.c.k_sp + slot * p.c.k_st;
    E *v_slot = static_cast<E *>(p.v_pages) + page * p.c.v_sp + slot * p.c.v_st;
    for (int base = h0; base < h1; base += 2 * kRows) {
        if (base != h0) fetch(base, u);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int h = base + half + 2 * i;
            const bool is_k = h < p.Hkv;
            if (math) {                                             // uniform over the warp; a pair may be a key and a value
                Head<E> z = u[i];
                head_math<E>(z, p.norm != 0, wl, wh, p.eps, p.turn.table != nullptr, c, s);
                if (is_k) u[i] = z;
            }
            if (h < h1) store_head(is_k ? k_slot + h * p.c.k_sh : v_slot + (h - p.Hkv) * p.c.v_sh, l, u[i]);
        }
    }
}

// Parts that a token's H heads are dealt to, one warp each: 16 heads a warp where there are tokens enough to fill the GPU (the
// angles are then worked out once for 16 heads), fewer where there are not, down to one pair.
inline void deal(int64_t T, int64_t H, int &parts, int &per)
{
    int64_t n = T * H / (148 * 32);
    n = n < 2 ? 2 : (n > 16 ? 16 : (n + 1) / 2 * 2);
    per = (int)(n < H ? n : H);
    parts = (int)((H + per - 1) / per);
}

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
    if (!a->positions && (a->pos0 < 0 || (a->rope_table && a->pos0 + a->T > a->n_pos))) {
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
    p.T = (int32_t)a->T; p.Hq = a->Hq; p.H = a->Hq + a->Hkv;
    p.qw = a->q_weight; p.kw = a->k_weight; p.norm = a->norm; p.eps = a->eps;
    p.turn = {a->rope_table, a->n_pos};
    p.positions = a->positions; p.pos0 = a->pos0; p.status = a->status;
    int parts, per;
    heads::deal(p.T, p.H, parts, per);
    const int64_t blocks = ((int64_t)p.T * parts + heads::kWarps - 1) / heads::kWarps;
    if (blocks > 0x7fffffff) { set_error("%s: grid too large", who); return PEC_ERR_UNSUPPORTED; }
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (esz == 2) heads::norm_rope_kernel<__nv_bfloat16><<<(unsigned)blocks, heads::kThreads, 0, stream>>>(p, parts, per);
    else          heads::norm_rope_kernel<float><<<(unsigned)blocks, heads::kThreads, 0, stream>>>(p, parts, per);
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
    int parts, per;
    heads::deal(a->T, 2 * (int64_t)a->Hkv, parts, per);
    const int64_t blocks = (a->T * parts + heads::kWarps - 1) / heads::kWarps;
    if (blocks > 0x7fffffff) { set_error("%s: grid too large", who); return PEC_ERR_UNSUPPORTED; }
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (esz == 2) heads::kv_append_kernel<__nv_bfloat16><<<(unsigned)blocks, heads::kThreads, 0, stream>>>(p, parts, per);
    else          heads::kv_append_kernel<float><<<(unsigned)blocks, heads::kThreads, 0, stream>>>(p, parts, per);
    const cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess) { set_error("%s: launch failed: %s", who, cudaGetErrorString(err)); return PEC_ERR_CUDA; }
    return PEC_OK;
}
