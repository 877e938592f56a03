// A paged K/V cache held in 4 bits: new keys (normalised and rotated on the way) and values into it (pec_kv_append_q4), and what it
// holds back into packed tensors (pec_kv_read_q4).
//
//     s = least number of six significant bits with 6 s >= max |z|,   code = nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 to |z| / s,
//     z = the head's channels; for keys after norm and rotation (see pec_heads.cu), which are worked out in fp64
//
// Both are bound by memory: a head of bf16 is 256 bytes on one side and 66 on the other.
//
// Which code is the nearest is decided exactly.  bf16 channels that are quantised as they are: x / s is either a border between two
// codes or 2^-10 away from it, while the product with the rounded reciprocal is off by 2^-23: rounded to 16 bits it is a border where x / s is
// one, and on its side elsewhere.  Everything else goes through fp64: z times 1 / s, rounded to 41 bits for the same reason (an
// fp32 x is 2^-25 away from a border at least), then to fp32 with the last bit set where anything was cut off, so that nothing
// becomes a border that is none.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include "pec_head_io.cuh"
#include "pec_host.h"
#include "pec_internal.h"
#include "pec_q4.cuh"

namespace pec {
namespace q4 {
using heads::Head;
using heads::Quad;
using heads::load_head;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kRows = 4;                     // heads of a half warp in flight
constexpr int kLdAngle = 66;

struct Turn { const float *table; int64_t n_pos; };
struct Angles { double cos[kWarps][kLdAngle], sin[kWarps][kLdAngle]; int32_t pos[kWarps]; };

// Cosines and sines of the block's tokens (position < 0: none) at p = 64 a + b by the addition theorem (see pec_rope_table).
__device__ __forceinline__ void angles(const Turn &t, Angles &a)
{
    const int tok = threadIdx.x & 7;
    const int32_t p = a.pos[tok];
    if (p < 0) return;
    const int64_t na = (t.n_pos + 63) / 64;
    const float *coarse = t.table + 2 * 4096 + (int64_t)(p >> 6) * 64, *fine = t.table + (p & 63);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int i = (threadIdx.x >> 3) + 32 * j;
        const double cc = __ldg(coarse + i), cs = __ldg(coarse + na * 64 + i), fc = __ldg(fine + i * 64), fs = __ldg(fine + 4096 + i * 64);
        a.cos[tok][i] = cc * fc - cs * fs;
        a.sin[tok][i] = cs * fc + cc * fs;
    }
}

// To fp32 towards zero, the last bit set where bits were cut off: compares with any number of fewer bits as z does.
__device__ __forceinline__ float to_odd(double z)
{
    const uint32_t f = __float_as_uint(__double2float_rz(z));
    return __uint_as_float(f | ((__double2loint(z) & 0x1fffffff) != 0 ? 1u : 0u));
}

__device__ __forceinline__ float half_warp_max(float x)
{
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
    return x;
}

// A lane's eight channels as codes: four in each half of the head.
struct Codes { uint16_t lo, hi; };

// Channels as they are: the head's scale (bits), and the codes.
template <class E>
__device__ __forceinline__ uint16_t quantise(const Head<E> &u, Codes &c)
{
    float x[8];
    Quad<E>::unpack(u.lo, *reinterpret_cast<float (*)[4]>(x));
    Quad<E>::unpack(u.hi, *reinterpret_cast<float (*)[4]>(x + 4));
    float most = 0.f;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        most = fmaxf(most, fabsf(x[i]));
        bad = bad || !(fabsf(x[i]) < INFINITY);
    }
    most = half_warp_max(bad ? INFINITY : most);
    const float s = scale_of(most);
    float y[8];
    if (sizeof(E) == 2) {
        const float r = __frcp_rn(s);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __uint_as_float((__float_as_uint(x[i] * r) + 0x80u) & 0xffffff00u);
    } else {
        const double r = 1.0 / (double)s;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = to_odd(__longlong_as_double((__double_as_longlong((double)x[i] * r) + 0x800) & ~0xfffll));
    }
    c.lo = (uint16_t)(encode2(y[0], y[1]) | encode2(y[2], y[3]) << 8);
    c.hi = (uint16_t)(encode2(y[4], y[5]) | encode2(y[6], y[7]) << 8);
    return most < INFINITY ? (uint16_t)(__float_as_uint(s) >> 16) : kNaN;
}

// The linear map of a lane's four pairs (see pec_heads.cu): z_lo = lo * lc - hi * hs, z_hi = hi * hc + lo * ls.
struct Map { double lc[4], hs[4], hc[4], ls[4]; };
template <class E>
__device__ __forceinline__ void make_map(Map &m, const void *w, const double *cos, const double *sin, int l)
{
    float wl[4] = {1.f, 1.f, 1.f, 1.f}, wh[4] = {1.f, 1.f, 1.f, 1.f};
    if (w) {
        const Head<E> u = load_head(static_cast<const E *>(w), l);
        Quad<E>::unpack(u.lo, wl);
        Quad<E>::unpack(u.hi, wh);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const double c = cos ? cos[4 * l + i] : 1.0, s = cos ? sin[4 * l + i] : 0.0;
        m.lc[i] = wl[i] * c; m.ls[i] = wl[i] * s; m.hc[i] = wh[i] * c; m.hs[i] = wh[i] * s;
    }
}

// Norm and rotation first.
template <class E, bool kTurn>
__device__ __forceinline__ uint16_t quantise(const Head<E> &u, bool norm, float eps, const Map &m, Codes &c)
{
    float a[4], b[4];
    Quad<E>::unpack(u.lo, a);
    Quad<E>::unpack(u.hi, b);
    double r = 1.0;
    if (norm) {
        double ss = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) { ss = fma((double)a[i], (double)a[i], ss); ss = fma((double)b[i], (double)b[i], ss); }
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
        r = rsqrt(ss * (1.0 / kHeadDim) + (double)eps);
    }
    double z[8];
    float most = 0.f;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const double lo = a[i], hi = b[i];
        z[i] = r * (kTurn ? fma(lo, m.lc[i], -hi * m.hs[i]) : lo * m.lc[i]);
        z[4 + i] = r * (kTurn ? fma(hi, m.hc[i], lo * m.ls[i]) : hi * m.hc[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float f = fabsf(to_odd(z[i]));
        most = fmaxf(most, f);
        bad = bad || !(fabs(z[i]) < INFINITY);
    }
    most = half_warp_max(bad ? INFINITY : most);
    const float s = scale_of(most);
    const double r_s = 1.0 / (double)s;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = to_odd(__longlong_as_double((__double_as_longlong(z[i] * r_s) + 0x800) & ~0xfffll));
    c.lo = (uint16_t)(encode2(y[0], y[1]) | encode2(y[2], y[3]) << 8);
    c.hi = (uint16_t)(encode2(y[4], y[5]) | encode2(y[6], y[7]) << 8);
    return most < INFINITY ? (uint16_t)(__float_as_uint(s) >> 16) : kNaN;
}

struct Append {
    const void *k, *v;
    int64_t k_st, k_sh, v_st, v_sh;                                 // elements
    Q4Cache q;
    const void *kw;
    int32_t norm;
    float eps;
    Turn turn;
    int32_t *status;
};

// Block: eight tokens, a warp each; blockIdx.y = a part of the key heads, or (from `parts` on) of the value heads.
template <class E, bool kTurn>
__global__ void __launch_bounds__(kThreads)
kv_append_q4_kernel(const Append p, const int parts, const int per)
{
    __shared__ __align__(16) Angles sh;
    const PagedCache &pc = p.q.c;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane & 15, half = lane >> 4;
    const int32_t t = blockIdx.x * kWarps + warp;
    const bool is_k = (int)blockIdx.y < parts;
    const int h0 = ((int)blockIdx.y - (is_k ? 0 : parts)) * per, h1 = min(h0 + per, p.q.Hkv);
    const int64_t s_in = is_k ? p.k_sh : p.v_sh;
    const E *src = static_cast<const E *>(is_k ? p.k : p.v) + t * (is_k ? p.k_st : p.v_st) + (h0 + half) * s_in;

    int left = t < pc.T ? (h1 - h0 - half + 1) / 2 : 0;
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
    if (t < pc.T && find_request(pc, t, p.status, b, start, end, kv)) {
        pos = (int64_t)kv - end + t;
        const int64_t nth = pos / pc.page_size;
        slot = pos - nth * pc.page_size;
        if (pos >= 0 && nth < pc.max_pages && (!kTurn || pos < p.turn.n_pos)) {
            page = pc.table[b * pc.table_stride + nth];             // looked at when the angles are done
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
    if (page < 0 || page >= pc.num_pages) {
        if (lane == 0) raise_status(p.status, PEC_ERR_BAD_INDEX);
        return;
    }
    Map m;
    if (math) make_map<E>(m, p.norm ? p.kw : nullptr, turn ? sh.cos[warp] : nullptr, sh.sin[warp], l);
    const int64_t s_codes = is_k ? pc.k_sh : pc.v_sh, s_scale = is_k ? p.q.ks_sh : p.q.vs_sh;
    uint8_t *codes = (is_k ? p.q.k : p.q.v) + page * (is_k ? pc.k_sp : pc.v_sp) + slot * (is_k ? pc.k_st : pc.v_st) + (h0 + half) * s_codes;
    uint16_t *scale = (is_k ? p.q.ks : p.q.vs) + page * (is_k ? p.q.ks_sp : p.q.vs_sp) + slot * (is_k ? p.q.ks_st : p.q.vs_st) + (h0 + half) * s_scale;
    const int rounds = ((h1 - h0 + 1) / 2 + kRows - 1) / kRows;     // the same for both halves: shuffles stay converged
    for (int r = 0; r < rounds; ++r) {
        if (r) fetch(u);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            Codes c;
            const uint16_t s = math ? quantise<E, kTurn>(u[i], p.norm != 0, p.eps, m, c) : quantise(u[i], c);
            if (i < todo) {
                *reinterpret_cast<uint16_t *>(codes + 2 * l) = s == kNaN ? 0 : c.lo;
                *reinterpret_cast<uint16_t *>(codes + 32 + 2 * l) = s == kNaN ? 0 : c.hi;
                if (l == 0) *scale = s;
            }
            codes += 2 * s_codes;
            scale += 2 * s_scale;
        }
        todo -= kRows;
    }
}

struct Read {
    Q4Cache q;
    void *k, *v;
    int64_t k_st, k_sh, v_st, v_sh;                                 // elements
    int32_t *status;
};

// Block: eight tokens, a warp each; blockIdx.y = a part of the key heads, or (from `parts` on) of the value heads.  A half warp
// takes a head, a lane eight channels of it: 64 contiguous bytes in, 256 or 512 out.
template <class E>
__global__ void __launch_bounds__(kThreads)
kv_read_q4_kernel(const Read p, const int parts, const int per)
{
    const PagedCache &pc = p.q.c;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane & 15, half = lane >> 4;
    const int32_t t = blockIdx.x * kWarps + warp;
    int32_t b, start, end, kv;
    if (t >= pc.T || !find_request(pc, t, p.status, b, start, end, kv)) return;
    const int64_t pos = (int64_t)kv - end + t, nth = pos / pc.page_size, slot = pos - nth * pc.page_size;
    int64_t page = -1;
    if (pos >= 0 && nth < pc.max_pages) page = pc.table[b * pc.table_stride + nth];
    if (page < 0 || page >= pc.num_pages) {
        if (lane == 0) raise_status(p.status, PEC_ERR_BAD_INDEX);
        return;
    }
    const bool is_k = (int)blockIdx.y < parts;
    const int h0 = ((int)blockIdx.y - (is_k ? 0 : parts)) * per, h1 = min(h0 + per, p.q.Hkv);
    const int64_t s_codes = is_k ? pc.k_sh : pc.v_sh, s_scale = is_k ? p.q.ks_sh : p.q.vs_sh, s_out = is_k ? p.k_sh : p.v_sh;
    const uint8_t *codes = (is_k ? p.q.k : p.q.v) + page * (is_k ? pc.k_sp : pc.v_sp) + slot * (is_k ? pc.k_st : pc.v_st);
    const uint16_t *scale = (is_k ? p.q.ks : p.q.vs) + page * (is_k ? p.q.ks_sp : p.q.vs_sp) + slot * (is_k ? p.q.ks_st : p.q.vs_st);
    E *out = static_cast<E *>(is_k ? p.k : p.v) + t * (is_k ? p.k_st : p.v_st) + 8 * l;
    for (int h = h0 + half; h < h1; h += 2 * kRows) {
        uint32_t w[kRows];
        uint16_t s[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (h + 2 * i >= h1) break;
            w[i] = *reinterpret_cast<const uint32_t *>(codes + (h + 2 * i) * s_codes + 4 * l);
            s[i] = scale[(h + 2 * i) * s_scale];
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (h + 2 * i >= h1) break;
            uint32_t r[4];
            decode8(w[i], twice(s[i]), r);
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

// As for the heads of the cache that is not quantised (see pec_heads.cu).
inline int heads_per_part(int64_t T, int64_t H) { return T * H < (int64_t)148 * 32 * 32 ? 2 * kRows : 8 * kRows; }

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
    p.kw = a->k_weight; p.norm = a->norm; p.eps = a->eps; p.turn = {a->rope_table, a->n_pos}; p.status = a->status;
    const int per = q4::heads_per_part(T, 2 * (int64_t)p.q.Hkv), parts = (p.q.Hkv + per - 1) / per;
    const dim3 grid((unsigned)((T + q4::kWarps - 1) / q4::kWarps), (unsigned)(2 * parts));
    const bool turn = p.turn.table != nullptr;
    const auto kernel = esz == 2 ? (turn ? q4::kv_append_q4_kernel<__nv_bfloat16, true> : q4::kv_append_q4_kernel<__nv_bfloat16, false>)
                                 : (turn ? q4::kv_append_q4_kernel<float, true> : q4::kv_append_q4_kernel<float, false>);
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
    const int per = q4::heads_per_part(T, 2 * (int64_t)p.q.Hkv), parts = (p.q.Hkv + per - 1) / per;
    const dim3 grid((unsigned)((T + q4::kWarps - 1) / q4::kWarps), (unsigned)(2 * parts));
    const auto kernel = esz == 2 ? q4::kv_read_q4_kernel<__nv_bfloat16> : q4::kv_read_q4_kernel<float>;
    kernel<<<grid, q4::kThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(p, parts, per);
    const cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess) { set_error("%s: launch failed: %s", who, cudaGetErrorString(err)); return PEC_ERR_CUDA; }
    return PEC_OK;
}
