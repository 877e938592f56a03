// Per-head steps between the QKV GEMM and the attention: RMS norm of every query and key head with the rotary encoding in
// the same pass (pec_qk_norm_rope), and the same for new keys on their way into a paged cache, the values beside them
// (pec_kv_append).
//
//     y = x / sqrt(mean(x^2) + eps) * w                         (norm)
//     z[i] = y[i] cos a - y[i + 64] sin a,   z[i + 64] = y[i + 64] cos a + y[i] sin a,   a = p theta^(-2 i / 128)
//
// Bound by memory: every element is read once and written once, rounded once at the end (sums and products in fp32).  A
// head's 128 elements are one 16-byte vector per lane: 16 lanes of a bf16 head, 32 of an fp32 head.  The sum of squares is
// a shuffle tree over those lanes and a channel's partner 64 away sits half the lanes away, one shuffle per element.  The
// angle depends on the token only, so a block works on whole tokens: it works out the 64 cosines and sines of each of its
// tokens once (two-level table of pec_rope_table: 16 KB of fine entries that stay in L1 plus one coarse row) and every head
// of the token reads them from shared memory.  Each lane issues the loads of kRows heads before anything else, so their
// latency runs beside the search for the token's request and the table reads.
#include <cmath>
#include <cstdio>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include "pec_host.h"
#include "pec_internal.h"
#include "pec_paged.h"

namespace pec {
namespace heads {

constexpr int kThreads = 256;
constexpr int kRows = 4;                     // rows of a lane group in flight
constexpr int kMaxTokens = 8;                // tokens of a block (one warp each looks a token up)

template <class E> struct Vec;
template <> struct Vec<__nv_bfloat16> {
    static constexpr int kN = 8;
    static __device__ __forceinline__ void unpack(const uint4 &u, float (&x)[8])
    {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 p = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&p);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <> struct Vec<float> {
    static constexpr int kN = 4;
    static __device__ __forceinline__ void unpack(const uint4 &u, float (&x)[4])
    {
        x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[4])
    {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};

struct Turn { const float *table; int64_t n_pos; };            // table of pec_rope_table, or NULL: no rotation
constexpr int kFine = 64 * 64;

// cos and sin of channel i at position p = 64 a + b by the addition theorem (see pec_rope_table).
__device__ __forceinline__ void angle(const Turn &t, int32_t p, int i, float &c, float &s)
{
    const int64_t na = (t.n_pos + 63) / 64, a = p >> 6;
    const int b = p & 63;
    const float *coarse = t.table + 2 * kFine + a * 64 + i;
    const float cc = __ldg(coarse), cs = __ldg(coarse + na * 64);
    const float fc = __ldg(t.table + i * 64 + b), fs = __ldg(t.table + kFine + i * 64 + b);
    c = cc * fc - cs * fs;
    s = cs * fc + cc * fs;
}

// Norm and rotation of one head held by a group of 128 / kN lanes, `l` the lane's place in it.  A lane of the lower half
// of the head holds y[i], its partner y[i + 64].  cs, sn: the token's 64 cosines and sines in shared memory, or NULL.
template <class E>
__device__ __forceinline__ void head_math(float (&x)[Vec<E>::kN], int l, bool norm, const float (&w)[Vec<E>::kN], float eps,
                                          const float *cs, const float *sn)
{
    constexpr int kN = Vec<E>::kN, kLanes = kHeadDim / kN;
    if (norm) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < kN; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
        for (int d = kLanes / 2; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
        const float r = 1.f / sqrtf(ss * (1.f / kHeadDim) + eps);
#pragma unroll
        for (int i = 0; i < kN; ++i) x[i] = x[i] * r * w[i];
    }
    if (cs) {
        const int i0 = (l * kN) & 63;
        const bool upper = l >= kLanes / 2;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const float other = __shfl_xor_sync(0xffffffffu, x[i], kLanes / 2);
            const float c = cs[i0 + i], s = sn[i0 + i];
            x[i] = upper ? fmaf(x[i], c, other * s) : fmaf(x[i], c, -other * s);
        }
    }
}

template <class E>
__device__ __forceinline__ void load_weight(const void *w, int l, float (&out)[Vec<E>::kN])
{
    if (w) {
        const uint4 u = *reinterpret_cast<const uint4 *>(static_cast<const E *>(w) + l * Vec<E>::kN);
        Vec<E>::unpack(u, out);
    } else {
#pragma unroll
        for (int i = 0; i < Vec<E>::kN; ++i) out[i] = 1.f;
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

// Block: tokens [tok * blockIdx.x, +tok), head rows dealt to lane groups; blockIdx.y takes its share of the heads.
template <class E>
__global__ void __launch_bounds__(kThreads)
norm_rope_kernel(const NormRope p, const int tok, const int heads_per_block)
{
    constexpr int kN = Vec<E>::kN, kLanes = kHeadDim / kN, kGroups = kThreads / kLanes;
    __shared__ float s_cos[kMaxTokens][64], s_sin[kMaxTokens][64];
    __shared__ int32_t s_ok[kMaxTokens];
    const int tid = threadIdx.x, l = tid % kLanes, grp = tid / kLanes;
    const int t0 = blockIdx.x * tok, nt = min(tok, p.T - t0);
    const int h0 = blockIdx.y * heads_per_block, nh = min(heads_per_block, p.H - h0);
    const int rows = nt * nh;

    auto src = [&](int r) -> const uint4 * {
        const int64_t t = t0 + r / nh;
        const int h = h0 + r % nh;
        const E *base = h < p.Hq ? static_cast<const E *>(p.q) + t * p.q_st + h * p.q_sh
                                 : static_cast<const E *>(p.k) + t * p.k_st + (h - p.Hq) * p.k_sh;
        return reinterpret_cast<const uint4 *>(base + l * kN);
    };
    auto fetch = [&](int r0, uint4 (&u)[kRows]) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            u[i] = make_uint4(0u, 0u, 0u, 0u);
            if (r0 + i * kGroups < rows) u[i] = *src(r0 + i * kGroups);
        }
    };
    uint4 u[kRows];
    fetch(grp, u);
    float qw[kN], kw[kN];
    load_weight<E>(p.norm ? p.qw : nullptr, l, qw);
    load_weight<E>(p.norm ? p.kw : nullptr, l, kw);
    // Positions and angles of the block's tokens.  A negative position marks a padding row; one past the table is reported.
    for (int i = tid; i < nt * 64; i += kThreads) {
        const int k = i >> 6, ch = i & 63;
        const int64_t pos = p.positions ? (int64_t)p.positions[t0 + k] : p.pos0 + t0 + k;
        bool ok = pos >= 0;
        if (ok && p.turn.table) {
            if (pos >= p.turn.n_pos) {
                ok = false;
                if (ch == 0) raise_status(p.status, PEC_ERR_BAD_INDEX);
            } else {
                angle(p.turn, (int32_t)pos, ch, s_cos[k][ch], s_sin[k][ch]);
            }
        }
        if (ch == 0) s_ok[k] = ok;
    }
    __syncthreads();
    for (int r0 = grp; r0 - grp < rows; r0 += kRows * kGroups) {
        if (r0 != grp) fetch(r0, u);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int r = r0 + i * kGroups;
            if (r - grp >= rows) break;                       // uniform over the block: shuffles stay converged
            const int rr = min(r, rows - 1), k = rr / nh, h = h0 + rr % nh;
            float x[kN];
            Vec<E>::unpack(u[i], x);
            const bool is_q = h < p.Hq;
            float w[kN];
#pragma unroll
            for (int c = 0; c < kN; ++c) w[c] = is_q ? qw[c] : kw[c];
            head_math<E>(x, l, p.norm != 0, w, p.eps, p.turn.table ? s_cos[k] : nullptr, s_sin[k]);
            if (r < rows && s_ok[k]) {
                const int64_t t = t0 + k;
                E *dst = is_q ? static_cast<E *>(p.qo) + t * p.qo_st + h * p.qo_sh
                              : static_cast<E *>(p.ko) + t * p.ko_st + (h - p.Hq) * p.ko_sh;
                *reinterpret_cast<uint4 *>(dst + l * kN) = Vec<E>::pack(x);
            }
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

template <class E>
__global__ void __launch_bounds__(kThreads)
kv_append_kernel(const Append p, const int tok, const int heads_per_block)
{
    constexpr int kN = Vec<E>::kN, kLanes = kHeadDim / kN, kGroups = kThreads / kLanes;
    __shared__ float s_cos[kMaxTokens][64], s_sin[kMaxTokens][64];
    __shared__ int32_t s_pos[kMaxTokens];                           // -1: nothing to store
    __shared__ int64_t s_k[kMaxTokens], s_v[kMaxTokens];            // the token's slot in either cache, elements
    const int tid = threadIdx.x, warp = tid >> 5, l = tid % kLanes, grp = tid / kLanes;
    const int t0 = blockIdx.x * tok, nt = min(tok, p.c.T - t0);
    const int H = 2 * p.Hkv, h0 = blockIdx.y * heads_per_block, nh = min(heads_per_block, H - h0);
    const int rows = nt * nh;

    auto fetch = [&](int r0, uint4 (&u)[kRows]) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int r = r0 + i * kGroups;
            u[i] = make_uint4(0u, 0u, 0u, 0u);
            if (r < rows) {
                const int64_t t = t0 + r / nh;
                const int h = h0 + r % nh;
                const E *base = h < p.Hkv ? static_cast<const E *>(p.k) + t * p.k_st + h * p.k_sh
                                          : static_cast<const E *>(p.v) + t * p.v_st + (h - p.Hkv) * p.v_sh;
                u[i] = *reinterpret_cast<const uint4 *>(base + l * kN);
            }
        }
    };
    uint4 u[kRows];
    fetch(grp, u);
    float kw[kN];
    load_weight<E>(p.norm ? p.kw : nullptr, l, kw);
    if (warp < nt) {                                                // one warp per token: request, position, page, slot
        const int32_t t = t0 + warp;
        int32_t b, end, pos = -1;
        if (find_request(p.c, t, p.status, b, end)) {
            const int64_t at = (int64_t)p.c.kv_lens[b] - end + t;
            const int64_t nth = at / p.c.page_size;
            bool ok = at >= 0 && nth < p.c.max_pages && (!p.turn.table || at < p.turn.n_pos);
            int64_t page = -1;
            if (ok) {
                page = p.c.table[b * p.c.table_stride + nth];
                ok = page >= 0 && page < p.c.num_pages;
            }
            if (ok) {
                pos = (int32_t)at;
                const int64_t slot = at - nth * p.c.page_size;
                s_k[warp] = page * p.c.k_sp + slot * p.c.k_st;
                s_v[warp] = page * p.c.v_sp + slot * p.c.v_st;
            } else if ((tid & 31) == 0) {
                raise_status(p.status, PEC_ERR_BAD_INDEX);
            }
        }
        s_pos[warp] = pos;
    }
    __syncthreads();
    if (p.turn.table) {
        for (int i = tid; i < nt * 64; i += kThreads) {
            const int k = i >> 6, ch = i & 63;
            if (s_pos[k] >= 0) angle(p.turn, s_pos[k], ch, s_cos[k][ch], s_sin[k][ch]);
        }
        __syncthreads();
    }
    for (int r0 = grp; r0 - grp < rows; r0 += kRows * kGroups) {
        if (r0 != grp) fetch(r0, u);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int r = r0 + i * kGroups;
            if (r - grp >= rows) break;                             // uniform over the block
            const int rr = min(r, rows - 1), k = rr / nh, h = h0 + rr % nh;
            const bool is_k = h < p.Hkv;
            if (__any_sync(0xffffffffu, is_k)) {                    // a bf16 warp holds two heads, perhaps a key and a value
                float x[kN];
                Vec<E>::unpack(u[i], x);
                head_math<E>(x, l, p.norm != 0, kw, p.eps, p.turn.table ? s_cos[k] : nullptr, s_sin[k]);
                if (is_k && (p.norm || p.turn.table)) u[i] = Vec<E>::pack(x);
            }
            if (r < rows && s_pos[k] >= 0) {
                E *dst = is_k ? static_cast<E *>(p.k_pages) + s_k[k] + h * p.c.k_sh
                              : static_cast<E *>(p.v_pages) + s_v[k] + (h - p.Hkv) * p.c.v_sh;
                *reinterpret_cast<uint4 *>(dst + l * kN) = u[i];
            }
        }
    }
}

// Tokens and heads of a block.  Large calls: whole tokens, so that the angles are worked out once per token, and about 64
// rows a block where a token has fewer heads than that.  Calls too small to fill the GPU that way (`rows` below two full
// waves of lane groups) take one token a block and split its heads over grid.y.
inline void block_shape(int64_t T, int H, int groups, int &tok, int &hpb)
{
    tok = 64 / H < 1 ? 1 : (64 / H > kMaxTokens ? kMaxTokens : 64 / H);
    hpb = H;
    if (T * H < (int64_t)2 * 148 * 8 * groups) {
        tok = 1;
        hpb = H > groups ? groups : H;
    }
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
    int tok, hpb;
    heads::block_shape(p.T, p.H, heads::kThreads / (esz == 2 ? 16 : 32), tok, hpb);
    const dim3 grid((unsigned)((p.T + tok - 1) / tok), (unsigned)((p.H + hpb - 1) / hpb));
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (esz == 2) heads::norm_rope_kernel<__nv_bfloat16><<<grid, heads::kThreads, 0, stream>>>(p, tok, hpb);
    else          heads::norm_rope_kernel<float><<<grid, heads::kThreads, 0, stream>>>(p, tok, hpb);
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
    int tok, hpb;
    heads::block_shape(a->T, 2 * a->Hkv, heads::kThreads / (esz == 2 ? 16 : 32), tok, hpb);
    const dim3 grid((unsigned)((a->T + tok - 1) / tok), (unsigned)((2 * (int64_t)a->Hkv + hpb - 1) / hpb));
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (esz == 2) heads::kv_append_kernel<__nv_bfloat16><<<grid, heads::kThreads, 0, stream>>>(p, tok, hpb);
    else          heads::kv_append_kernel<float><<<grid, heads::kThreads, 0, stream>>>(p, tok, hpb);
    const cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess) { set_error("%s: launch failed: %s", who, cudaGetErrorString(err)); return PEC_ERR_CUDA; }
    return PEC_OK;
}
