// Attention of a batch's new tokens over a paged K/V cache: the entry point, the FMA kernel (fp32 products and state) and the
// kernel that merges partial results.
#include <cuda_bf16.h>
#include <cmath>
#include <cuda_runtime.h>
#include "pec_host.h"
#include "pec_internal.h"
#include "pec_paged.h"
#include "pec_paged_plan.cuh"

namespace pec {
namespace paged {

// ------------------------------------------------------------------------------------------ FMA kernel
// One CTA = 64 packed rows of one KV head against one slice of the request's keys, 64 keys at a time.  256 threads as 16 x 16:
// thread (ty, tx) owns score rows 4 ty .. + 3 and keys tx + 16 j, and output rows 4 ty .. + 3 with channels 4 tx .. + 3 and
// 64 + 4 tx .. + 3.  Rows, keys and values past their ends are zero in shared memory, so that what a page holds past the
// request's end never meets a product.
constexpr int kBM = 64, kBN = 64, kThreads = 256;
constexpr int kLd = kHeadDim + 4, kLdP = kBN + 4;
constexpr size_t kSimpleSmem = sizeof(float) * (2 * kBM * kLd + kBN * kHeadDim + kBM * kLdP);

__device__ __forceinline__ float4 load4(const float *p) { return *reinterpret_cast<const float4 *>(p); }

__global__ void __launch_bounds__(kThreads)
paged_simple_kernel(const Params p)
{
    extern __shared__ __align__(16) float smem[];
    float *sQ = smem;                       // [kBM][kLd]
    float *sK = sQ + kBM * kLd;             // [kBN][kLd]
    float *sV = sK + kBN * kLd;             // [kBN][kHeadDim]
    float *sP = sV + kBN * kHeadDim;        // [kBM][kLdP]
    __shared__ Item s_item;
    __shared__ int s_found;
    __shared__ int32_t s_page[kBN];
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, kvh = blockIdx.y;
    if (tid < 32) {
        Item it;
        const bool found = locate_many(p, blockIdx.x, it);
        if (tid == 0) { s_found = found; if (found) s_item = it; }
    }
    __syncthreads();
    if (!s_found) return;
    const Item it = s_item;
    const int32_t row0 = it.block * kBM, rows = min(kBM, it.r.n * p.g - row0);

    for (int i = tid; i < kBM * (kHeadDim / 4); i += kThreads) {
        const int r = i / (kHeadDim / 4), c = (i % (kHeadDim / 4)) * 4;
        float4 val = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < rows) {
            const int32_t t = (row0 + r) / p.g, h = kvh * p.g + (row0 + r) % p.g;
            val = load4(static_cast<const float *>(p.q) + (int64_t)(it.r.start + t) * p.q_st + (int64_t)h * p.q_sh + c);
        }
        *reinterpret_cast<float4 *>(sQ + r * kLd + c) = val;
    }

    float m_run[4], l_run[4], acc[4][8];
    int32_t lim[4];                          // keys below it are visible to the row
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m_run[i] = -INFINITY; l_run[i] = 0.f;
        const int32_t r = row0 + ty * 4 + i, pos = it.r.pos0() + r / p.g;
        lim[i] = p.causal ? min(it.key_hi, pos + 1) : it.key_hi;
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[i][c] = 0.f;
    }
    const int32_t last = it.r.pos0() + (row0 + rows - 1) / p.g;
    const int32_t end = p.causal ? min(it.key_hi, last + 1) : it.key_hi;

    for (int32_t k0 = it.key_lo; k0 < end; k0 += kBN) {
        __syncthreads();                     // the previous tile's reads are done (also orders the Q stores)
        if (tid < kBN) {                     // page of each key of the tile; -1: past the end, or a bad page number
            int32_t page = -1;
            if (k0 + tid < it.key_hi) {
                page = p.c.table[it.b * p.c.table_stride + (k0 + tid) / p.c.page_size];
                if (page < 0 || page >= p.c.num_pages) { raise_status(p.status, PEC_ERR_BAD_INDEX); page = -1; }
            }
            s_page[tid] = page;
        }
        __syncthreads();
        for (int i = tid; i < kBN * (kHeadDim / 4); i += kThreads) {
            const int r = i / (kHeadDim / 4), c = (i % (kHeadDim / 4)) * 4;
            float4 kk = make_float4(0.f, 0.f, 0.f, 0.f), vv = kk;
            const int64_t page = s_page[r];
            if (page >= 0) {
                const int64_t slot = (k0 + r) % p.c.page_size;
                kk = load4(static_cast<const float *>(p.k_pages) + page * p.c.k_sp + slot * p.c.k_st + (int64_t)kvh * p.c.k_sh + c);
                vv = load4(static_cast<const float *>(p.v_pages) + page * p.c.v_sp + slot * p.c.v_st + (int64_t)kvh * p.c.v_sh + c);
            }
            *reinterpret_cast<float4 *>(sK + r * kLd + c) = kk;
            *reinterpret_cast<float4 *>(sV + r * kHeadDim + c) = vv;
        }
        __syncthreads();

        float s[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
        for (int d = 0; d < kHeadDim; d += 4) {
            float4 qa[4], kb[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) qa[i] = *reinterpret_cast<const float4 *>(sQ + (ty * 4 + i) * kLd + d);
#pragma unroll
            for (int j = 0; j < 4; ++j) kb[j] = *reinterpret_cast<const float4 *>(sK + (tx + 16 * j) * kLd + d);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[i][j] = fmaf(qa[i].x, kb[j].x, s[i][j]);
                    s[i][j] = fmaf(qa[i].y, kb[j].y, s[i][j]);
                    s[i][j] = fmaf(qa[i].z, kb[j].z, s[i][j]);
                    s[i][j] = fmaf(qa[i].w, kb[j].w, s[i][j]);
                }
        }
        // Mask by choice, not by adding -inf: a masked score may be anything.  State replicated over a row's 16 threads.
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float mx = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[i][j] = (k0 + tx + 16 * j < lim[i]) ? s[i][j] * p.scale_log2 : -INFINITY;
                mx = fmaxf(mx, s[i][j]);
            }
#pragma unroll
            for (int o = 8; o >= 1; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float m_new = fmaxf(m_run[i], mx);
            const float m_use = (m_new == -INFINITY) ? 0.f : m_new;
            const float alpha = exp2f(m_run[i] - m_use);           // 0 while the row is still empty
            float rs = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float pj = exp2f(s[i][j] - m_use);
                rs += pj;
                sP[(ty * 4 + i) * kLdP + tx + 16 * j] = pj;
            }
#pragma unroll
            for (int o = 8; o >= 1; o >>= 1) rs += __shfl_xor_sync(0xffffffffu, rs, o);
            l_run[i] = l_run[i] * alpha + rs;
            m_run[i] = m_new;
#pragma unroll
            for (int c = 0; c < 8; ++c) acc[i][c] *= alpha;
        }
        __syncthreads();
#pragma unroll 4
        for (int j = 0; j < kBN; ++j) {
            const float4 v0 = *reinterpret_cast<const float4 *>(sV + j * kHeadDim + tx * 4);
            const float4 v1 = *reinterpret_cast<const float4 *>(sV + j * kHeadDim + 64 + tx * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float pij = sP[(ty * 4 + i) * kLdP + j];
                acc[i][0] = fmaf(pij, v0.x, acc[i][0]); acc[i][1] = fmaf(pij, v0.y, acc[i][1]);
                acc[i][2] = fmaf(pij, v0.z, acc[i][2]); acc[i][3] = fmaf(pij, v0.w, acc[i][3]);
                acc[i][4] = fmaf(pij, v1.x, acc[i][4]); acc[i][5] = fmaf(pij, v1.y, acc[i][5]);
                acc[i][6] = fmaf(pij, v1.z, acc[i][6]); acc[i][7] = fmaf(pij, v1.w, acc[i][7]);
            }
        }
    }

    const int64_t slot = it.slot * p.Hkv + kvh;
    if (it.slices > 1 && slot >= p.many_cap) return;               // cannot happen (see many_slice); never write past the scratch
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int32_t r = ty * 4 + i;
        if (r >= rows) continue;
        const float inv = l_run[i] > 0.f ? 1.f / l_run[i] : 0.f;
        const float lse = l_run[i] > 0.f ? m_run[i] * 0.6931471805599453f + logf(l_run[i]) : -INFINITY;
        float out[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) out[c] = l_run[i] > 0.f ? acc[i][c] * inv : 0.f;
        if (it.slices > 1) {
            float *o = p.many_o + (slot * p.many_rows + r) * kHeadDim;
            *reinterpret_cast<float4 *>(o + tx * 4) = make_float4(out[0], out[1], out[2], out[3]);
            *reinterpret_cast<float4 *>(o + 64 + tx * 4) = make_float4(out[4], out[5], out[6], out[7]);
            if (tx == 0) p.many_lse[slot * p.many_rows + r] = lse;
        } else {
            const int64_t item = (int64_t)(it.r.start + (row0 + r) / p.g) * p.Hq + kvh * p.g + (row0 + r) % p.g;
            float *o = static_cast<float *>(p.o) + item * kHeadDim;
            *reinterpret_cast<float4 *>(o + tx * 4) = make_float4(out[0], out[1], out[2], out[3]);
            *reinterpret_cast<float4 *>(o + 64 + tx * 4) = make_float4(out[4], out[5], out[6], out[7]);
            if (tx == 0) p.lse[item] = lse;
        }
    }
}

// ------------------------------------------------------------------------------------------ combining partials
// A CTA merges the partial results of eight packed rows (few class) or 64 (many class) of one unit: a (request, KV head) whose
// tiles cross a cut of the line, or a block of rows whose keys are cut into slices.  Units are enumerated by what splits them -
// CTA c of the few class looks at cut c and takes the unit around it if this is the unit's first cut - so that the grid has the
// size of what can be split, not of the batch, and a CTA without a unit ends after one look at the tables.  (A CTA per token and
// KV head took 66 us to find nothing to do for 2048 tokens.)  All of that runs before the attention kernels end (the tables were
// complete before they began); the partials are read afterwards, and no CTA ends before that wait, so that whatever follows on
// the stream follows the attention kernels too.
// A warp merges one row at a time, a lane owning four channels: the largest LSE first, then the weighted sum.
constexpr int kCombineWarps = 8, kFewGroup = 8, kManyGroup = 64;

__device__ __forceinline__ void combine_row(const Params &p, const float *po, const float *pl, int64_t at0, int64_t shift, int64_t step,
                                            int count, int64_t item, int lane)
{
    auto place = [&](int s) { return at0 + s * step + (s == 0 ? shift : 0); };     // of partial s, in rows
    float m = -INFINITY;
    for (int s = lane; s < count; s += 32) m = fmaxf(m, pl[place(s)]);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    float tot = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (m != -INFINITY) {
#pragma unroll 4
        for (int s = 0; s < count; ++s) {
            const int64_t at = place(s);
            const float l = pl[at], w = (l == -INFINITY) ? 0.f : expf(l - m);
            const float4 v = *reinterpret_cast<const float4 *>(po + at * kHeadDim + 4 * lane);
            acc.x = fmaf(w, v.x, acc.x); acc.y = fmaf(w, v.y, acc.y); acc.z = fmaf(w, v.z, acc.z); acc.w = fmaf(w, v.w, acc.w);
            tot += w;
        }
    }
    const float inv = tot > 0.f ? 1.f / tot : 0.f;
    acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
    if (p.o_is_bf16) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(acc.x, acc.y), hi = __floats2bfloat162_rn(acc.z, acc.w);
        *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(p.o) + item * kHeadDim + 4 * lane) =
            make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
    } else {
        *reinterpret_cast<float4 *>(static_cast<float *>(p.o) + item * kHeadDim + 4 * lane) = acc;
    }
    if (lane == 0) p.lse[item] = (m == -INFINITY) ? -INFINITY : m + logf(tot);
}

__global__ void __launch_bounds__(kCombineWarps * 32, 4)
paged_combine_kernel(const Params p, const int few_groups, const int few_blocks, const int many_groups)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if ((int)blockIdx.x < few_blocks) {
        const int64_t cut = blockIdx.x / few_groups + 1;
        const int group = blockIdx.x % few_groups;
        int64_t all, rest;
        batch_tiles(p, all, rest);
        const int64_t piece = few_piece(p, all), at = cut * piece;
        Walk w;
        w.u0 = at;
        if (at < all * p.Hkv) walk_to(p, w, at, lane);
        const bool mine = w.u0 < at && w.u0 >= at - piece;       // else the cut falls between units, or is not the unit's first
        asm volatile("griddepcontrol.wait;" ::: "memory");
        if (!mine) return;
        const int64_t u1 = w.u0 + w.r.tiles();
        const int64_t first = cut - 1;                           // piece with the unit's first tiles
        const int count = (int)((u1 - 1) / piece - first) + 1;
        const int row = group * kFewGroup + warp;
        if (row >= w.r.n * p.g) return;
        const int64_t item = (int64_t)(w.r.start + row / p.g) * p.Hq + w.kvh * p.g + row % p.g;
        combine_row(p, p.few_o, p.few_lse, 2 * first * p.few_rows + row, w.u0 > first * piece ? p.few_rows : 0, 2 * (int64_t)p.few_rows, count,
                    item, lane);
    } else {
        int64_t x = blockIdx.x - few_blocks;
        const int group = (int)(x % many_groups);
        x /= many_groups;
        const int kvh = (int)(x % p.Hkv);
        SplitBlock sb;
        const bool mine = locate_split(p, x / p.Hkv, sb);
        asm volatile("griddepcontrol.wait;" ::: "memory");
        if (!mine) return;
        for (int i = warp; i < kManyGroup; i += kCombineWarps) {
            const int row = group * kManyGroup + i;              // of the block
            const int64_t packed = (int64_t)sb.block * p.many_rows + row;
            if (row >= p.many_rows || packed >= (int64_t)sb.r.n * p.g) return;
            const int64_t item = (sb.r.start + packed / p.g) * p.Hq + kvh * p.g + packed % p.g;
            combine_row(p, p.many_o, p.many_lse, (sb.first * p.Hkv + kvh) * p.many_rows + row, 0, (int64_t)p.Hkv * p.many_rows, sb.slices, item,
                        lane);
        }
    }
}

}  // namespace paged

using namespace paged;

int launch_paged_simple(const Params &p, int64_t items, cudaStream_t stream)
{
    static unsigned char ready[host::kMaxDevices] = {};
    static std::mutex ready_mutex;
    if (!host::once_per_device(ready, ready_mutex, [] {
            return cudaFuncSetAttribute(paged_simple_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSimpleSmem) == cudaSuccess; })) {
        (void)cudaGetLastError();
        set_error("pec_paged_attn: cannot raise the shared-memory limit");
        return PEC_ERR_CUDA;
    }
    if (items > 0x7fffffff) { set_error("pec_paged_attn: grid too large"); return PEC_ERR_UNSUPPORTED; }
    paged_simple_kernel<<<dim3((unsigned)items, (unsigned)p.Hkv), kThreads, kSimpleSmem, stream>>>(p);
    const cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess) { set_error("pec_paged_attn: launch failed: %s", cudaGetErrorString(err)); return PEC_ERR_CUDA; }
    return PEC_OK;
}

int launch_paged_combine(const Params &p, cudaStream_t stream)
{
    // Every cut of the line; every block that can be cut: one has two slots or more.
    const int few_groups = (p.few_rows + kFewGroup - 1) / kFewGroup, few_blocks = p.few ? (p.few_ctas - 1) * few_groups : 0;
    const int many_groups = (p.many_rows + kManyGroup - 1) / kManyGroup;
    const int64_t many_blocks = (int64_t)((p.many_cap / 2 + p.Hkv - 1) / p.Hkv) * p.Hkv * many_groups;
    if (few_blocks + many_blocks == 0) return PEC_OK;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(few_blocks + many_blocks));
    cfg.blockDim = dim3(kCombineWarps * 32);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t err = cudaLaunchKernelEx(&cfg, paged_combine_kernel, p, few_groups, few_blocks, many_groups);
    if (err == cudaSuccess) err = cudaGetLastError();
    if (err != cudaSuccess) { set_error("pec_paged_attn: launch failed: %s", cudaGetErrorString(err)); return PEC_ERR_CUDA; }
    return PEC_OK;
}

// ------------------------------------------------------------------------------------------ entry point
namespace paged {

struct Call {
    Params p;
    int64_t many_items;                       // grid bound of the many class; 0: no request can be of it
    size_t bytes;                             // workspace
};

inline bool aligned16(const void *x) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Checks the arguments and works out the launch.
static int resolve(const char *who, const pec_paged_args *a, Call &c)
{
    if (!a) { set_error("%s: args is NULL", who); return PEC_ERR_INVALID_ARG; }
    if (!a->q || !a->o || !a->lse) { set_error("%s: q, o and lse must be non-NULL", who); return PEC_ERR_INVALID_ARG; }
    Params &p = c.p;
    p = Params{};
    p.c = {a->k_pages_stride_p, a->k_pages_stride_t, a->k_pages_stride_h, a->v_pages_stride_p, a->v_pages_stride_t, a->v_pages_stride_h,
           a->block_table, a->table_stride, a->max_pages, a->page_size, a->num_pages, a->cu_q, a->kv_lens, a->B, (int32_t)a->T};
    const int rc = check_paged_cache(who, a->k_pages, a->v_pages, p.c, a->T, a->Hkv, a->D, a->dtype, a->status);
    if (rc != PEC_OK) return rc;
    if (a->Hq < 1 || a->Hq % a->Hkv != 0 || a->Hq / a->Hkv > 128) {
        set_error("%s: need Hkv | Hq and at most 128 query heads per KV head (got %d, %d)", who, a->Hq, a->Hkv);
        return PEC_ERR_INVALID_ARG;
    }
    if (a->o_dtype != PEC_BF16 && a->o_dtype != PEC_F32) { set_error("%s: unknown o_dtype %d", who, a->o_dtype); return PEC_ERR_UNSUPPORTED; }
    if (a->dtype == PEC_F32 && a->o_dtype != PEC_F32) { set_error("%s: fp32 inputs produce fp32 output only", who); return PEC_ERR_UNSUPPORTED; }
    if (a->causal != 0 && a->causal != 1) { set_error("%s: causal must be 0 or 1", who); return PEC_ERR_INVALID_ARG; }
    if (!(a->softmax_scale >= 0.f) || std::isinf(a->softmax_scale)) { set_error("%s: softmax_scale must be finite and >= 0", who); return PEC_ERR_INVALID_ARG; }
    if (a->max_q_len < 0) { set_error("%s: max_q_len must be >= 0", who); return PEC_ERR_INVALID_ARG; }
    const int64_t esz = a->dtype == PEC_BF16 ? 2 : 4;
    for (const int64_t s : {a->q_stride_t, a->q_stride_h}) {
        if (s < kHeadDim) { set_error("%s: strides must be >= D", who); return PEC_ERR_INVALID_ARG; }
        if ((s * esz) % 16 != 0) { set_error("%s: strides must be multiples of 16 bytes", who); return PEC_ERR_ALIGNMENT; }
    }
    if (!aligned16(a->q) || !aligned16(a->o) || (reinterpret_cast<uintptr_t>(a->lse) & 3u)) {
        set_error("%s: q and o must be 16-byte aligned (lse 4-byte)", who);
        return PEC_ERR_ALIGNMENT;
    }
    p.q = a->q; p.k_pages = a->k_pages; p.v_pages = a->v_pages;
    p.q_st = a->q_stride_t; p.q_sh = a->q_stride_h;
    p.o = a->o; p.lse = a->lse; p.o_is_bf16 = a->o_dtype == PEC_BF16;
    p.Hq = a->Hq; p.Hkv = a->Hkv; p.g = a->Hq / a->Hkv;
    p.causal = a->causal;
    const float scale = a->softmax_scale > 0.f ? a->softmax_scale : (float)(1.0 / std::sqrt((double)kHeadDim));
    p.scale_log2 = (float)((double)scale * 1.4426950408889634074);
    p.max_q = (int32_t)(a->max_q_len > 0 && a->max_q_len < a->T ? a->max_q_len : a->T);
    p.status = a->status;
    p.wait_cycles = wait_limit_cycles();
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1) {
        (void)cudaGetLastError();
        sms = 148;                            // no device here (size queries on a host without one): a B200's
    }
    // bf16 requests with at most 128 packed rows go to the persistent kernel.
    const bool tensor = a->dtype == PEC_BF16;
    p.few = tensor ? 1 : 0;
    p.few_ctas = sms;
    size_t floats = 0;
    if (p.few) {
        p.few_rows = (int32_t)((int64_t)p.max_q * p.g < kFewRows ? p.max_q * p.g : kFewRows);
        floats = 2 * (size_t)p.few_ctas * p.few_rows * (kHeadDim + 1);
        floats = (floats + 3) & ~(size_t)3;
    }
    // Blocks of the many class, the grid bound and the partial slots it may take (see many_slice).
    const int tps = kFewRows / p.g;           // tensor cores: two stages of whole tokens; FMA: 64 packed rows
    p.blk_mul = tensor ? 1 : p.g; p.blk_div = tensor ? 2 * tps : kBM;
    p.many_rows = tensor ? 2 * tps * p.g : kBM;
    p.many_slots = 2 * sms;
    c.many_items = 0;
    if (!p.few || (int64_t)p.max_q * p.g > kFewRows) {
        const int64_t shortest = p.few ? kFewRows / p.g + 1 : 1, most = a->T / shortest;       // new tokens of such a request; how many there can be
        const int64_t blocks = a->T * p.blk_mul / p.blk_div + (a->B < most ? a->B : most);
        c.many_items = blocks + ceil_div(p.many_slots, p.Hkv);
        const int64_t most_slices = ceil_div(ceil_div((int64_t)a->max_pages * a->page_size, kKeyTile), kMinSliceTiles);
        int64_t cap = 2 * (int64_t)p.many_slots;
        if (most_slices <= 1) cap = 0;
        else if (blocks * most_slices * p.Hkv < cap) cap = blocks * most_slices * p.Hkv;
        p.many_cap = (int32_t)cap;
    }
    c.bytes = (floats + (size_t)p.many_cap * p.many_rows * (kHeadDim + 1)) * sizeof(float);
    if (a->workspace) {
        float *ws = static_cast<float *>(a->workspace);
        p.few_o = ws;
        p.few_lse = ws + 2 * (size_t)p.few_ctas * p.few_rows * kHeadDim;
        p.many_o = ws + floats;
        p.many_lse = p.many_o + (size_t)p.many_cap * p.many_rows * kHeadDim;
    }
    return PEC_OK;
}

}  // namespace paged
}  // namespace pec

using namespace pec;

extern "C" size_t pec_paged_workspace_size(const pec_paged_args *args)
{
    paged::Call c;
    if (paged::resolve("pec_paged_workspace_size", args, c) != PEC_OK) return 0;
    return c.bytes;
}

extern "C" int pec_paged_attn(const pec_paged_args *args, void *cuda_stream)
{
    const char *who = "pec_paged_attn";
    paged::Call c;
    int rc = paged::resolve(who, args, c);
    if (rc != PEC_OK) return rc;
    if (c.bytes > 0 && (!args->workspace || args->workspace_bytes < c.bytes || !paged::aligned16(args->workspace))) {
        set_error("%s: workspace missing, misaligned or too small (%zu < %zu)", who, args->workspace_bytes, c.bytes);
        return PEC_ERR_WORKSPACE;
    }
    if (args->T == 0) return PEC_OK;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (c.many_items > 0) rc = args->dtype == PEC_BF16 ? launch_paged_many(c.p, c.many_items, stream) : launch_paged_simple(c.p, c.many_items, stream);
    if (rc == PEC_OK && c.p.few) rc = launch_paged_few(c.p, stream);
    if (rc != PEC_OK || c.bytes == 0) return rc;
    return launch_paged_combine(c.p, stream);
}
