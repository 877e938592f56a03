// Host-side description of a paged K/V cache and of the batch that is appended to it or attends over it, shared by the
// entry points that take one (pec_kv_append, pec_paged_attn).  Not part of the ABI.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>
#include "pec_internal.h"

namespace pec {

struct PagedCache {
    int64_t k_sp, k_st, k_sh;        // elements: page, token of a page, head
    int64_t v_sp, v_st, v_sh;
    const int32_t *table;            // [B][table_stride], the first max_pages entries of a row are its pages
    int64_t table_stride;
    int32_t max_pages, page_size;
    int64_t num_pages;
    const int32_t *cu_q;             // [B + 1]
    const int32_t *kv_lens;          // [B]
    int32_t B;
    int32_t T;                       // token rows of the call's buffers; rows outside [cu_q[0], cu_q[B]) are padding
};

// First error wins; the host reads the word after synchronising.
__device__ __forceinline__ void raise_status(int32_t *status, int32_t code)
{
    if (status) atomicCAS(status, 0, code);
}

// The request that owns token row t and that request's entry of kv_lens, searched by one converged warp, 32 requests at a
// time: every lane's loads are independent of one another (a binary search would be a chain of log2(B) dependent ones) and the
// owner's values come by shuffle.  Returns false for padding rows.  Offsets that are not ascending, or pass T, raise the status word in
// each group that is looked at; the last row's warp looks at those after its owner's too, so that the rows together see all of them.
__device__ __forceinline__ bool find_request(const PagedCache &c, int32_t t, int32_t *status, int32_t &b, int32_t &start, int32_t &end, int32_t &kv)
{
    const int lane = threadIdx.x & 31;
    const int32_t first = c.cu_q[0];
    int32_t prev = first;                                       // the end of the request before this group of 32
    bool found = false, bad = first < 0;
    for (int b0 = 0; b0 < c.B; b0 += 32) {
        int32_t e = INT32_MAX, k = 0;
        const bool real = b0 + lane < c.B;
        if (real) { e = c.cu_q[b0 + lane + 1]; k = c.kv_lens[b0 + lane]; }
        int32_t before = __shfl_up_sync(0xffffffffu, e, 1);
        if (lane == 0) before = prev;
        bad = bad || e < before || (real && e > c.T);
        const int src = __popc(__ballot_sync(0xffffffffu, e <= t));       // requests of the group that end at or before t
        if (src < 32 && !found) {
            b = b0 + src;
            start = __shfl_sync(0xffffffffu, before, src);
            end = __shfl_sync(0xffffffffu, e, src);
            kv = __shfl_sync(0xffffffffu, k, src);
            found = b < c.B && t >= first;
            if (t != c.T - 1) break;
        }
        prev = __shfl_sync(0xffffffffu, e, 31);
    }
    if (__any_sync(0xffffffffu, bad) && lane == 0) raise_status(status, PEC_ERR_BAD_INDEX);
    return found && start >= 0 && t >= start && t < end && end <= c.T;
}

// Host checks common to the entry points; each returns a pec_status.
int check_batch(const char *who, const PagedCache &c, int64_t T, int32_t Hkv);           // sizes of the batch and its tables
int check_norm_rope(const char *who, int32_t norm, float eps, const float *table, int64_t n_pos);
int check_paged_cache(const char *who, const void *k_pages, const void *v_pages, const PagedCache &c, int64_t T, int32_t Hkv,
                      int32_t D, int32_t dtype, const int32_t *status);

}  // namespace pec
