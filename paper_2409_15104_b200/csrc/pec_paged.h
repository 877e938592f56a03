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

// The request that owns token row t, searched by one converged warp: lane l looks at cu_q[l + 1], cu_q[l + 33], ... (the
// loads are independent of one another; a binary search would be a chain of log2(B) dependent ones) and b is the number of
// requests that end at or before t.  Returns false for padding rows; a table that is not ascending around t raises the
// status word and returns false.
__device__ __forceinline__ bool find_request(const PagedCache &c, int32_t t, int32_t *status, int32_t &b, int32_t &end)
{
    const int lane = threadIdx.x & 31;
    b = 0;
    for (int b0 = 0; b0 < c.B; b0 += 32) {
        const bool past = (b0 + lane < c.B) && c.cu_q[b0 + lane + 1] <= t;
        b += __popc(__ballot_sync(0xffffffffu, past));
    }
    if (b >= c.B) return false;
    const int32_t start = c.cu_q[b];
    end = c.cu_q[b + 1];
    if (t < start || t >= end || end > c.T) {
        if (lane == 0 && t >= c.cu_q[0]) raise_status(status, PEC_ERR_BAD_INDEX);
        return false;
    }
    return true;
}

// Host checks common to the entry points; returns a pec_status.
int check_paged_cache(const char *who, const void *k_pages, const void *v_pages, const PagedCache &c, int64_t T, int32_t Hkv,
                      int32_t D, int32_t dtype, const int32_t *status);

}  // namespace pec
