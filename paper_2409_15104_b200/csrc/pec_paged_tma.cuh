// Tile loads of the paged attention kernels: tensor maps of the packed queries and of the pages, and the copies themselves.
#pragma once
#include <cuda.h>
#include <cstring>
#include "pec_host.h"
#include "pec_paged_plan.cuh"
#include "pec_sm100.cuh"

namespace pec {
namespace paged {
using namespace sm100;

constexpr uint32_t kHalfTileBytes = 128 * 64 * 2;          // 128 rows x 64 channels, 128-byte swizzle
constexpr uint32_t kTileBytes = 2 * kHalfTileBytes;

// 4-D tiled load, coordinates innermost first.
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void *tmap, uint32_t bar, int c0, int c1, int c2, int c3)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(dst), "l"(tmap), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}

// A 128-key tile comes in boxes of `box` = gcd(page_size, 128) rows x 64 channels: such a box never crosses a page, whatever the
// page size (a multiple of 8, so that a box is whole 8-row swizzle groups and lands on a 1024-byte boundary).  Lane i of the
// loading warp takes rows (i / 2) * box .. of channel half i % 2; boxes past the request's end are not loaded.
struct BoxLane { int32_t first; uint32_t offset; int half; bool used; };
__device__ __forceinline__ BoxLane box_lane(int box, int lane)
{
    BoxLane l;
    l.half = lane & 1;
    l.first = (lane >> 1) * box;
    l.used = l.first < kKeyTile;
    l.offset = (uint32_t)l.half * kHalfTileBytes + (uint32_t)l.first * 128u;
    return l;
}
// Where this lane's box of a key tile lies: the number in the request's list of pages and the row of the page.  Walked from tile
// to tile without divisions, which would sit between a free slot and its next load.
struct BoxPlace { int32_t nth, row; };
struct BoxStep { int32_t nth, row, page_size; };
__device__ __forceinline__ BoxStep box_step(int32_t page_size) { return {kKeyTile / page_size, kKeyTile % page_size, page_size}; }
__device__ __forceinline__ BoxPlace box_place(int32_t page_size, int32_t k0, const BoxLane &l)
{
    const int32_t nth = (k0 + l.first) / page_size;
    return {nth, k0 + l.first - nth * page_size};
}
__device__ __forceinline__ BoxPlace box_next(const BoxPlace &b, const BoxStep &s)
{
    BoxPlace n = {b.nth + s.nth, b.row + s.row};
    if (n.row >= s.page_size) { n.row -= s.page_size; ++n.nth; }
    return n;
}
// Page of this lane's box of the key tile that begins at position k0 (0 where the box is not loaded, or the number is bad).
__device__ __forceinline__ int32_t box_page(const Params &p, int b, int32_t k0, int32_t kv, const BoxLane &l, const BoxPlace &at)
{
    if (!l.used || k0 + l.first >= kv) return 0;
    const int32_t page = __ldg(p.c.table + b * p.c.table_stride + at.nth);
    if (page >= 0 && page < p.c.num_pages) return page;
    raise_status(p.status, PEC_ERR_BAD_INDEX);
    return 0;
}
// Bytes of the tile's boxes that are loaded (box is a power of two).
__device__ __forceinline__ uint32_t tile_bytes(int32_t k0, int32_t kv, int box)
{
    int32_t n = kv - k0;
    n = n < 0 ? 0 : (n > kKeyTile ? kKeyTile : n);
    return (uint32_t)((n + box - 1) & -box) * 256u;
}
// What a page holds past the request's end may be anything; 0 * NaN would reach every row's output.  The whole warp that issues
// the product P V clears those rows of the V tile first (once per request: only its last tile has such rows).
__device__ __forceinline__ void clear_tail(uint32_t tile, int32_t valid, int lane)
{
    if (valid < 0) valid = 0;
    for (int i = valid * 16 + lane; i < kKeyTile * 16; i += 32) {
        const uint32_t a = tile + (uint32_t)(i & 8 ? kHalfTileBytes : 0u) + (uint32_t)(i >> 4) * 128u + (uint32_t)(i & 7) * 16u;
        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(a), "r"(0) : "memory");
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
}

// Ends of a CTA that gives up (a wait of its own or of an earlier CTA has run out): a wait with the usual limit that raises
// nothing and does not look at the abort flag, for copies and products under way.
__device__ __forceinline__ void wait_quietly(uint64_t *bar, uint32_t parity, const Params &p)
{
    const long long t0 = clock64();
    while (!mbar_try_wait_suspend(smem_u32(bar), parity, 2000u) && clock64() - t0 < p.wait_cycles) {}
}
// Until the products that the calling warp's `leader` lane has issued are complete: tensor memory may not be given back before.
__device__ __forceinline__ void drain_products(uint64_t *bar, bool leader, const Params &p)
{
    if (leader) tc_commit(smem_u32(bar));
    __syncwarp();
    wait_quietly(bar, 0, p);
}

namespace host_map {
// bf16, 128-byte swizzle, rank 4.  Encoded for every call (well under a microsecond each).
inline bool encode(CUtensorMap *map, const void *base, const uint64_t (&dims)[4], const int64_t (&strides)[3], const uint32_t (&box)[4])
{
    const host::EncodeTiledFn fn = host::encode_fn();
    if (!fn) return false;
    const cuuint64_t d[4] = {dims[0], dims[1], dims[2], dims[3]};
    const cuuint64_t s[3] = {(cuuint64_t)strides[0] * 2, (cuuint64_t)strides[1] * 2, (cuuint64_t)strides[2] * 2};
    const cuuint32_t b[4] = {box[0], box[1], box[2], box[3]}, e[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(base), d, s, b, e, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Queries as packed rows: channel, head of the group, KV head, token; a box is `tokens` tokens of one group.
inline bool queries(CUtensorMap *map, const Params &p, int tokens)
{
    return encode(map, p.q, {(uint64_t)kHeadDim, (uint64_t)p.g, (uint64_t)p.Hkv, (uint64_t)p.c.T}, {p.q_sh, p.q_sh * p.g, p.q_st},
                  {64u, (uint32_t)p.g, 1u, (uint32_t)tokens});
}
// Pages: channel, KV head, token of the page, page.
inline bool pages(CUtensorMap *map, const Params &p, const void *base, int64_t sp, int64_t st, int64_t sh, int box)
{
    return encode(map, base, {(uint64_t)kHeadDim, (uint64_t)p.Hkv, (uint64_t)p.c.page_size, (uint64_t)p.c.num_pages}, {sh, st, sp},
                  {64u, 1u, (uint32_t)box, 1u});
}
inline int box_rows(int page_size)
{
    int b = kKeyTile;
    while (page_size % b) b /= 2;
    return b;
}
}  // namespace host_map

}  // namespace paged
}  // namespace pec
