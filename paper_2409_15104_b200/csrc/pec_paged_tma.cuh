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

// 5-D tiled load, coordinates innermost first.
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const void *tmap, uint32_t bar, int c0, int c1, int c2, int c3, int c4)
{
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
        ::"r"(dst), "l"(tmap), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4) : "memory");
}

// A 128-key tile lies in shared memory as 16 groups of eight keys, a group as its two channel halves of eight 128-byte rows
// (128-byte swizzle): groups 2048 bytes apart, halves 1024.  It comes in boxes of `box` = gcd(page_size, 128) keys, both halves at
// once: such a box never crosses a page, whatever the page size (a multiple of 8, so that a box is whole groups).  Lane i of the
// loading warp takes keys i * box ..; boxes past the request's end are not loaded.
// The copy unit takes 85 to 110 cycles a box whatever its size, and a tile of K and V has 2800 at the rate of HBM: with a box per
// half (the halves 16 KB apart) pages of 16 tokens took 244 us where pages of 64 took 191 (three requests of 131072 keys), pages of
// 8 tokens 381; with both halves in one box 198, 190 and 246.
constexpr uint32_t kGroupBytes = 2048, kGroupHalf = 1024;
struct BoxLane { int32_t first; uint32_t offset; bool used; };
__device__ __forceinline__ BoxLane box_lane(int box, int lane)
{
    const int32_t first = lane * box;
    return {first, (uint32_t)(first >> 3) * kGroupBytes, first < kKeyTile};
}
__device__ __forceinline__ void load_box(uint32_t tile, const void *tmap, uint32_t bar, const BoxLane &l, const FoldedPages &f, int kvh, int row, int page)
{
    tma_load_5d(tile + l.offset, tmap, bar, 0, 0, 0, row >> 3, page * f.page + kvh * f.head);
}
// Four K steps (16 keys each) of D (+)= A B with A in tensor memory (8 columns per step) and B the N-major V tile.
__device__ __forceinline__ void mma_pv_k64(uint32_t d_tmem, uint32_t a_tmem, uint64_t b0, uint32_t idesc, uint32_t accumulate)
{
    mma_ts(d_tmem, a_tmem, b0, idesc, accumulate);
#pragma unroll
    for (uint32_t ks = 1; ks < 4; ++ks) mma_ts(d_tmem, a_tmem + 8 * ks, b0 + (2 * kGroupBytes >> 4) * ks, idesc, 1u);
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
        const uint32_t a = tile + (uint32_t)(i >> 7) * kGroupBytes + (i & 8 ? kGroupHalf : 0u) + (uint32_t)((i >> 4) & 7) * 128u + (uint32_t)(i & 7) * 16u;
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
// Pages: 64 channels, eight tokens, channel half, eight-token groups of a page, page and head (FoldedPages).
inline bool pages(CUtensorMap *map, const Params &p, const void *base, int64_t st, const FoldedPages &f, int box)
{
    const host::EncodeTiledFn fn = host::encode_fn();
    if (!fn) return false;
    const cuuint64_t last = (cuuint64_t)(p.c.num_pages - 1) * f.page + (cuuint64_t)(p.Hkv - 1) * f.head;
    const cuuint64_t d[5] = {64, 8, 2, (cuuint64_t)p.c.page_size / 8, last + 1};
    const cuuint64_t s[4] = {(cuuint64_t)st * 2, 128, (cuuint64_t)st * 16, (cuuint64_t)f.unit * 2};
    const cuuint32_t b[5] = {64, 8, 2, (cuuint32_t)box / 8, 1}, e[5] = {1, 1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void *>(base), d, s, b, e, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
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
