// How a batch's work is cut for the kernels behind pec_paged_attn, worked out on the device from the tables themselves (no host
// plan: a captured graph replays with whatever lengths the tables then hold).
//
// Query rows are packed: the g = Hq / Hkv heads of a KV head and the new tokens of a request are the rows of one matrix,
// row = token * g + head of the group, so that a key tile read once serves all of them.
//
// Two classes of requests, by their packed rows n * g:
//   few  (at most 128: decode steps; fp32 has none)  worked on by a persistent grid.  The key tiles of all (request, KV head) pairs lie on
//        one line that is cut into equal pieces, one per CTA; a pair that crosses a cut leaves one partial result per piece.
//   many (chunks)                     items of one block of rows against all or a slice of its keys, listed longest first by a
//        kernel of one CTA ahead of the attention kernel, which has one CTA per (item, KV head).  (With every CTA working out
//        its own item from the tables a CTA spent 4-6 us on it: five waves of 64-token blocks lost 20 of 210 us.)
// Both sides of 128 rows, measured (64 requests of 3000 keys, 8 KV heads, few / many): 4 rows a request 128 / 163 us, 32 138 / 174,
// 128 160 / 181; 200 requests of 132 keys, 64 rows 49 / 99; one request of 32000 keys, 128 rows 40 / 55.
// A cache held in 4 bits: few is at most 16 rows, what its kernel's registers take (bf16 queries; fp32 has none here either).  16 rows a
// request, 8 KV heads, few / many: 32 requests of 4000 keys 71 / 144 us, 8 of 64000 152 / 575, 256 of 600 122 / 272, one of 8000 23 / 35.
// Partials are merged by their LSE by one kernel for both classes (combine), which finds them by the same arithmetic.
#pragma once
#include "pec_internal.h"
#include "pec_paged.h"

namespace pec {
namespace paged {

constexpr int kKeyTile = 128;                 // keys per tile
constexpr int kFewRows = 128;                 // packed rows of the few class
constexpr int kFewRowsQ4 = 16, kFewCtasQ4 = 2;   // the same of a cache held in 4 bits, and its kernel's CTAs on an SM
// Device-side description of one call, passed to the kernels by value.
// Where the rows of a page's head begin, as one number for the tensor maps, whose five dimensions a box of both channel halves
// takes up: (page * .page + head * .head) units of `unit` elements, the greatest common divisor of the two strides.
struct FoldedPages { int64_t unit; int32_t page, head; };

struct Params {
    const char *who;                          // entry point, for the host's error texts
    const void *q, *k_pages, *v_pages;
    int64_t q_st, q_sh;
    PagedCache c;
    FoldedPages fk, fv;                       // bf16
    const uint16_t *k_scales, *v_scales;      // a cache held in 4 bits: bf16 bits, strides in elements (those of `c` are in bytes)
    int64_t ks_sp, ks_st, ks_sh, vs_sp, vs_st, vs_sh;
    void *o;
    float *lse;
    int32_t o_is_bf16;
    int32_t Hq, Hkv, g;
    int32_t causal;
    float scale_log2;
    int32_t max_q;                            // a request with more new tokens is a bad index
    int32_t *status;
    int64_t wait_cycles;
    // few class
    int32_t few;                              // 0: every request is of the many class (fp32)
    int32_t few_limit;                        // packed rows of such a request at most
    int32_t few_ctas;
    int32_t few_rows;                         // rows of a partial slot
    float *few_o, *few_lse;                   // [2 * few_ctas][few_rows][128], [..][few_rows]
    // many class: blocks of a request = ceil(n * blk_mul / blk_div)
    int32_t blk_mul, blk_div;
    int32_t many_ctas;                        // CTAs of the many class that run at a time
    int32_t min_slice;                        // key tiles of the shortest slice
    int32_t item_cost, merge_cost;            // start and end of a CTA, a slice's partial: 1/32 of a tile's time (see paged_plan_kernel)
    int32_t many_rows;                        // rows of a partial slot
    int32_t many_blocks;                      // bound of the batch's blocks, from which many_cap and items_cap follow
    int32_t many_cap, items_cap;              // slots and items that the workspace holds
    float *many_o, *many_lse;
    int32_t *many_count;                      // [2]: items, blocks that are cut
    struct Item *many_items, *many_split;     // the items, longest first; slice 0 of each block that is cut
};

struct Request {
    int32_t start, n, kv;                     // first packed token row, new tokens, cached tokens
    __device__ __forceinline__ int32_t pos0() const { return kv - n; }
    __device__ __forceinline__ int32_t tiles() const { return kv > 0 ? (kv + kKeyTile - 1) / kKeyTile : 1; }
};

// The request's entry in the tables, checked: anything out of range is reported and gives a request without new tokens.
__device__ __forceinline__ Request load_request(const Params &p, int b)
{
    Request r;
    const int64_t start = p.c.cu_q[b], end = p.c.cu_q[b + 1], kv = p.c.kv_lens[b], n = end - start;
    if (start < 0 || n < 0 || end > p.c.T || kv < 0 || n > p.max_q || kv > (int64_t)p.c.max_pages * p.c.page_size) {
        raise_status(p.status, PEC_ERR_BAD_INDEX);
        r.start = 0; r.n = 0; r.kv = 0;
        return r;
    }
    r.start = (int32_t)start; r.n = (int32_t)n; r.kv = (int32_t)kv;
    return r;
}
__device__ __forceinline__ bool is_few(const Params &p, const Request &r) { return p.few && r.n > 0 && (int64_t)r.n * p.g <= p.few_limit; }
__device__ __forceinline__ bool is_many(const Params &p, const Request &r) { return r.n > 0 && !is_few(p, r); }
__device__ __forceinline__ int32_t blocks_of(const Params &p, const Request &r) { return (r.n * p.blk_mul + p.blk_div - 1) / p.blk_div; }   // T * g < 2^31

__device__ __forceinline__ int64_t warp_sum(int64_t v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
__device__ __forceinline__ int64_t warp_prefix(int64_t v, int lane)    // inclusive
{
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t up = __shfl_up_sync(0xffffffffu, v, d);
        if (lane >= d) v += up;
    }
    return v;
}

// One item of the many class: rows of one request's block against one slice of its keys, for every KV head.
struct __align__(16) Item {
    Request r;
    int32_t b, block, slices;
    int32_t key_lo, key_hi;                   // key positions of the slice
    int32_t slot;                             // partial slot of KV head 0 (slot * Hkv + kvh), where slices > 1
    int32_t pad[3];
};

// A warp's walk along the few class's line.  The 32 requests around the current one sit in the lanes' registers.  Places on the
// line fit in 32 bits (walk_tiles).
struct Walk {
    int32_t b0, b;                                         // first request of the lanes' group; current request
    Request mine, r;                                       // this lane's, the current one
    int32_t kvh, tile;                                     // current KV head and tile of the request
    int32_t u0;                                            // the unit's first tile on the line
};
__device__ __forceinline__ int32_t warp_prefix32(int32_t v, int lane)    // inclusive
{
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int32_t up = __shfl_up_sync(0xffffffffu, v, d);
        if (lane >= d) v += up;
    }
    return v;
}
__device__ __forceinline__ void walk_take(Walk &w, int src)
{
    w.b = w.b0 + src;
    w.r.start = __shfl_sync(0xffffffffu, w.mine.start, src);
    w.r.n = __shfl_sync(0xffffffffu, w.mine.n, src);
    w.r.kv = __shfl_sync(0xffffffffu, w.mine.kv, src);
}
__device__ __forceinline__ void walk_group(const Params &p, Walk &w, int lane)
{
    w.mine.start = w.mine.n = w.mine.kv = 0;
    if (w.b0 + lane < p.c.B) w.mine = load_request(p, w.b0 + lane);
}
// Tiles of the whole line; leaves the walk's first group of requests in the lanes.  A batch of 2^30 tiles or more (a tile of one
// head is 64 KB: no cache holds as much, but requests may share pages) is reported and given none.
__device__ __forceinline__ int32_t walk_tiles(const Params &p, Walk &w, int lane)
{
    int64_t few = 0;
    for (w.b0 = (p.c.B - 1) & ~31; w.b0 >= 0; w.b0 -= 32) {
        walk_group(p, w, lane);
        if (is_few(p, w.mine)) few += w.mine.tiles();
    }
    few = warp_sum(few) * p.Hkv;
    if (few >= 1 << 30) {
        raise_status(p.status, PEC_ERR_BAD_INDEX);
        few = 0;
    }
    return (int32_t)few;
}
// Tiles per CTA.
__device__ __forceinline__ int32_t few_piece(const Params &p, int32_t all) { return all > 0 ? (all + p.few_ctas - 1) / p.few_ctas : 1; }
// To place `at` on the line (below its end), from the state that walk_tiles leaves.
__device__ __forceinline__ void walk_to(const Params &p, Walk &w, int32_t at, int lane)
{
    int32_t before = 0;
    for (w.b0 = 0; w.b0 < p.c.B; w.b0 += 32) {
        if (w.b0 > 0) walk_group(p, w, lane);
        const int32_t len = is_few(p, w.mine) ? w.mine.tiles() * p.Hkv : 0, end = before + warp_prefix32(len, lane);
        const unsigned who = __ballot_sync(0xffffffffu, at >= end - len && at < end);
        if (who) {
            const int src = __ffs(who) - 1;
            walk_take(w, src);
            const int32_t off = at - __shfl_sync(0xffffffffu, end - len, src), t = w.r.tiles();
            w.kvh = off / t;
            w.tile = off - w.kvh * t;
            w.u0 = at - w.tile;
            return;
        }
        before = __shfl_sync(0xffffffffu, end, 31);
    }
}
// To the first tile of unit `u` in line order; false where there are not so many.
__device__ __forceinline__ bool walk_unit(const Params &p, Walk &w, int32_t u, int lane)
{
    int32_t before = 0, tiles = 0;
    for (w.b0 = 0; w.b0 < p.c.B; w.b0 += 32) {
        if (w.b0 > 0) walk_group(p, w, lane);
        const bool few = is_few(p, w.mine);
        const int32_t units = few ? p.Hkv : 0, len = few ? w.mine.tiles() * p.Hkv : 0;
        const int32_t end = before + warp_prefix32(units, lane), t_end = tiles + warp_prefix32(len, lane);
        const unsigned who = __ballot_sync(0xffffffffu, u >= end - units && u < end);
        if (who) {
            const int src = __ffs(who) - 1;
            walk_take(w, src);
            w.kvh = u - __shfl_sync(0xffffffffu, end - units, src);
            w.tile = 0;
            w.u0 = __shfl_sync(0xffffffffu, t_end - len, src) + w.kvh * w.r.tiles();
            return true;
        }
        before = __shfl_sync(0xffffffffu, end, 31);
        tiles = __shfl_sync(0xffffffffu, t_end, 31);
    }
    return false;
}
// To the next unit (there is one).
__device__ __forceinline__ void walk_next(const Params &p, Walk &w, int lane)
{
    w.u0 += w.r.tiles();
    w.tile = 0;
    if (++w.kvh < p.Hkv) return;
    w.kvh = 0;
    unsigned left = __ballot_sync(0xffffffffu, is_few(p, w.mine) && w.b0 + lane > w.b);
    while (!left && w.b0 + 32 < p.c.B) {
        w.b0 += 32;
        walk_group(p, w, lane);
        left = __ballot_sync(0xffffffffu, is_few(p, w.mine));
    }
    walk_take(w, left ? __ffs(left) - 1 : 0);
}

}  // namespace paged

// Launch that may (`dependent`) start before the preceding kernel of the stream has ended, where that kernel says so.
template <class... A, class... B>
inline cudaError_t launch_dependent(void (*kernel)(A...), dim3 grid, int threads, size_t smem, cudaStream_t stream, bool dependent, B... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = dependent ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, (A)args...);
}

// Launchers (each returns a pec_status).
int launch_paged_plan(const paged::Params &p, cudaStream_t stream);                        // items of the many class
int launch_paged_f32(const paged::Params &p, int64_t items, cudaStream_t stream);       // fp32
int launch_paged_many(const paged::Params &p, int64_t items, cudaStream_t stream);         // bf16
int launch_paged_few(const paged::Params &p, bool after_many, cudaStream_t stream);         // bf16; after_many: overlaps that kernel's end
int launch_paged_many_q4(const paged::Params &p, int64_t items, cudaStream_t stream);      // bf16 queries, a cache held in 4 bits
int launch_paged_few_q4(const paged::Params &p, bool after_many, cudaStream_t stream);      // the same of a cache held in 4 bits, at most kFewRowsQ4 rows
int launch_paged_combine(const paged::Params &p, cudaStream_t stream);

}  // namespace pec
