// How a batch's work is cut for the kernels behind pec_paged_attn, worked out on the device by every CTA from the tables
// themselves (no host plan: a captured graph replays with whatever lengths the tables then hold).
//
// Query rows are packed: the g = Hq / Hkv heads of a KV head and the new tokens of a request are the rows of one matrix,
// row = token * g + head of the group, so that a key tile read once serves all of them.
//
// Two classes of requests, by their packed rows n * g:
//   few  (at most 128: decode steps)  worked on by a persistent grid.  The key tiles of all (request, KV head) pairs lie on
//        one line that is cut into equal pieces, one per CTA; a pair that crosses a cut leaves one partial result per piece.
//   many (chunks)                     blocks of rows, each block's keys cut into slices where a unit of work would be longer
//        than an SM's fair share of the whole.
// Partials are merged by their LSE by one kernel for both classes (combine), which finds them by the same arithmetic.
#pragma once
#include "pec_internal.h"
#include "pec_paged.h"

namespace pec {
namespace paged {

constexpr int kKeyTile = 128;                 // keys per tile
constexpr int kFewRows = 128;                 // packed rows of the few class
constexpr int kMinSliceTiles = 4;             // shortest slice of the many class: its partial costs as much traffic as 1-2 tiles
constexpr int64_t kNoSplit = (int64_t)1 << 40;

// Device-side description of one call, passed to the kernels by value.
struct Params {
    const void *q, *k_pages, *v_pages;
    int64_t q_st, q_sh;
    PagedCache c;
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
    int32_t few_ctas;
    int32_t few_rows;                         // rows of a partial slot
    float *few_o, *few_lse;                   // [2 * few_ctas][few_rows][128], [..][few_rows]
    // many class: blocks of a request = ceil(n * blk_mul / blk_div)
    int32_t blk_mul, blk_div;
    int32_t many_slots;                       // fair share = all tiles / many_slots
    int32_t many_rows;                        // rows of a partial slot
    int32_t many_cap;                         // slots that the workspace holds
    float *many_o, *many_lse;
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
__device__ __forceinline__ bool is_few(const Params &p, const Request &r) { return p.few && r.n > 0 && (int64_t)r.n * p.g <= kFewRows; }
__device__ __forceinline__ bool is_many(const Params &p, const Request &r) { return r.n > 0 && !is_few(p, r); }
__device__ __forceinline__ int32_t blocks_of(const Params &p, const Request &r) { return (int32_t)(((int64_t)r.n * p.blk_mul + p.blk_div - 1) / p.blk_div); }

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

// Key tiles of the whole batch, per KV head.  One converged warp.
__device__ __forceinline__ void batch_tiles(const Params &p, int64_t &few, int64_t &many)
{
    const int lane = threadIdx.x & 31;
    few = many = 0;
    for (int b = lane; b < p.c.B; b += 32) {
        const Request r = load_request(p, b);
        if (is_few(p, r)) few += r.tiles();
        else if (is_many(p, r)) many += (int64_t)blocks_of(p, r) * r.tiles();
    }
    few = warp_sum(few);
    many = warp_sum(many);
}
// few: tiles per CTA.  many: tiles per slice; a request is cut into ceil(tiles / slice) slices of equal length.
// Slots that split requests take: each has tiles > S, so ceil(tiles / S) < 2 tiles / S, and S >= many * Hkv / many_slots makes
// the sum over all of them, times Hkv, less than 2 * many_slots.
__device__ __forceinline__ int64_t few_piece(const Params &p, int64_t few)
{
    const int64_t all = few * p.Hkv;
    return all > 0 ? (all + p.few_ctas - 1) / p.few_ctas : 1;
}
__device__ __forceinline__ int64_t many_slice(const Params &p, int64_t many)
{
    const int64_t s = (many * p.Hkv + p.many_slots - 1) / p.many_slots;
    return s < kMinSliceTiles ? kMinSliceTiles : s;
}
__device__ __forceinline__ int32_t slices_of(const Request &r, int64_t slice) { return (int32_t)((r.tiles() + slice - 1) / slice); }

// One item of the many class: rows of one request's block against one slice of its keys (for one KV head, the grid's y).
struct Item {
    Request r;
    int32_t b, block, slices;
    int32_t key_lo, key_hi;                   // key positions of the slice
    int64_t slot;                             // partial slot of KV head 0 (slot * Hkv + kvh), where slices > 1
};
// Item `idx`; one converged warp, every lane returns the same.  False past the last item.
__device__ __forceinline__ bool locate_many(const Params &p, int64_t idx, Item &it)
{
    const int lane = threadIdx.x & 31;
    int64_t few, many;
    batch_tiles(p, few, many);
    if (many == 0) return false;
    const int64_t slice = many_slice(p, many);
    int64_t before = 0, slots = 0;            // items and partial slots of earlier groups of 32 requests
    for (int b0 = 0; b0 < p.c.B; b0 += 32) {
        Request r;
        r.start = r.n = r.kv = 0;
        if (b0 + lane < p.c.B) r = load_request(p, b0 + lane);
        int64_t items = 0, mine = 0;
        int32_t ns = 0;
        if (is_many(p, r)) {
            ns = slices_of(r, slice);
            items = (int64_t)blocks_of(p, r) * ns;
            mine = ns > 1 ? items : 0;
        }
        const int64_t incl = warp_prefix(items, lane), incl_s = warp_prefix(mine, lane);
        const unsigned who = __ballot_sync(0xffffffffu, idx >= before + incl - items && idx < before + incl);
        if (who) {
            const int src = __ffs(who) - 1;
            it.b = b0 + src;
            it.r.start = __shfl_sync(0xffffffffu, r.start, src);
            it.r.n = __shfl_sync(0xffffffffu, r.n, src);
            it.r.kv = __shfl_sync(0xffffffffu, r.kv, src);
            it.slices = __shfl_sync(0xffffffffu, ns, src);
            const int64_t at = idx - __shfl_sync(0xffffffffu, before + incl - items, src);
            const int64_t first_slot = __shfl_sync(0xffffffffu, slots + incl_s - mine, src);
            // The last block sees the most keys: it goes first.
            const int32_t nb = blocks_of(p, it.r), blk = (int32_t)(at / it.slices), sl = (int32_t)(at % it.slices);
            it.block = nb - 1 - blk;
            const int32_t per = (it.r.tiles() + it.slices - 1) / it.slices;
            it.key_lo = min((int64_t)sl * per * kKeyTile, (int64_t)it.r.kv);
            it.key_hi = min((int64_t)(sl + 1) * per * kKeyTile, (int64_t)it.r.kv);
            it.slot = first_slot + (int64_t)it.block * it.slices + sl;
            return true;
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
        slots += __shfl_sync(0xffffffffu, incl_s, 31);
    }
    return false;
}

// A warp's walk along the few class's line.  The 32 requests around the current one sit in the lanes' registers.
struct Walk {
    int32_t b0, b;                                         // first request of the lanes' group; current request
    Request mine, r;                                       // this lane's, the current one
    int32_t kvh, tile;                                     // current KV head and tile of the request
    int64_t u0;                                            // the unit's first tile on the line
};
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
// To place `at` on the line (below its end).
__device__ __forceinline__ void walk_to(const Params &p, Walk &w, int64_t at, int lane)
{
    int64_t before = 0;
    for (w.b0 = 0; w.b0 < p.c.B; w.b0 += 32) {
        walk_group(p, w, lane);
        const int64_t len = is_few(p, w.mine) ? (int64_t)w.mine.tiles() * p.Hkv : 0, incl = warp_prefix(len, lane);
        const unsigned who = __ballot_sync(0xffffffffu, at >= before + incl - len && at < before + incl);
        if (who) {
            const int src = __ffs(who) - 1;
            walk_take(w, src);
            const int64_t off = at - __shfl_sync(0xffffffffu, before + incl - len, src);
            w.kvh = (int32_t)(off / w.r.tiles());
            w.tile = (int32_t)(off % w.r.tiles());
            w.u0 = at - w.tile;
            return;
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
    }
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

// Block `idx` of the requests of the many class whose keys are cut (in the order of their slots); one converged warp.
struct SplitBlock {
    Request r;
    int32_t block, slices;
    int64_t first;                            // slots (first + s) * Hkv + kvh
};
__device__ __forceinline__ bool locate_split(const Params &p, int64_t idx, SplitBlock &out)
{
    const int lane = threadIdx.x & 31;
    int64_t few, many;
    batch_tiles(p, few, many);
    if (many == 0) return false;
    const int64_t slice = many_slice(p, many);
    int64_t before = 0, slots = 0;
    for (int b0 = 0; b0 < p.c.B; b0 += 32) {
        Request r;
        r.start = r.n = r.kv = 0;
        if (b0 + lane < p.c.B) r = load_request(p, b0 + lane);
        const int32_t ns = is_many(p, r) ? slices_of(r, slice) : 0;
        const int64_t blocks = ns > 1 ? blocks_of(p, r) : 0, incl = warp_prefix(blocks, lane), incl_s = warp_prefix(blocks * ns, lane);
        const unsigned who = __ballot_sync(0xffffffffu, idx >= before + incl - blocks && idx < before + incl);
        if (who) {
            const int src = __ffs(who) - 1;
            out.r.start = __shfl_sync(0xffffffffu, r.start, src);
            out.r.n = __shfl_sync(0xffffffffu, r.n, src);
            out.r.kv = __shfl_sync(0xffffffffu, r.kv, src);
            out.slices = __shfl_sync(0xffffffffu, ns, src);
            out.block = (int32_t)(idx - __shfl_sync(0xffffffffu, before + incl - blocks, src));
            out.first = __shfl_sync(0xffffffffu, slots + incl_s - blocks * ns, src) + (int64_t)out.block * out.slices;
            return true;
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
        slots += __shfl_sync(0xffffffffu, incl_s, 31);
    }
    return false;
}

}  // namespace paged

// Launchers (each returns a pec_status).
int launch_paged_simple(const paged::Params &p, int64_t items, cudaStream_t stream);       // fp32
int launch_paged_many(const paged::Params &p, int64_t items, cudaStream_t stream);         // bf16
int launch_paged_few(const paged::Params &p, cudaStream_t stream);
int launch_paged_combine(const paged::Params &p, cudaStream_t stream);

}  // namespace pec
