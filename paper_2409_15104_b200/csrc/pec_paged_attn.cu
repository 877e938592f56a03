// Attention of a batch's new tokens over a paged K/V cache: the entry point, the FMA kernel (fp32 products and state) and the
// kernel that merges partial results.
#include <cuda_bf16.h>
#include <cmath>
#include <numeric>
#include <cuda_runtime.h>
#include "pec_host.h"
#include "pec_internal.h"
#include "pec_paged.h"
#include "pec_paged_plan.cuh"

namespace pec {
namespace paged {

// ------------------------------------------------------------------------------------------ plan
// Items of the many class (bf16: chunks; fp32: every request), one CTA.
//
// Blocks are counted request by request, a request's last block (the one that sees the most keys) first.  A unit of work is a
// block for one KV head; its length is the number of its request's key tiles.  Units up to the last full wave of many_ctas CTAs stay
// whole, unless one is longer than an SM's fair share of all tiles (slice0); of the rest, which would leave SMs idle for a whole
// unit's time, the keys are cut into slices (slice1): as many as fill one, two or three waves, whichever has the shortest
// estimated time, or none.  That holds for units of nearly one length, or for a batch of less than a wave; units of all lengths fill
// the SMs by going longest first, and cutting some of them only adds work.  Both sides (cut / not), 32 / 8 heads: 24 requests of 1 to
// 600 tokens on some 2000, 280-283 / 272-280 us; 40 of 128 on 100 to 3000, 167-199 / 157-174; three of 1024 on 1000, 4000 and 9000,
// 251 / 221; nine of 256 on 4000 and one on 20000, 248 / 226; twelve of 256 on 1000 to 8000, 221-292 / 221-278; six of 512 on 2000 to
// 12000 come out on either side.
// The estimate, in 1/32 of a tile's time: a wave of slices takes its tiles and item_cost for a CTA's
// start and end; a slice's partial, written and read once, merge_cost.  On the tensor cores a tile takes 1.5 us at the full clock (2.1
// in a run of a millisecond and more, at the power limit), start and end 3.5 to 6 us (148 to 888 units of 16 tiles: 27 to 31 us a
// wave), a partial of 132 KB 0.04 us both ways; with the FMA kernel, 17 us a tile, both are next to nothing.
// Slots that cut units take: cutting units of length l into slices of S takes less than sum l / S + their number.  slice0 >= all
// tiles / many_ctas, and units longer than that are fewer than many_ctas: 2 many_ctas.  The tail has less than many_ctas + Hkv
// units of mean length m and slice1 >= m / cuts with cuts * units <= 3 many_ctas: 4 many_ctas + Hkv.
// Items that cutting adds (the grid has a CTA for each, used or not, and one that finds nothing takes its SM 0.6 to 1.5 us: 888 more of
// them, six an SM, cost 24 requests of 300 tokens 9 us of 195, 296 fewer saved 1.2 of 174.9): ceil(l / S) - 1 < l / S of a unit, in all many_ctas for slice0 and 3 many_ctas for slice1.
// Items go into the list longest first (by 256 classes of visible tiles): an SM that falls free late finds short work.  The order
// inside a class is whatever the atomics make it; it changes when an item runs, never what it computes.
constexpr int kPlanThreads = 256, kClasses = 256;

// Inclusive prefix sums of two values per thread over the block, and their totals.
struct Pair { int64_t x, y; };
__device__ __forceinline__ Pair block_prefix(int64_t x, int64_t y, Pair *s_warp, Pair &total)
{
    constexpr int kWarps = kPlanThreads / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Pair v = {warp_prefix(x, lane), warp_prefix(y, lane)};
    __syncthreads();                                                // the previous call's reads are done
    if (lane == 31) s_warp[warp] = v;
    __syncthreads();
    total = {0, 0};
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        const Pair o = s_warp[w];
        if (w < warp) { v.x += o.x; v.y += o.y; }
        total.x += o.x; total.y += o.y;
    }
    return v;
}

__global__ void __launch_bounds__(kPlanThreads)
paged_plan_kernel(const Params p, const int items_cap, const int split_cap)
{
    __shared__ Pair s_warp[kPlanThreads / 32];
    __shared__ int32_t s_item[kPlanThreads], s_split[kPlanThreads], s_slot[kPlanThreads];   // ends (s_slot: starts) of the requests' ranges
    __shared__ int32_t s_start[kPlanThreads], s_n[kPlanThreads], s_kv[kPlanThreads], s_n0[kPlanThreads];
    __shared__ int32_t s_class[kClasses], s_most, s_least;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x;
    const bool one = p.c.B <= kPlanThreads;                         // a request per thread: looked up once
    s_class[tid] = 0;
    if (tid == 0) { s_most = 1; s_least = INT32_MAX; }
    Request r;
    int32_t nb = 0;
    auto take = [&](int b0) {                                       // this thread's request of the group from b0 on
        r.start = r.n = r.kv = 0;
        if (b0 + tid < p.c.B) r = load_request(p, b0 + tid);
        nb = is_many(p, r) ? blocks_of(p, r) : 0;
    };

    // Blocks and tiles of the whole batch; with one group, the place of this thread's first block too.
    int64_t blocks = 0, tiles = 0, place = 0;
    int32_t most = 1, least = INT32_MAX;                            // visible tiles of any block
    for (int b0 = 0; b0 < p.c.B; b0 += kPlanThreads) {
        take(b0);
        blocks += nb; tiles += (int64_t)nb * r.tiles();
        if (nb > 0) {
            most = max(most, r.tiles());
            const int32_t see = p.causal ? min(r.kv, r.pos0() + p.blk_div / p.blk_mul + 1) : r.kv;   // the first block's
            least = min(least, see > 0 ? (see + kKeyTile - 1) / kKeyTile : 1);
        }
    }
    Pair all;
    place = block_prefix(blocks, tiles, s_warp, all).x - blocks;
    // Offsets that go back and forth make requests whose tokens overlap, each fine by itself: more blocks than T tokens can have,
    // and with them more items and slots than the workspace holds.  Such a batch gets no items.
    if (all.x > p.many_blocks) {
        if (tid == 0) {
            raise_status(p.status, PEC_ERR_BAD_INDEX);
            p.many_count[0] = p.many_count[1] = 0;
        }
        return;
    }
    atomicMax(&s_most, most);
    atomicMin(&s_least, least);
    const int32_t tail_at = (int32_t)(all.x * p.Hkv / p.many_ctas * p.many_ctas / p.Hkv);
    const int64_t tail_blocks = all.x - tail_at, units = tail_blocks * p.Hkv;
    const int32_t slice0 = (int32_t)max((all.y * p.Hkv + p.many_ctas - 1) / p.many_ctas, (int64_t)p.min_slice);
    int32_t slice1 = slice0;
    Pair sum;
    if (units > 0) {
        int64_t tail = 0, before = 0;
        for (int b0 = 0; b0 < p.c.B; b0 += kPlanThreads) {
            if (!one) {
                take(b0);
                place = before + block_prefix(nb, 0, s_warp, sum).x - nb;
                before += sum.x;
            }
            tail += min((int64_t)nb, max(place + nb - tail_at, (int64_t)0)) * r.tiles();
        }
        block_prefix(tail, 0, s_warp, sum);
        tail = sum.x;
        const int64_t mean = (tail + tail_blocks - 1) / tail_blocks;
        int64_t best = (units + p.many_ctas - 1) / p.many_ctas * (32 * mean + p.item_cost), len = mean;
        const bool even = 3LL * s_least >= 2LL * s_most;            // (block_prefix has synchronised the block)
        for (int w = 1; w <= 3 && (even || tail_at == 0); ++w) {
            const int32_t cuts = w * p.many_ctas / (int32_t)units;  // slices of a unit of mean length that w waves have room for
            if (cuts < 2) continue;
            const int64_t l = max((mean + cuts - 1) / cuts, (int64_t)p.min_slice);
            const int64_t time = w * (32 * l + p.item_cost) + p.merge_cost * cuts * units;
            if (time < best) { best = time; len = l; }
        }
        if (len < mean) slice1 = (int32_t)min(len, (int64_t)slice0);
    }
    __syncthreads();
    most = s_most;

    int64_t n_items = 0, n_split = 0;
    for (int pass = 0; pass < 2; ++pass) {                          // count the classes; write the items
        int64_t places = 0, slots = 0;
        n_items = n_split = 0;
        for (int b0 = 0; b0 < p.c.B; b0 += kPlanThreads) {
            if (!one) {
                take(b0);
                place = places + block_prefix(nb, 0, s_warp, sum).x - nb;
                places += sum.x;
            }
            const int32_t n0 = (int32_t)min(max(tail_at - place, (int64_t)0), (int64_t)nb), n1 = nb - n0;
            const int32_t c0 = (r.tiles() + slice0 - 1) / slice0, c1 = (r.tiles() + slice1 - 1) / slice1;
            const int64_t items = (int64_t)n0 * c0 + (int64_t)n1 * c1, split = (c0 > 1 ? n0 : 0) + (c1 > 1 ? n1 : 0);
            const int64_t mine = (c0 > 1 ? (int64_t)n0 * c0 : 0) + (c1 > 1 ? (int64_t)n1 * c1 : 0);
            Pair chunk;                                             // items with split blocks above them; slots
            const Pair end = block_prefix(items | split << 32, mine, s_warp, chunk);
            const int32_t chunk_items = (int32_t)chunk.x;
            s_item[tid] = (int32_t)end.x;
            s_split[tid] = (int32_t)(end.x >> 32);
            s_slot[tid] = (int32_t)(slots + end.y - mine);
            s_start[tid] = r.start; s_n[tid] = r.n; s_kv[tid] = r.kv; s_n0[tid] = n0;
            __syncthreads();
            for (int i = tid; i < chunk_items; i += kPlanThreads) {
                int lo = 0, hi = kPlanThreads - 1;                  // the first request whose range ends past i
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (s_item[mid] > i) hi = mid; else lo = mid + 1;
                }
                Item it;
                it.r.start = s_start[lo]; it.r.n = s_n[lo]; it.r.kv = s_kv[lo];
                it.b = b0 + lo;
                const int32_t t = it.r.tiles(), d0 = (t + slice0 - 1) / slice0, d1 = (t + slice1 - 1) / slice1, m0 = s_n0[lo];
                int32_t at = i - (lo > 0 ? s_item[lo - 1] : 0), split_at = lo > 0 ? s_split[lo - 1] : 0, blk, sl;
                it.slot = s_slot[lo];
                if (at < m0 * d0) {
                    blk = at / d0; sl = at - blk * d0;
                    it.slices = d0; it.slot += at; split_at += blk;
                } else {
                    at -= m0 * d0;
                    blk = at / d1; sl = at - blk * d1;
                    it.slices = d1; it.slot += (d0 > 1 ? m0 * d0 : 0) + at; split_at += (d0 > 1 ? m0 : 0) + blk;
                    blk += m0;
                }
                it.block = blocks_of(p, it.r) - 1 - blk;
                const int32_t per = (t + it.slices - 1) / it.slices;
                it.key_lo = (int32_t)min((int64_t)sl * per * kKeyTile, (int64_t)it.r.kv);
                it.key_hi = (int32_t)min((int64_t)(sl + 1) * per * kKeyTile, (int64_t)it.r.kv);
                // Visible tiles: the block's last token sees up to its own position.
                const int32_t last = (int32_t)min((int64_t)it.r.n, (int64_t)(it.block + 1) * p.blk_div / p.blk_mul + 1);
                const int32_t see = p.causal ? min(it.key_hi, it.r.pos0() + last) : it.key_hi;
                const int32_t w = see > it.key_lo ? (see - it.key_lo + kKeyTile - 1) / kKeyTile : 0;
                const int32_t cls = kClasses - 1 - (int32_t)((float)w / (float)most * (kClasses - 1));
                if (pass == 0) {
                    atomicAdd(&s_class[cls], 1);
                } else {
                    const int to = atomicAdd(&s_class[cls], 1);
                    it.pad[0] = it.pad[1] = it.pad[2] = 0;
                    if (to < items_cap) p.many_items[to] = it;
                    if (it.slices > 1 && sl == 0 && n_split + split_at < split_cap) p.many_split[n_split + split_at] = it;
                }
            }
            n_items += chunk_items; n_split += chunk.x >> 32; slots += chunk.y;
            __syncthreads();
        }
        if (pass == 0) {                                            // sizes of the classes -> their starts
            const int32_t size = s_class[tid];
            const int64_t end = block_prefix(size, 0, s_warp, sum).x;
            s_class[tid] = (int32_t)end - size;
            __syncthreads();
        }
    }
    if (tid == 0) {
        p.many_count[0] = (int32_t)min(n_items, (int64_t)items_cap);   // (the caps are never reached, see above)
        p.many_count[1] = (int32_t)min(n_split, (int64_t)split_cap);
    }
}
static_assert(kClasses == kPlanThreads, "a class per thread");

// ------------------------------------------------------------------------------------------ FMA kernel
// One CTA = 64 packed rows of one KV head against one slice of the request's keys, 64 keys at a time.  256 threads as 16 x 16:
// thread (ty, tx) owns score rows 4 ty .. + 3 and keys tx + 16 j, and output rows 4 ty .. + 3 with channels 4 tx .. + 3 and
// 64 + 4 tx .. + 3.  Rows, keys and values past their ends are zero in shared memory, so that what a page holds past the
// request's end never meets a product.
// Bound by the FMA pipe: per four channels a warp's 16 + 16 micro-tile takes 32 packed FMA instructions (64 issue slots of the
// pipe) and 12 shared-memory wavefronts, per four keys of P V 64 (128) and 20; packed, they leave issue slots for the rest.
// The probabilities take the place of the key tile, which keeps a CTA at 100 KB and two of them on an SM: one's loads and
// barriers run under the other's arithmetic.  Tiles come by asynchronous copies, the values' while the scores are worked out.
// Measured on three fp32 requests (741 rows, 8 heads, 2.5 GFLOP visible, 3.2 computed): 108 us, where the FMA pipe alone would take
// 45 (8 x 4 scores a thread, 128 threads, a third less shared-memory traffic: 113 us).
constexpr int kBM = 64, kBN = 64, kThreads = 256;
constexpr int kLd = kHeadDim + 4, kLdP = kBN + 4;
constexpr size_t kF32Smem = sizeof(float) * (2 * kBM * kLd + kBN * kHeadDim);

// 16 bytes to shared memory, zeros where !ok (nothing is read then).
__device__ __forceinline__ void copy16(float *dst, const float *src, bool ok)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

__global__ void __launch_bounds__(kThreads, 2)
paged_f32_kernel(const Params p)
{
    extern __shared__ __align__(16) float smem[];
    float *sQ = smem;                       // [kBM][kLd]
    float *sK = sQ + kBM * kLd;             // [kBN][kLd]
    float *sV = sK + kBN * kLd;             // [kBN][kHeadDim]
    float *sP = sK;                         // [kBM][kLdP], once the scores are done with the keys
    __shared__ int32_t s_page[kBN];
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, kvh = blockIdx.x % p.Hkv;
    asm volatile("griddepcontrol.wait;" ::: "memory");              // launched ahead of the plan's end
    if ((int)(blockIdx.x / p.Hkv) >= p.many_count[0]) return;
    const Item it = p.many_items[blockIdx.x / p.Hkv];
    const int32_t row0 = it.block * kBM, rows = min(kBM, it.r.n * p.g - row0);

    for (int i = tid; i < kBM * (kHeadDim / 4); i += kThreads) {
        const int r = i / (kHeadDim / 4), c = (i % (kHeadDim / 4)) * 4;
        const int32_t rr = min(r, rows - 1), t = (row0 + rr) / p.g, h = kvh * p.g + (row0 + rr) % p.g;
        copy16(sQ + r * kLd + c, static_cast<const float *>(p.q) + (int64_t)(it.r.start + t) * p.q_st + (int64_t)h * p.q_sh + c, r < rows);
    }

    float m_run[4], l_run[4];
    float2 acc[4][4];                        // channels 4 tx .. + 3, 64 + 4 tx .. + 3
    int32_t lim[4];                          // keys below it are visible to the row
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m_run[i] = -INFINITY; l_run[i] = 0.f;
        const int32_t r = row0 + ty * 4 + i, pos = it.r.pos0() + r / p.g;
        lim[i] = p.causal ? min(it.key_hi, pos + 1) : it.key_hi;
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[i][c] = make_float2(0.f, 0.f);
    }
    const int32_t last = it.r.pos0() + (row0 + rows - 1) / p.g;
    const int32_t end = p.causal ? min(it.key_hi, last + 1) : it.key_hi;

    for (int32_t k0 = it.key_lo; k0 < end; k0 += kBN) {
        if (tid < kBN) {                     // page of each key of the tile; -1: past the end, or a bad page number
            int32_t page = -1;
            if (k0 + tid < it.key_hi) {
                page = p.c.table[it.b * p.c.table_stride + (k0 + tid) / p.c.page_size];
                if (page < 0 || page >= p.c.num_pages) { raise_status(p.status, PEC_ERR_BAD_INDEX); page = -1; }
            }
            s_page[tid] = page;
        }
        __syncthreads();                     // ... and the previous tile's reads are done
        // A warp copies whole rows of 512 bytes, eight of each tile: warp w rows w, w + 8, ...
        const int c4 = (tid & 31) * 4;
        int64_t page[8];
        int32_t slot[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = (tid >> 5) + 8 * i;
            page[i] = s_page[r];
            slot[i] = (k0 + r) % p.c.page_size;
            const bool ok = page[i] >= 0;
            const float *src = static_cast<const float *>(p.k_pages) + (ok ? page[i] * p.c.k_sp + slot[i] * p.c.k_st : 0) + (int64_t)kvh * p.c.k_sh + c4;
            copy16(sK + r * kLd + c4, src, ok);
        }
        copy_commit();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = (tid >> 5) + 8 * i;
            const bool ok = page[i] >= 0;
            const float *src = static_cast<const float *>(p.v_pages) + (ok ? page[i] * p.c.v_sp + slot[i] * p.c.v_st : 0) + (int64_t)kvh * p.c.v_sh + c4;
            copy16(sV + r * kHeadDim + c4, src, ok);
        }
        copy_commit();
        copy_wait<1>();                      // the keys (and Q)
        __syncthreads();

        // Packed FMAs: each half of s2 sums every second channel.
        float2 s2[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) s2[i][j] = make_float2(0.f, 0.f);
#pragma unroll 2
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
                    s2[i][j] = __ffma2_rn(make_float2(qa[i].x, qa[i].y), make_float2(kb[j].x, kb[j].y), s2[i][j]);
                    s2[i][j] = __ffma2_rn(make_float2(qa[i].z, qa[i].w), make_float2(kb[j].z, kb[j].w), s2[i][j]);
                }
        }
        __syncthreads();                     // every warp is done with the keys: P may take their place
        // Mask by choice, not by adding -inf: a masked score may be anything.  State replicated over a row's 16 threads.
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float mx = -INFINITY, s[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[j] = (k0 + tx + 16 * j < lim[i]) ? (s2[i][j].x + s2[i][j].y) * p.scale_log2 : -INFINITY;
                mx = fmaxf(mx, s[j]);
            }
#pragma unroll
            for (int o = 8; o >= 1; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float m_new = fmaxf(m_run[i], mx);
            const float m_use = (m_new == -INFINITY) ? 0.f : m_new;
            const float alpha = exp2f(m_run[i] - m_use);           // 0 while the row is still empty
            float rs = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float pj = exp2f(s[j] - m_use);
                rs += pj;
                sP[(ty * 4 + i) * kLdP + tx + 16 * j] = pj;
            }
#pragma unroll
            for (int o = 8; o >= 1; o >>= 1) rs += __shfl_xor_sync(0xffffffffu, rs, o);
            l_run[i] = l_run[i] * alpha + rs;
            m_run[i] = m_new;
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[i][c] = __fmul2_rn(acc[i][c], make_float2(alpha, alpha));
        }
        copy_wait<0>();                      // the values
        __syncthreads();
#pragma unroll 2
        for (int j = 0; j < kBN; j += 4) {
            float pr[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<float4 *>(pr[i]) = *reinterpret_cast<const float4 *>(sP + (ty * 4 + i) * kLdP + j);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float4 v0 = *reinterpret_cast<const float4 *>(sV + (j + x) * kHeadDim + tx * 4);
                const float4 v1 = *reinterpret_cast<const float4 *>(sV + (j + x) * kHeadDim + 64 + tx * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 w = make_float2(pr[i][x], pr[i][x]);
                    acc[i][0] = __ffma2_rn(w, make_float2(v0.x, v0.y), acc[i][0]);
                    acc[i][1] = __ffma2_rn(w, make_float2(v0.z, v0.w), acc[i][1]);
                    acc[i][2] = __ffma2_rn(w, make_float2(v1.x, v1.y), acc[i][2]);
                    acc[i][3] = __ffma2_rn(w, make_float2(v1.z, v1.w), acc[i][3]);
                }
            }
        }
    }
    copy_wait<0>();                          // Q's copies, where there was no tile

    const int64_t slot = (int64_t)it.slot * p.Hkv + kvh;
    if (it.slices > 1 && slot >= p.many_cap) return;               // cannot happen (see paged_plan_kernel); never write past the scratch
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int32_t r = ty * 4 + i;
        if (r >= rows) continue;
        const bool empty = l_run[i] == 0.f;                          // a NaN sum is not: it reaches o and lse
        const float inv = empty ? 0.f : 1.f / l_run[i];
        const float lse = empty ? -INFINITY : m_run[i] * 0.6931471805599453f + logf(l_run[i]);
        float out[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) out[c] = empty ? 0.f : (c & 1 ? acc[i][c / 2].y : acc[i][c / 2].x) * inv;
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
// A CTA merges the partial results of some packed rows of one unit: a (request, KV head) whose tiles cross a cut of the line, or a
// block of rows whose keys are cut into slices (listed by the plan).  Units are enumerated by what splits them - CTA c of the few
// class looks at cut c and takes the unit around it if this is the unit's first cut - or, where there are fewer units than cuts, one
// by one, so that the grid has the size of what can be split, not of the batch.  (A CTA per token and KV head took 66 us to find
// nothing to do for 2048 tokens; 32 tokens over 32000, 8 units: 61 us by cut, 40 by unit.)  The few class looks its unit up before
// the attention kernels end (the tables were complete before they began); partials are read afterwards, and no CTA ends before that
// wait, so that whatever follows on the stream follows those kernels too.
// A warp merges one row at a time, a lane owning four channels: the largest LSE first, then the weighted sum, sixteen partials'
// loads in flight.  Bound by latency: two dependent reads, 3 to 4 us with the launch.
constexpr int kCombineWarps = 8, kManyGroup = 32;

__device__ __forceinline__ void combine_row(const Params &p, const float *po, const float *pl, int64_t at0, int64_t shift, int64_t step,
                                            int count, int64_t item, int lane)
{
    constexpr int kBatch = 16;                                    // partials' rows in flight
    auto place = [&](int s) { return at0 + s * step + (s == 0 ? shift : 0); };     // of partial s, in rows
    float l = lane < count ? pl[place(lane)] : -INFINITY, m = l;   // lane s: the LSE of partial s of the current 32
    bool some = l != -INFINITY;                                   // a partial with keys, NaN among them (which the maximum passes over)
    for (int s = lane + 32; s < count; s += 32) {
        const float x = pl[place(s)];
        some = some || x != -INFINITY;
        m = fmaxf(m, x);
    }
    some = __any_sync(0xffffffffu, some);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    float tot = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < count && some; s0 += 32) {
        if (s0 > 0) l = s0 + lane < count ? pl[place(s0 + lane)] : -INFINITY;
        const float w = l == -INFINITY ? 0.f : expf(l - m);
        tot += w;
        for (int b = 0; b < 32 && s0 + b < count; b += kBatch) {
            float4 v[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (s0 + b + i < count) v[i] = *reinterpret_cast<const float4 *>(po + place(s0 + b + i) * kHeadDim + 4 * lane);
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const float x = __shfl_sync(0xffffffffu, w, b + i);
                acc.x = fmaf(x, v[i].x, acc.x); acc.y = fmaf(x, v[i].y, acc.y); acc.z = fmaf(x, v[i].z, acc.z); acc.w = fmaf(x, v[i].w, acc.w);
            }
        }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) tot += __shfl_xor_sync(0xffffffffu, tot, d);
    const float inv = some ? 1.f / tot : 0.f;
    acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
    if (p.o_is_bf16) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(acc.x, acc.y), hi = __floats2bfloat162_rn(acc.z, acc.w);
        *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(p.o) + item * kHeadDim + 4 * lane) =
            make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
    } else {
        *reinterpret_cast<float4 *>(static_cast<float *>(p.o) + item * kHeadDim + 4 * lane) = acc;
    }
    if (lane == 0) p.lse[item] = some ? m + logf(tot) : -INFINITY;
}

__global__ void __launch_bounds__(kCombineWarps * 32, 2)
paged_combine_kernel(const Params p, const int by_unit, const int few_groups, const int few_blocks, const int many_groups)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if ((int)blockIdx.x < few_blocks) {
        const int32_t nth = blockIdx.x / few_groups;
        const int group = blockIdx.x % few_groups;
        Walk w;
        const int32_t all = walk_tiles(p, w, lane), piece = few_piece(p, all);
        bool mine;
        if (by_unit) {
            mine = all > 0 && walk_unit(p, w, nth, lane);
        } else {
            const int32_t at = (nth + 1) * piece;                // few_ctas * 2^23 at most
            mine = at < all;
            if (mine) walk_to(p, w, at, lane);
            mine = mine && w.u0 < at && w.u0 >= at - piece;      // else the cut falls between units, or is not the unit's first
        }
        asm volatile("griddepcontrol.wait;" ::: "memory");
        if (!mine) return;
        const int64_t first = w.u0 / piece;                      // piece with the unit's first tiles
        const int count = (w.u0 + w.r.tiles() - 1) / piece - (int)first + 1;
        if (count == 1) return;
        for (int row = group * kCombineWarps + warp; row < w.r.n * p.g; row += few_groups * kCombineWarps) {
            const int64_t item = (int64_t)(w.r.start + row / p.g) * p.Hq + w.kvh * p.g + row % p.g;
            combine_row(p, p.few_o, p.few_lse, 2 * first * p.few_rows + row, w.u0 > first * piece ? p.few_rows : 0, 2 * (int64_t)p.few_rows,
                        count, item, lane);
        }
    } else {
        // The blocks that are cut, from the plan's list.
        asm volatile("griddepcontrol.wait;" ::: "memory");
        const int64_t n = (int64_t)p.many_count[1] * p.Hkv * many_groups;
        for (int64_t x = blockIdx.x - few_blocks; x < n; x += gridDim.x - few_blocks) {
            const int group = (int)(x % many_groups), kvh = (int)(x / many_groups % p.Hkv);
            const Item it = p.many_split[x / many_groups / p.Hkv];
            for (int i = warp; i < kManyGroup; i += kCombineWarps) {
                const int row = group * kManyGroup + i;          // of the block
                const int32_t packed = it.block * p.many_rows + row;
                if (row >= p.many_rows || packed >= it.r.n * p.g) break;
                const int64_t item = (int64_t)(it.r.start + packed / p.g) * p.Hq + kvh * p.g + packed % p.g;
                combine_row(p, p.many_o, p.many_lse, ((int64_t)it.slot * p.Hkv + kvh) * p.many_rows + row, 0, (int64_t)p.Hkv * p.many_rows,
                            it.slices, item, lane);
            }
        }
    }
}

}  // namespace paged

using namespace paged;

// The kernel that follows starts as this one does and waits for its end before it reads the list.
int launch_paged_plan(const Params &p, cudaStream_t stream)
{
    paged_plan_kernel<<<1, kPlanThreads, 0, stream>>>(p, p.items_cap, p.many_cap / 2);
    const cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess) { set_error("pec_paged_attn: launch failed: %s", cudaGetErrorString(err)); return PEC_ERR_CUDA; }
    return PEC_OK;
}

int launch_paged_f32(const Params &p, int64_t items, cudaStream_t stream)
{
    static unsigned char ready[host::kMaxDevices] = {};
    static std::mutex ready_mutex;
    if (!host::once_per_device(ready, ready_mutex, [] {
            return cudaFuncSetAttribute(paged_f32_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kF32Smem) == cudaSuccess; })) {
        (void)cudaGetLastError();
        set_error("pec_paged_attn: cannot raise the shared-memory limit");
        return PEC_ERR_CUDA;
    }
    if (items * p.Hkv > 0x7fffffff) { set_error("pec_paged_attn: grid too large"); return PEC_ERR_UNSUPPORTED; }
    cudaError_t err = launch_dependent(paged_f32_kernel, dim3((unsigned)(items * p.Hkv)), kThreads, kF32Smem, stream, true, p);
    if (err == cudaSuccess) err = cudaGetLastError();
    if (err != cudaSuccess) { set_error("pec_paged_attn: launch failed: %s", cudaGetErrorString(err)); return PEC_ERR_CUDA; }
    return PEC_OK;
}

int launch_paged_combine(const Params &p, cudaStream_t stream)
{
    // Every cut of the line; every block that can be cut: one has two slots or more.
    // One row a warp where the units are so few that this takes no more than two CTAs per SM.
    const int64_t units = (int64_t)(p.c.B < p.c.T ? p.c.B : p.c.T) * p.Hkv;
    const int by_unit = units < p.few_ctas, most_groups = (p.few_rows + kCombineWarps - 1) / kCombineWarps;
    int few_groups = by_unit ? (int)(2 * p.few_ctas / units) : 2, few_blocks = 0;
    if (few_groups > most_groups) few_groups = most_groups;
    if (p.few) few_blocks = (by_unit ? (int)units : p.few_ctas - 1) * few_groups;
    const int many_groups = (p.many_rows + kManyGroup - 1) / kManyGroup;
    const int64_t most = (int64_t)p.many_cap / 2 * many_groups;      // a block that is cut has two slots or more
    const int many_blocks = (int)(most < 2 * p.many_ctas ? most : 2 * p.many_ctas);
    if (few_blocks + many_blocks == 0) return PEC_OK;
    cudaError_t err = launch_dependent(paged_combine_kernel, dim3((unsigned)(few_blocks + many_blocks)), kCombineWarps * 32, 0, stream, true,
                                       p, by_unit, few_groups, few_blocks, many_groups);
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

// false: the numbers do not fit a tensor map's 32-bit coordinate.
static bool fold_pages(int64_t sp, int64_t sh, int64_t num_pages, int64_t Hkv, FoldedPages &f)
{
    if (num_pages == 1) sp = 0;               // strides that no address uses
    if (Hkv == 1) sh = 0;
    const int64_t unit = std::gcd(sp, sh), most = ((int64_t)1 << 31) - 1;
    f = {unit > 0 ? unit : kHeadDim, 0, 0};
    const int64_t page = sp / f.unit, head = sh / f.unit;
    if (page > most || head > most || (num_pages - 1) * page > most || (num_pages - 1) * page + (Hkv - 1) * head > most) return false;
    f.page = (int32_t)page; f.head = (int32_t)head;
    return true;
}

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
    if (a->T * (a->Hq / a->Hkv) > ((int64_t)1 << 31) - 1024) { set_error("%s: T * Hq / Hkv near 2^31 or above unsupported", who); return PEC_ERR_UNSUPPORTED; }
    if (a->dtype == PEC_BF16 && !(fold_pages(p.c.k_sp, p.c.k_sh, p.c.num_pages, a->Hkv, p.fk) && fold_pages(p.c.v_sp, p.c.v_sh, p.c.num_pages, a->Hkv, p.fv))) {
        set_error("%s: the pages reach over 2^31 times the greatest common divisor of their page and head strides", who);
        return PEC_ERR_UNSUPPORTED;
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
    // Blocks of the many class, the grid bound and the partial slots it may take (see paged_plan_kernel).
    const int tps = kFewRows / p.g;           // tensor cores: two stages of whole tokens; FMA: 64 packed rows
    p.blk_mul = tensor ? 1 : p.g; p.blk_div = tensor ? 2 * tps : kBM;
    p.many_rows = tensor ? 2 * tps * p.g : kBM;
    p.many_ctas = tensor ? sms : 2 * sms;
    p.min_slice = tensor ? 2 : 1;
    p.item_cost = tensor ? 96 : 8;
    p.merge_cost = tensor ? 1 : 0;
    c.many_items = 0;
    if (!p.few || (int64_t)p.max_q * p.g > kFewRows) {
        const int64_t shortest = p.few ? kFewRows / p.g + 1 : 1, most = a->T / shortest;       // new tokens of such a request; how many there can be
        const int64_t blocks = a->T * p.blk_mul / p.blk_div + (a->B < most ? a->B : most);
        c.many_items = blocks + ceil_div(4 * (int64_t)p.many_ctas, p.Hkv) + 2;                 // blocks and what cutting adds to them
        const int64_t most_slices = ceil_div(ceil_div((int64_t)a->max_pages * a->page_size, kKeyTile), p.min_slice);
        int64_t cap = 6 * (int64_t)p.many_ctas + p.Hkv;
        if (most_slices <= 1) cap = 0;
        else if (blocks * most_slices * p.Hkv < cap) cap = blocks * most_slices * p.Hkv;
        p.many_cap = (int32_t)cap;
        if (c.many_items > ((int64_t)1 << 26)) { set_error("%s: more than 2^26 blocks of rows unsupported", who); return PEC_ERR_UNSUPPORTED; }
        p.many_blocks = (int32_t)blocks;
    }
    p.items_cap = (int32_t)c.many_items;
    const size_t slots = (((size_t)p.many_cap * p.many_rows * (kHeadDim + 1)) + 3) & ~(size_t)3;
    const size_t list = c.many_items > 0 ? 4 + (c.many_items + p.many_cap / 2) * sizeof(Item) / sizeof(float) : 0;
    c.bytes = (floats + slots + list) * sizeof(float);
    if (a->workspace) {
        float *ws = static_cast<float *>(a->workspace);
        p.few_o = ws;
        p.few_lse = ws + 2 * (size_t)p.few_ctas * p.few_rows * kHeadDim;
        p.many_o = ws + floats;
        p.many_lse = p.many_o + (size_t)p.many_cap * p.many_rows * kHeadDim;
        p.many_count = reinterpret_cast<int32_t *>(ws + floats + slots);
        p.many_items = reinterpret_cast<Item *>(p.many_count + 4);
        p.many_split = p.many_items + p.items_cap;
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
    if (c.many_items > 0) rc = launch_paged_plan(c.p, stream);
    if (rc == PEC_OK && c.many_items > 0) rc = args->dtype == PEC_BF16 ? launch_paged_many(c.p, c.many_items, stream) : launch_paged_f32(c.p, c.many_items, stream);
    if (rc == PEC_OK && c.p.few) rc = launch_paged_few(c.p, c.many_items > 0, stream);
    if (rc != PEC_OK || c.bytes == 0) return rc;
    return launch_paged_combine(c.p, stream);
}
