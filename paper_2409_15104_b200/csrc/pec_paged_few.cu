// Paged attention of requests with few packed rows (n * g <= 128: decode steps) on the sm_100a tensor cores.
//
// Bound by the K/V stream from HBM: 2 * kv * Hkv * 256 bytes a request, each byte read once for all the rows of its KV head.
// The kernel is persistent, one CTA per SM.  The key tiles of all (request, KV head) units lie on one line, request by request
// and head by head, and each CTA walks an equal piece of it (few_piece), so that every SM streams the same number of bytes
// whatever the requests' lengths; a unit inside one piece is finished there, one that crosses a cut leaves a partial result
// per piece for the combining kernel.  A unit's part in a piece is a "segment".
//
// Warp roles (three warpgroups):
//   warps 0-3, 4-7  softmax and epilogue of even and odd segments; with two groups the epilogue of one segment runs beside the
//                   first tiles of the next
//   warp 8          MMA issuer       warp 9  TMA loader: segment descriptors, Q (two buffers), K and V tiles (a ring)
//   warps 10-11     idle
// The loader runs through segment borders, so the stream from memory does not stop at them.
//
// Two forms of the products, by the number of packed rows that a request can have:
//   wide    S = Q K^T and O = P V with the rows as the 128 rows of the product (a thread = a row = a TMEM lane; warps whose 32
//           rows are all past the segment's only keep the barriers in step).  P (bf16) is written over S.
//           TMEM columns: S [0, 256), two buffers; O [256, 512), one per group.
//   narrow  up to 16 rows: S^T = K Q^T and O^T = V^T P^T with the rows as 16 columns (a thread = a key, then a channel).  A row's
//           maximum and sum run across threads, but a tile costs 3/16 of the tensor work and 1/16 of the exponentials.  P goes
//           through 8 KB of shared memory, as two bf16 parts: 0 to 2.5 % slower than as one, and a bf16 result errs by its own
//           rounding alone.  What it is for is a long run: the wide form draws the 1 kW limit, the SM clock falls to 1.5 GHz and
//           the stream with it - three requests of 131072 keys, 64 / 8 heads, 5.55 TB/s for seconds (6.37 in a short run)
//           against 6.46 (6.65); 64 requests of 2400 keys on average, 32 / 8 heads, 4.88 against 5.65.
//           Both sides of 16 rows, short runs, 64 requests of 3000 keys: 16 rows 131 us against the wide form's 135; 32 rows in 32
//           columns 260 against 138, the exponentials and stores of P per key no longer fit under the stream.
//           TMEM columns: S^T [0, 32), two buffers; O^T [32, 64), one per group.
//
// Per tile: S(n) into one of two TMEM buffers, P(n) into its place or one of two shared buffers, O += P V.  The issuer's order
// S(n + 1), PV(n) has the next scores ready when the softmax comes back for them; S(n + 2) may overwrite S(n) or P(n) because
// the issuing thread's products execute in order.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include "pec_paged_tma.cuh"

namespace pec {
using namespace sm100;
namespace paged {
namespace few {

constexpr int kThreads = 384;
constexpr int kMmaWarp = 8, kLoadWarp = 9, kSpareWarp = 10;
constexpr int kLightRegs = 56, kSoftmaxRegs = 224;         // 256 * 224 + 128 * 56 = 384 * 168 (the launch allocation)
constexpr int kNarrowRows = 16;
// Shared memory: two Q buffers (and two P buffers), then the ring.
template <bool kNarrow> struct Cfg {
    static constexpr int kSlots = kNarrow ? 6 : 5;
    static constexpr uint32_t kHalfQ = kNarrow ? kNarrowRows * 128u : kHalfTileBytes, kQBytes = 2 * kHalfQ;   // 64 channels of the rows; both halves
    static constexpr uint32_t kRing = kNarrow ? 6 * kQBytes : 2 * kQBytes;   // two P buffers of two parts, each as large as Q's
    static constexpr uint32_t kTmemCols = kNarrow ? 64 : 512, kCols = kNarrow ? kNarrowRows : 128, kColO = 2 * kCols;
};
constexpr float kRescaleThreshold = 8.0f;                  // log2 units

struct Segment {
    int32_t tiles;                                         // 0: no more segments
    int32_t key0;                                          // position of the first tile's first key
    int32_t kv, pos0, rows;
    int32_t tile0;                                         // the CTA's count of tiles before this segment
    int64_t out;                                           // whole unit: (first token row * Hq + first head); else partial slot * few_rows
    int32_t whole;
};

struct Shared {
    uint64_t q_full[2], q_empty[2];                        // per group: descriptor and Q of its next segment
    uint64_t kv_full[6], kv_empty[6];
    uint64_t s_full[2][2], p_ready[2][2];                  // [group][TMEM buffer]
    uint64_t pv_done[2], o_free[2];                        // [group]
    uint64_t drained;
    Segment seg[2];
    float4 red[2][2][kNarrowRows];                         // [group][every other exchange][row], one component per warp
    int32_t count;                                         // tiles of this CTA's piece of the line
    uint32_t tmem_base;
    volatile int abort_flag;
};
template <bool kNarrow> constexpr size_t smem_bytes() { return Cfg<kNarrow>::kRing + Cfg<kNarrow>::kSlots * kTileBytes + 1024 /*alignment slack*/ + sizeof(Shared); }

__device__ __forceinline__ bool wait_bar(uint64_t *bar, uint32_t parity, Shared *sh, const Params &p)
{
    return mbar_wait_bounded(smem_u32(bar), parity, &sh->abort_flag, p.status, p.wait_cycles, (int)PEC_ERR_TIMEOUT);
}
__device__ __forceinline__ bool wait_all(uint64_t *bar, uint32_t parity, Shared *sh, const Params &p)   // warp-uniform
{
    return __all_sync(0xffffffffu, wait_bar(bar, parity, sh, p));
}

// Eight K steps of D (+)= A B as one statement: descriptors are the first one's plus constants (in 16-byte units).  A: a tile of the
// ring, kA = 0 K-major (K: 16 channels a step, the second 64 in the groups' second halves), 1 M-major (V: two groups a step).  B: K-major, 16
// rows, its second 64 columns 2048 bytes on.
template <int kA>
__device__ __forceinline__ void mma_narrow(uint32_t d, uint64_t a0, uint64_t b0, uint32_t idesc, uint32_t accumulate)
{
    constexpr int h = kGroupHalf >> 4, s = 2 * kGroupBytes >> 4;
    constexpr int a1 = kA ? s : 2, a2 = kA ? 2 * s : 4, a3 = kA ? 3 * s : 6, a4 = kA ? 4 * s : h, a5 = kA ? 5 * s : h + 2;
    constexpr int a6 = kA ? 6 * s : h + 4, a7 = kA ? 7 * s : h + 6;
    asm volatile(
        "{\n\t.reg .pred p0, pt;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.u32 p0, %4, 0;\n\t"
        "setp.eq.u32 pt, %0, %0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p0;\n\t"
        "add.s64 da, %1, %5;\n\tadd.s64 db, %2, 2;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, pt;\n\t"
        "add.s64 da, %1, %6;\n\tadd.s64 db, %2, 4;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, pt;\n\t"
        "add.s64 da, %1, %7;\n\tadd.s64 db, %2, 6;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, pt;\n\t"
        "add.s64 da, %1, %8;\n\tadd.s64 db, %2, 128;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, pt;\n\t"
        "add.s64 da, %1, %9;\n\tadd.s64 db, %2, 130;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, pt;\n\t"
        "add.s64 da, %1, %10;\n\tadd.s64 db, %2, 132;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, pt;\n\t"
        "add.s64 da, %1, %11;\n\tadd.s64 db, %2, 134;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, pt;\n\t}"
        ::"r"(d), "l"(a0), "l"(b0), "r"(idesc), "r"(accumulate), "n"(a1), "n"(a2), "n"(a3), "n"(a4), "n"(a5), "n"(a6), "n"(a7) : "memory");
}
// 16 consecutive columns of this warp's 32 TMEM lanes, and back.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};\n\t"
        "tcgen05.wait::st.sync.aligned;"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
// Barrier of the 128 threads of a softmax group that also tells whether any of them says so.  It has no limit of its own, so the
// four warps of a group reach every one of them together: whether to go on is always decided by such a vote.
__device__ __forceinline__ bool group_any(int g, bool say)
{
    uint32_t any;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %2, 0;\n\t"
        "barrier.cta.red.or.pred q, %1, 128, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(any) : "r"(1 + g), "r"((uint32_t)say) : "memory");
    return any != 0;
}
// Lane c (and c + 16) gets the result over the warp's lanes of value c: each step halves the values a lane is in charge of.
template <class F>
__device__ __forceinline__ float warp_reduce16(const float (&x)[kNarrowRows], int lane, F f)
{
    float y[kNarrowRows];
#pragma unroll
    for (int c = 0; c < kNarrowRows; ++c) y[c] = x[c];
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) {
        const bool upper = lane & d;
#pragma unroll
        for (int i = 0; i < d; ++i) {
            const float keep = upper ? y[i + d] : y[i], send = upper ? y[i] : y[i + d];
            y[i] = f(keep, __shfl_xor_sync(0xffffffffu, send, d));
        }
    }
    return f(y[0], __shfl_xor_sync(0xffffffffu, y[0], 16));
}

template <bool kNarrow>
__global__ void __launch_bounds__(kThreads, 1)
paged_few_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                 const __grid_constant__ CUtensorMap tm_v, const Params p, const int box, const int q_tokens, const int skip_last)
{
    typedef Cfg<kNarrow> C;
    constexpr int kSlots = C::kSlots;
    constexpr uint32_t kTmemCols = C::kTmemCols, kColO = C::kColO;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t sQ = (raw + 1023u) & ~1023u, sRing = sQ + C::kRing;
    Shared *sh = reinterpret_cast<Shared *>(smem_raw + (sQ - raw) + C::kRing + kSlots * kTileBytes);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    // The loader warp sets up the barriers and works out this CTA's piece of the line; it does not wait for the tensor memory and
    // goes on to the first loads while the others gather.
    Walk walk;
    int32_t first = 0, n_tiles = 0;
    if (warp == kLoadWarp) {
        if (lane == 0) {
            griddep_launch_dependents();                   // the combining kernel may be launched; it waits for this one's end
            sh->abort_flag = 0;
            for (int g = 0; g < 2; ++g) {
                mbar_init(smem_u32(&sh->q_full[g]), 1);
                mbar_init(smem_u32(&sh->q_empty[g]), 5);   // four softmax warps, the issuer's commit
                for (int i = 0; i < 2; ++i) {
                    mbar_init(smem_u32(&sh->s_full[g][i]), 1);
                    mbar_init(smem_u32(&sh->p_ready[g][i]), 4);
                }
                mbar_init(smem_u32(&sh->pv_done[g]), 1);
                mbar_init(smem_u32(&sh->o_free[g]), 4);
            }
            for (int s = 0; s < kSlots; ++s) { mbar_init(smem_u32(&sh->kv_full[s]), 1); mbar_init(smem_u32(&sh->kv_empty[s]), 1); }
            mbar_init(smem_u32(&sh->drained), 1);
            mbar_init_fence();
        }
        const int32_t all = walk_tiles(p, walk, lane), piece = few_piece(p, all);
        first = (int32_t)blockIdx.x * piece;
        n_tiles = min(max(all - first, 0), piece);
        if (n_tiles > 0) walk_to(p, walk, first, lane);
        if (lane == 0) sh->count = n_tiles;
        __syncwarp();
        asm volatile("barrier.cta.arrive 3, %0;" ::"n"(kThreads) : "memory");
        if (n_tiles == 0) {
            griddep_wait();
            return;
        }
    } else {
        if (warp == 4) {
            tmem_alloc(smem_u32(&sh->tmem_base), kTmemCols);
            tmem_relinquish();
        } else if (tid == 0) {
            prefetch_tmap(&tm_q); prefetch_tmap(&tm_k); prefetch_tmap(&tm_v);
        }
        tc_fence_before();
        asm volatile("barrier.cta.sync 3, %0;" ::"n"(kThreads) : "memory");
        tc_fence_after();
        n_tiles = sh->count;
        if (n_tiles == 0) {
            if (warp == 4) tmem_dealloc(sh->tmem_base, kTmemCols);
            return;
        }
    }
    const int32_t count = n_tiles;
    const uint32_t tmem = warp == kLoadWarp ? 0 : sh->tmem_base;

    if (warp == kLoadWarp) {
        // ------------------------------------------------------------------ loader
        if (!kNarrow) reg_dealloc<kLightRegs>();
        const BoxLane bl = box_lane(box, lane);
        const int32_t end = first + count;
        const BoxStep step = box_step(p.c.page_size);
        BoxPlace at = box_place(p.c.page_size, walk.tile * kKeyTile, bl);      // this lane's box of the current tile, and its page
        int32_t page = box_page(p, walk.b, walk.tile * kKeyTile, walk.r.kv, bl, at);
        int segs = 0, n = 0;
        uint32_t issued = 0, q_issued = 0;                 // ring items and segments whose loads are under way
        bool ok = true;
        while (n < count && ok) {
            // a segment: descriptor and Q
            const int g = segs & 1;
            const int32_t tiles = min(walk.u0 + walk.r.tiles(), end) - max(walk.u0, first);
            if (segs >= 2) ok = wait_all(&sh->q_empty[g], ((segs >> 1) - 1) & 1, sh, p);
            if (!ok) break;
            if (lane == 0) {
                Segment s;
                s.tiles = tiles;
                s.key0 = walk.tile * kKeyTile;
                s.kv = walk.r.kv; s.pos0 = walk.r.pos0(); s.rows = walk.r.n * p.g;
                s.tile0 = n;
                s.whole = tiles == walk.r.tiles();
                s.out = s.whole ? (int64_t)walk.r.start * p.Hq + (int64_t)walk.kvh * p.g
                                : (2 * (int64_t)blockIdx.x + (walk.u0 > first ? 1 : 0)) * p.few_rows;
                sh->seg[g] = s;
                const uint32_t bar = smem_u32(&sh->q_full[g]), dst = sQ + (uint32_t)g * C::kQBytes;
                mbar_arrive_expect_tx(bar, (uint32_t)(q_tokens * p.g) * 256u);
                tma_load_4d(dst, &tm_q, bar, 0, 0, walk.kvh, walk.r.start);
                tma_load_4d(dst + C::kHalfQ, &tm_q, bar, 64, 0, walk.kvh, walk.r.start);
            }
            __syncwarp();
            ++segs; ++q_issued;
            // its tiles; the pages of the tile after the current one are looked up ahead
            const int32_t b = walk.b, kv = walk.r.kv, kvh = walk.kvh;
            int32_t k0 = walk.tile * kKeyTile;
            if (n + tiles < count) walk_next(p, walk, lane);
            for (int j = 0; j < tiles && ok; ++j, ++n, k0 += kKeyTile) {
                int32_t page_next = 0;
                BoxPlace at_next = box_next(at, step);
                if (j + 1 < tiles) {
                    page_next = box_page(p, b, k0 + kKeyTile, kv, bl, at_next);
                } else if (n + 1 < count) {                // the next unit, from its first tile
                    at_next = box_place(p.c.page_size, 0, bl);
                    page_next = box_page(p, walk.b, 0, walk.r.kv, bl, at_next);
                }
                const uint32_t bytes = tile_bytes(k0, kv, box);
#pragma unroll
                for (int which = 0; which < 2; ++which) {  // K, V
                    const int item = 2 * n + which, slot = item % kSlots, fill = item / kSlots;
                    if (skip_last && count > 1 && item == 2 * count - 1) { ok = false; break; }   // test hook: the wait for it runs out
                    if (fill > 0) ok = wait_all(&sh->kv_empty[slot], (fill - 1) & 1, sh, p);
                    if (!ok) break;
                    const uint32_t bar = smem_u32(&sh->kv_full[slot]);
                    if (lane == 0) mbar_arrive_expect_tx(bar, bytes);
                    __syncwarp();
                    if (bl.used && k0 + bl.first < kv)
                        load_box(sRing + (uint32_t)slot * kTileBytes, which ? (const void *)&tm_v : (const void *)&tm_k, bar, bl, which ? p.fv : p.fk,
                                 kvh, at.row, page);
                    ++issued;
                }
                page = page_next;
                at = at_next;
            }
        }
        // No more segments for either group.
        for (int e = 0; e < 2 && ok; ++e, ++segs) {
            const int g = segs & 1;
            if (segs >= 2) ok = wait_all(&sh->q_empty[g], ((segs >> 1) - 1) & 1, sh, p);
            if (ok && lane == 0) { sh->seg[g].tiles = 0; mbar_arrive(smem_u32(&sh->q_full[g])); }
        }
        if (!ok && lane == 0) {
            // Given up: the copies under way must land before the CTA may leave.
            auto landed = [&](uint64_t *bar, uint32_t parity) { wait_quietly(bar, parity, p); };
            for (uint32_t i = issued > kSlots ? issued - kSlots : 0; i < issued; ++i) landed(&sh->kv_full[i % kSlots], (i / kSlots) & 1);
            for (uint32_t i = q_issued > 2 ? q_issued - 2 : 0; i < q_issued; ++i) landed(&sh->q_full[i & 1], (i >> 1) & 1);
        }
        __syncwarp();
    } else if (warp == kMmaWarp) {
        // ------------------------------------------------------------------ MMA issuer (the whole warp walks, one lane issues)
        if (!kNarrow) reg_dealloc<kLightRegs>();
        const bool leader = elect_one();
        constexpr uint32_t narrow_qk = idesc_bf16_f32(128, kNarrowRows, 0, 0), narrow_pv = idesc_bf16_f32(kHeadDim, kNarrowRows, 1, 0);
        constexpr uint32_t idesc_qk = idesc_bf16_f32(128, 128, 0, 0), idesc_pv = idesc_bf16_f32(128, kHeadDim, 0, 1);
        const uint64_t k_ring = smem_desc_sw128(sRing, 16, kGroupBytes), v_ring = smem_desc_sw128(sRing, kGroupHalf, kGroupBytes);
        uint32_t p_phase = 0;                              // bit 2 g + buffer: parity of the next p_ready
        auto kv_wait = [&](int item) { return wait_all(&sh->kv_full[item % kSlots], (item / kSlots) & 1, sh, p); };
        auto kv_release = [&](int item) { if (leader) tc_commit(smem_u32(&sh->kv_empty[item % kSlots])); };
        // S(n) of a segment of group g; `last`: the segment's Q is not needed after it
        auto issue_qk = [&](int n, int g, bool last) {
            if (!kv_wait(2 * n)) return false;
            if (leader) {
                const uint64_t k0 = k_ring + (uint32_t)(((2 * n) % kSlots) * (kTileBytes >> 4));
                if constexpr (kNarrow) {
                    mma_narrow<0>(tmem + (uint32_t)(n & 1) * C::kCols, k0, smem_desc_sw128(sQ + (uint32_t)g * C::kQBytes, 16, 1024), narrow_qk, 0u);
                    tc_commit(smem_u32(&sh->s_full[g][n & 1]));
                } else {
                    uint64_t a[8];
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)
                        a[ks] = smem_desc_sw128(sQ + (uint32_t)g * kTileBytes + (uint32_t)(ks >> 2) * kHalfTileBytes + (uint32_t)(ks & 3) * 32u, 16, 1024);
                    mma_ss_k128_commit<(kGroupHalf >> 4)>(tmem + (uint32_t)(n & 1) * C::kCols, a, k0, idesc_qk, smem_u32(&sh->s_full[g][n & 1]));
                }
                if (last) tc_commit(smem_u32(&sh->q_empty[g]));
            }
            kv_release(2 * n);
            return true;
        };
        int segs = 0;
        bool ok = wait_all(&sh->q_full[0], 0, sh, p);
        Segment cur = sh->seg[0];
        if (ok) ok = issue_qk(0, 0, cur.tiles == 1);
        int n = 0;
        while (ok) {
            const int g = segs & 1, k = segs >> 1;         // k: the group's count of segments before this one
            Segment next;
            next.tiles = 0;
            for (int j = 0; j < cur.tiles && ok; ++j, ++n) {
                if (j + 1 < cur.tiles) {
                    ok = issue_qk(n + 1, g, j + 2 == cur.tiles);
                } else if (n + 1 < count) {
                    ok = wait_all(&sh->q_full[g ^ 1], ((segs + 1) >> 1) & 1, sh, p);
                    if (!ok) break;
                    next = sh->seg[g ^ 1];
                    ok = issue_qk(n + 1, g ^ 1, next.tiles == 1);
                }
                if (!ok) break;
                ok = kv_wait(2 * n + 1);
                if (!ok) break;
                const uint32_t slot = (uint32_t)((2 * n + 1) % kSlots);
                const int32_t valid = cur.kv - cur.key0 - j * kKeyTile;
                if (valid < kKeyTile) clear_tail(sRing + slot * kTileBytes, valid, lane);
                if (j == 0 && k > 0) ok = wait_all(&sh->o_free[g], (k - 1) & 1, sh, p);
                const int bit = 2 * g + (n & 1);
                if (ok) ok = wait_all(&sh->p_ready[g][n & 1], (p_phase >> bit) & 1, sh, p);
                if (!ok) break;
                p_phase ^= 1u << bit;
                tc_fence_after();
                if (leader) {
                    const uint64_t v0 = v_ring + slot * (kTileBytes >> 4);
                    const uint32_t tO = tmem + kColO + (uint32_t)g * C::kCols, tP = tmem + (uint32_t)(n & 1) * C::kCols;
                    if constexpr (kNarrow) {
                        const uint64_t p0 = smem_desc_sw128(sQ + (uint32_t)(2 + 2 * (n & 1)) * C::kQBytes, 16, 1024);
                        mma_narrow<1>(tO, v0, p0, narrow_pv, j > 0 ? 1u : 0u);
                        mma_narrow<1>(tO, v0, p0 + (C::kQBytes >> 4), narrow_pv, 1u);
                    } else {
                        mma_pv_k64(tO, tP, v0, idesc_pv, j > 0 ? 1u : 0u);
                        mma_pv_k64(tO, tP + 32, v0 + (8 * kGroupBytes >> 4), idesc_pv, 1u);
                    }
                    tc_commit(smem_u32(&sh->pv_done[g]));
                }
                kv_release(2 * n + 1);
            }
            if (next.tiles == 0) break;
            cur = next;
            ++segs;
        }
        if (!ok) drain_products(&sh->drained, leader, p);
        __syncwarp();
    } else if (warp > kLoadWarp) {
        if (!kNarrow) reg_dealloc<kLightRegs>();
        // An earlier CTA's wait has run out: the launch is lost, every wait of this CTA gives up at its next try.
        if (warp == kSpareWarp && lane == 0 && *reinterpret_cast<volatile int32_t *>(p.status) == PEC_ERR_TIMEOUT) sh->abort_flag = 1;
    } else if constexpr (kNarrow) {
        // ------------------------------------------------------------------ softmax and epilogue, narrow form
        const int g = warp >> 2, quarter = warp & 3, key = quarter * 32 + lane;      // and channel `key` of the accumulator
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const uint32_t tO = tmem + lane_base + kColO + (uint32_t)g * C::kCols;
        // P^T as the K-major operand: row c at 128 c, 64 keys a row (the second 64 in a second half), 16-byte chunks XOR-swizzled by row.
        const uint32_t p_half = (uint32_t)(key >> 6) * C::kHalfQ + (uint32_t)(key & 7) * 2u, p_chunk = (uint32_t)(key & 63) >> 3;
        uint32_t s_phase = 0, pv = 0;
        // Exchanges between the group's warps take turns in two buffers: whoever writes one has passed the vote of the exchange
        // after its last use, which its readers reached after reading.
        int turn = 0;
        for (int k = 0;; ++k) {
            bool ok = wait_all(&sh->q_full[g], k & 1, sh, p);
            if (group_any(g, !ok)) break;
            const Segment s = sh->seg[g];
            __syncwarp();
            if (s.tiles == 0) break;
            if (lane == 0) mbar_arrive(smem_u32(&sh->q_empty[g]));
            const bool wide = s.rows > 8;                  // columns 8 - 15 are used
            const int32_t see_all = (p.causal && s.pos0 + 1 < s.kv) ? s.pos0 + 1 : s.kv;           // keys below it are visible to every row
            float m[kNarrowRows], l[kNarrowRows];          // per row: reference maximum (log2 units, the same in all threads), this thread's sum
#pragma unroll
            for (int c = 0; c < kNarrowRows; ++c) { m[c] = -INFINITY; l[c] = 0.f; }
            float m_row = -INFINITY;                       // m of row lane % 16
            int32_t k0 = s.key0;
            bool stop = false;
            for (int j = 0; j < s.tiles; ++j, k0 += kKeyTile) {
                const int buf = (s.tile0 + j) & 1;
                ok = wait_all(&sh->s_full[g][buf], (s_phase >> buf) & 1, sh, p);
                s_phase ^= 1u << buf;
                tc_fence_after();
                uint32_t r[kNarrowRows];
                tmem_ld16(tmem + lane_base + (uint32_t)buf * C::kCols, r);
                tc_fence_before();
                float x[kNarrowRows];
#pragma unroll
                for (int c = 0; c < kNarrowRows; ++c) x[c] = __uint_as_float(r[c]);
                if (k0 + kKeyTile > see_all) {             // by choice, not by arithmetic: a masked score may be anything
#pragma unroll
                    for (int c = 0; c < kNarrowRows; ++c) {
                        const int32_t see = p.causal ? min(s.kv, s.pos0 + c / p.g + 1) : s.kv;
                        x[c] = k0 + key < see ? x[c] : -INFINITY;
                    }
                }
                bool grow = false;
#pragma unroll
                for (int c = 0; c < kNarrowRows; ++c) {
                    if (c < s.rows) grow = grow || x[c] * p.scale_log2 > m[c] + kRescaleThreshold;
                }
                // The reference maxima move only when one is outgrown by 2^8 (and from -inf); O then waits for its product in flight.
                if (j == 0 || group_any(g, grow || !ok)) {
                    if (j > 0 && ok) ok = wait_all(&sh->pv_done[g], (pv + j - 1) & 1, sh, p);
                    stop = group_any(g, !ok);
                    if (stop) break;
                    const float most = warp_reduce16(x, lane, [](float a, float b) { return fmaxf(a, b); });
                    float4 *red = sh->red[g][turn ^= 1];
                    if (lane < kNarrowRows) reinterpret_cast<float *>(red + lane)[quarter] = most;
                    group_any(g, false);
                    // Lane c works out row c's new reference; the others get it by shuffle.
                    const float4 t = red[lane & (kNarrowRows - 1)];
                    const float top = fmaxf(fmaxf(t.x, t.y), fmaxf(t.z, t.w)) * p.scale_log2;
                    const bool move = (lane & (kNarrowRows - 1)) < s.rows && top > m_row + kRescaleThreshold;
                    const float a_row = move ? ex2(m_row - top) : 1.f;     // 0 when the row had no key so far
                    if (move) m_row = top;
                    float alpha[kNarrowRows];
#pragma unroll
                    for (int c = 0; c < kNarrowRows; ++c) {
                        if (c < 8 || wide) {
                            m[c] = __shfl_sync(0xffffffffu, m_row, c);
                            alpha[c] = __shfl_sync(0xffffffffu, a_row, c);
                            l[c] *= alpha[c];
                        } else {
                            alpha[c] = 1.f;
                        }
                    }
                    if (j > 0) {
                        tc_fence_after();
                        uint32_t o[kNarrowRows];
                        tmem_ld16(tO, o);
#pragma unroll
                        for (int c = 0; c < kNarrowRows; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * alpha[c]);
                        tmem_st16(tO, o);
                        tc_fence_before();
                    }
                } else if (j > 0) {
                    // Waited for in every tile (see the wide form); what it says is voted on with the next tile.
                    if (!wait_all(&sh->pv_done[g], (pv + j - 1) & 1, sh, p)) sh->abort_flag = 1;
                }
                // p = 2^(s scale - m) as the sum of two bf16 operands (16 bits of it; the second product costs next to nothing at
                // 16 columns); the row's sum takes p itself.  S(n) is complete, and with it PV(n - 2), which read this P buffer.
                const uint32_t dst = sQ + (uint32_t)(2 + 2 * buf) * C::kQBytes + p_half;
#pragma unroll
                for (int c = 0; c < kNarrowRows; ++c) {
                    if (c < 8 || wide) {
                        const float e = ex2(fmaf(x[c], p.scale_log2, m[c] == -INFINITY ? 0.f : -m[c]));
                        l[c] += e;
                        const __nv_bfloat16 hi = __float2bfloat16_rn(e), lo = __float2bfloat16_rn(e - __bfloat162float(hi));
                        const uint32_t to = dst + (uint32_t)c * 128u + ((p_chunk ^ (uint32_t)(c & 7)) << 4);
                        asm volatile("st.shared.b16 [%0], %1;" ::"r"(to), "h"(*reinterpret_cast<const unsigned short *>(&hi)) : "memory");
                        asm volatile("st.shared.b16 [%0], %1;" ::"r"(to + C::kQBytes), "h"(*reinterpret_cast<const unsigned short *>(&lo)) : "memory");
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->p_ready[g][buf]));
            }
            if (stop) break;
            pv += s.tiles;
            ok = wait_all(&sh->pv_done[g], (pv - 1) & 1, sh, p);
            const float part = warp_reduce16(l, lane, [](float a, float b) { return a + b; });
            float4 *red = sh->red[g][turn ^= 1];
            if (lane < kNarrowRows) reinterpret_cast<float *>(red + lane)[quarter] = part;
            if (group_any(g, !ok)) break;
            tc_fence_after();
            uint32_t o[kNarrowRows];
            tmem_ld16(tO, o);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->o_free[g]));
            // Lane c works out row c's factor, place and LSE.
            const int row = lane & (kNarrowRows - 1);
            const float4 t = red[row];
            const float sum = (t.x + t.y) + (t.z + t.w);
            const int64_t at = s.whole ? s.out + (int64_t)(row / p.g) * p.Hq + row % p.g : s.out + row;
            const float f_row = sum == 0.f ? 0.f : 1.f / sum;
            if (quarter == 0 && lane < s.rows && lane < kNarrowRows)
                (s.whole ? p.lse : p.few_lse)[at] = sum == 0.f ? -INFINITY : m_row * 0.6931471805599453f + logf(sum);
#pragma unroll
            for (int c = 0; c < kNarrowRows; ++c) {
                if (c >= s.rows) break;
                const float f = __shfl_sync(0xffffffffu, f_row, c);
                const int64_t to = __shfl_sync(0xffffffffu, at, c) * kHeadDim + key;
                const float y = f == 0.f ? 0.f : __uint_as_float(o[c]) * f;
                if (s.whole && p.o_is_bf16) static_cast<__nv_bfloat16 *>(p.o)[to] = __float2bfloat16_rn(y);
                else (s.whole ? static_cast<float *>(p.o) : p.few_o)[to] = y;
            }
        }
    } else {
        // ------------------------------------------------------------------ softmax and epilogue, wide form
        reg_alloc<kSoftmaxRegs>();
        const int g = warp >> 2, quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const uint32_t tO = tmem + lane_base + kColO + (uint32_t)g * C::kCols;
        const int32_t tok = row / p.g, head = row - tok * p.g;
        uint32_t s_phase = 0;                              // bit: parity of the buffer's next s_full
        uint32_t pv = 0;                                   // the group's PV products before this segment
        for (int k = 0;; ++k) {
            bool ok = wait_all(&sh->q_full[g], k & 1, sh, p);
            if (!ok) break;
            const Segment s = sh->seg[g];
            __syncwarp();
            if (s.tiles == 0) break;
            if (lane == 0) mbar_arrive(smem_u32(&sh->q_empty[g]));
            const bool works = quarter * 32 < s.rows;
            const int32_t see_all = (p.causal && s.pos0 + 1 < s.kv) ? s.pos0 + 1 : s.kv;           // keys below it are visible to every row
            const int32_t see = (p.causal && s.pos0 + tok + 1 < s.kv) ? s.pos0 + tok + 1 : s.kv;   // ... to this row
            float m_ref = -INFINITY, l_run = 0.f;          // m_ref in log2 units of the scaled scores
            int32_t k0 = s.key0;
            for (int j = 0; j < s.tiles; ++j, k0 += kKeyTile) {
                const int buf = (s.tile0 + j) & 1;
                const uint32_t tS = tmem + lane_base + (uint32_t)buf * C::kCols;
                ok = wait_all(&sh->s_full[g][buf], (s_phase >> buf) & 1, sh, p);
                if (!ok) break;
                s_phase ^= 1u << buf;
                if (works) {
                    tc_fence_after();
                    uint32_t r[kKeyTile];
                    tmem_ld128(tS, r);
                    if (k0 + kKeyTile > see_all) {         // by choice, not by arithmetic: a masked score may be anything
                        int n_vis = see - k0;
                        n_vis = n_vis < 0 ? 0 : (n_vis > kKeyTile ? kKeyTile : n_vis);
#pragma unroll
                        for (int c = 0; c < kKeyTile; ++c) r[c] = (c < n_vis) ? r[c] : 0xff800000u;
                    }
                    float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
#pragma unroll
                    for (int c = 0; c < kKeyTile; c += 8) {
                        mx0 = fmax3(mx0, __uint_as_float(r[c + 0]), __uint_as_float(r[c + 1]));
                        mx1 = fmax3(mx1, __uint_as_float(r[c + 2]), __uint_as_float(r[c + 3]));
                        mx2 = fmax3(mx2, __uint_as_float(r[c + 4]), __uint_as_float(r[c + 5]));
                        mx3 = fmax3(mx3, __uint_as_float(r[c + 6]), __uint_as_float(r[c + 7]));
                    }
                    const float m_new = fmax3(mx0, mx1, fmaxf(mx2, mx3)) * p.scale_log2;
                    // The reference maximum moves only when outgrown by 2^8; O then waits for its product in flight.
                    float alpha = 1.f;
                    const bool grow = m_new > m_ref + kRescaleThreshold;
                    if (grow) {
                        alpha = ex2(m_ref - m_new);        // 0 when the row had no key so far
                        m_ref = m_new;
                        l_run *= alpha;
                    }
                    // PV(j - 1) is waited for in every tile: before O is rescaled where that is needed, before P(j) is handed over
                    // otherwise.  S(j) is complete, and with it PV(j - 2), issued before it, and PV(j) needs this warp's P(j),
                    // so the barrier's parity tells exactly that phase; a wait left out would make the next one ambiguous.
                    bool pv_waited = j == 0;
                    if (j > 0 && __any_sync(0xffffffffu, grow)) {
                        ok = wait_all(&sh->pv_done[g], (pv + j - 1) & 1, sh, p);
                        if (!ok) break;
                        pv_waited = true;
                        tc_fence_after();
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t o[32];
                            tmem_ld32(tO + c * 32, o);
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                            tmem_st32(tO + c * 32, o);
                        }
                    }
                    const float neg_m = (m_ref == -INFINITY) ? 0.f : -m_ref;
                    const float2 sc2 = make_float2(p.scale_log2, p.scale_log2), nm2 = make_float2(neg_m, neg_m);
                    float2 sum[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[i] = make_float2(0.f, 0.f);
                    // p = 2^(s scale - m), rounded to bf16 as the product's operand (the tensor cores take no wider one beside a
                    // bf16 V); the row's sum takes p before it is rounded.  A second part, as the narrow form has, would be a third
                    // 128-row product a tile, in the form that draws the power limit already.
#pragma unroll
                    for (int i = 0; i < kKeyTile / 2; ++i) {
                        const float2 x = __ffma2_rn(make_float2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])), sc2, nm2);
                        const float2 e = make_float2(ex2(x.x), ex2(x.y));
                        sum[i & 3] = __fadd2_rn(sum[i & 3], e);
                        r[i] = pack_bf16(e.x, e.y);
                    }
                    const float2 s01 = __fadd2_rn(__fadd2_rn(sum[0], sum[1]), __fadd2_rn(sum[2], sum[3]));
                    l_run += s01.x + s01.y;
                    if (!pv_waited) {
                        ok = wait_all(&sh->pv_done[g], (pv + j - 1) & 1, sh, p);
                        if (!ok) break;
                    }
                    tmem_st32(tS, r);
                    tmem_st32(tS + 32, r + 32);
                    tmem_st_wait();
                    tc_fence_before();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->p_ready[g][buf]));
            }
            if (!ok) break;
            pv += s.tiles;
            if (works) {
                ok = wait_all(&sh->pv_done[g], (pv - 1) & 1, sh, p);
                if (!ok) break;
                tc_fence_after();
                const bool valid = row < s.rows, empty = l_run == 0.f;
                const float inv = empty ? 0.f : 1.f / l_run;
                const int64_t at = s.whole ? s.out + (int64_t)tok * p.Hq + head : s.out + row;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t r[32];
                    tmem_ld32(tO + c * 32, r);
                    if (!valid) continue;
                    float f[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) f[i] = empty ? 0.f : __uint_as_float(r[i]) * inv;
                    if (s.whole && p.o_is_bf16) {
                        __nv_bfloat16 *o = static_cast<__nv_bfloat16 *>(p.o) + at * kHeadDim + c * 32;
#pragma unroll
                        for (int i = 0; i < 32; i += 8)
                            *reinterpret_cast<uint4 *>(o + i) = make_uint4(pack_bf16(f[i], f[i + 1]), pack_bf16(f[i + 2], f[i + 3]),
                                                                           pack_bf16(f[i + 4], f[i + 5]), pack_bf16(f[i + 6], f[i + 7]));
                    } else {
                        float *o = (s.whole ? static_cast<float *>(p.o) : p.few_o) + at * kHeadDim + c * 32;
#pragma unroll
                        for (int i = 0; i < 32; i += 4) *reinterpret_cast<float4 *>(o + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
                    }
                }
                if (valid) (s.whole ? p.lse : p.few_lse)[at] = empty ? -INFINITY : m_ref * 0.6931471805599453f + logf(l_run);
                tc_fence_before();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->o_free[g]));
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 4) tmem_dealloc(tmem, kTmemCols);
    // Beside the last CTAs of the kernel for many rows, which write other rows; but whoever waits for this kernel waits for that one.
    griddep_wait();
}

}  // namespace few
}  // namespace paged

int launch_paged_few(const paged::Params &p, bool after_many, cudaStream_t stream)
{
    using namespace paged;
    const int box = host_map::box_rows(p.c.page_size);
    const int tps = kFewRows / p.g, q_tokens = tps < p.max_q ? tps : p.max_q;
    CUtensorMap tm_q, tm_k, tm_v;
    if (!host_map::queries(&tm_q, p, q_tokens) || !host_map::pages(&tm_k, p, p.k_pages, p.c.k_st, p.fk, box) ||
        !host_map::pages(&tm_v, p, p.v_pages, p.c.v_st, p.fv, box)) {
        set_error("pec_paged_attn: cuTensorMapEncodeTiled failed (driver too old, or strides/addresses not encodable)");
        return PEC_ERR_CUDA;
    }
    static unsigned char ready[host::kMaxDevices] = {};
    static std::mutex ready_mutex;
    if (!host::once_per_device(ready, ready_mutex, [] {
            cudaFuncAttributes attr;
            return cudaFuncSetAttribute(few::paged_few_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)few::smem_bytes<true>()) == cudaSuccess &&
                   cudaFuncSetAttribute(few::paged_few_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)few::smem_bytes<false>()) == cudaSuccess &&
                   cudaFuncGetAttributes(&attr, few::paged_few_kernel<false>) == cudaSuccess &&
                   attr.numRegs * few::kThreads >= 256 * few::kSoftmaxRegs + 128 * few::kLightRegs; })) {
        (void)cudaGetLastError();
        set_error("pec_paged_attn: kernel set-up failed (shared-memory limit, or the register allocation does not cover the warp-role split)");
        return PEC_ERR_CUDA;
    }
    // The narrow form where no request can have more than 16 rows (p.few_rows is the most any can have).
    const dim3 grid((unsigned)p.few_ctas);
    const int skip = test_skip_last_load();
    cudaError_t err =
        p.few_rows <= few::kNarrowRows
            ? launch_dependent(few::paged_few_kernel<true>, grid, few::kThreads, few::smem_bytes<true>(), stream, after_many, tm_q, tm_k, tm_v, p, box, q_tokens, skip)
            : launch_dependent(few::paged_few_kernel<false>, grid, few::kThreads, few::smem_bytes<false>(), stream, after_many, tm_q, tm_k, tm_v, p, box, q_tokens, skip);
    if (err == cudaSuccess) err = cudaGetLastError();
    if (err != cudaSuccess) { set_error("pec_paged_attn: launch failed: %s", cudaGetErrorString(err)); return PEC_ERR_CUDA; }
    return PEC_OK;
}

}  // namespace pec
