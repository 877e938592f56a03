// Attention over a cache held in 4 bits of requests with at most 16 packed rows (decode steps) on the sm_100a tensor cores.
//
// Bound by the stream of codes from HBM: 2 * kv * Hkv * 66 bytes a request, a quarter of a bf16 cache's, so that a key tile has a
// quarter of the time that the kernel for bf16 has: no code is touched by a thread on its way.  The copy unit spreads a tile's codes
// as the tensor cores take 4-bit operands (16 codes in the first 8 of 16 bytes), and the products are of kind f8f6f4, codes (e2m1) by
// 8-bit numbers, with the scales left to the other side:
//     S^T = K_codes Q^T,  s[j][r] = S^T[j][r] * sk_j * (row factor),      a thread = a key, up to 16 rows as columns
//     O^T = V_codes^T P'^T,  P'[r][j] = p[r][j] * sv_j                    a thread = a channel
// The operands that are not codes come in parts, each the rest of the one before scaled up, in columns of their own that are added
// up in fp32:
//     Q   two parts of e4m3 of the row divided by a power of two (its largest channel in [2^7, 2^8)): 4 + 4 significant bits are a
//         bf16's eight; channels under 2^-13 of the row's largest are held to 2^-22 of it
//     P'  four parts of e5m2, to 2^-12 of itself down to 2^-24 of the largest and to 2^-36 of that below, so that a bf16 result errs by
//         its own rounding alone.  (Parts of e4m3, three for as many bits, end at 2^-21: a hundred thousand keys behind one that takes
//         most of the weight, which long prompts have, would be held to two bits.)
// Products of such numbers are exact and their sums are kept in fp32.
//
// The split of the work is that of pec_paged_few.cu: the key tiles of all (request, KV head) units on one line, an equal piece of it
// for each CTA, units that cross a cut merged by the combining kernel.  Two CTAs per SM, so that one's exchange of maxima and its
// epilogues run beside the other's.
//
// Warp roles:
//   warps 0-3  softmax and epilogue
//   warp 4     MMA issuer      warp 5  TMA loader of the codes (a ring of K and V tiles)
//   warp 6     segment descriptors and Q (two buffers)      warp 7  scales (a ring of tiles)
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include "pec_paged_tma.cuh"
#include "pec_q4.cuh"

namespace pec {
using namespace sm100;
namespace paged {
namespace few_q4 {

constexpr int kThreads = 256;
constexpr int kMmaWarp = 4, kLoadWarp = 5, kQueryWarp = 6, kScaleWarp = 7;
constexpr int kScaleSlots = 4;
constexpr int kSoftmaxRegs = 176, kLightRegs = 80;         // 128 * (176 + 80) = 256 * 128 (the launch allocation)
constexpr float kNoKey = -3.0e38f;                         // reference maximum of a row that has seen no key
constexpr uint32_t kCodeTile = 128 * 128;                  // 128 tokens, their 64 bytes spread over 128
constexpr float kGrow = 3.0f;                              // log2 units: a row's reference maximum moves when outgrown by 2^3
constexpr float kBase = 1024.0f;                           // p * sv / v_ref is at most 2^3 * 4; times 2^10 it stays below e5m2's 57344

template <int kRows> struct Cfg {
    static constexpr int kSlots = kRows == 16 ? 5 : 6;
    static constexpr int kColsS = kRows == 4 ? 16 : 2 * kRows, kColsO = 4 * kRows;      // (a product has 16 columns at least)
    static constexpr uint32_t kQBytes = kColsS * 128, kPRow = kRows == 16 ? 64 : 32, kPBytes = 128 * kPRow;
    static constexpr uint32_t kTmemCols = kRows == 16 ? 128 : 64, kColO = 2 * kColsS;
    static constexpr uint32_t kOffQ = 0, kOffP = 2 * kQBytes, kOffRing = kOffP + 2 * kPBytes;
};

struct Segment {
    int32_t tiles;                                         // 0: no more segments
    int32_t key0;                                          // position of the first tile's first key
    int32_t kv, pos0, rows;
    int64_t out;                                           // whole unit: (first token row * Hq + first head); else partial slot * few_rows
    int32_t whole;
};
struct Shared {
    uint64_t q_full[2], q_empty[2];                        // descriptor and Q of every other segment
    uint64_t kv_full[6], kv_empty[6];
    uint64_t sc_full[kScaleSlots], sc_empty[kScaleSlots];
    uint64_t s_full[2], p_ready[2];                        // [TMEM buffer]
    uint64_t pv_done, drained;
    Segment seg[2];
    float q_factor[2][16];                                 // of a row's scores: log2 units of the scaled score over that of the product
    float4 red[2][17];                                     // every other exchange: rows, the scales of V; one component per warp
    uint32_t scale[kScaleSlots][kKeyTile];                 // bf16 bits: K, V << 16
    int32_t count;
    uint32_t tmem_base;
    volatile int abort_flag;
};
template <int kRows> constexpr size_t smem_bytes()
{
    return Cfg<kRows>::kOffRing + Cfg<kRows>::kSlots * kCodeTile + 1024 /*alignment slack*/ + sizeof(Shared);
}
// An SM has 228 KB, of which each CTA takes 1 KB for itself.
static_assert(smem_bytes<4>() <= 113 * 1024 && smem_bytes<8>() <= 113 * 1024 && smem_bytes<16>() <= 113 * 1024, "two CTAs per SM");

__device__ __forceinline__ bool wait_all(uint64_t *bar, uint32_t parity, Shared *sh, const Params &p)   // warp-uniform
{
    return __all_sync(0xffffffffu, mbar_wait_bounded(smem_u32(bar), parity, &sh->abort_flag, p.status, p.wait_cycles, (int)PEC_ERR_TIMEOUT));
}

// Shared-memory descriptor of an N-major operand whose rows (one per K index) are kRow bytes, swizzled in atoms of eight rows.
template <uint32_t kRow>
__device__ __forceinline__ uint64_t desc_rows(uint32_t saddr)
{
    constexpr uint64_t layout = kRow == 32 ? 6 : 4;        // 32-byte, 64-byte swizzle
    return (uint64_t)((saddr >> 4) & 0x3fffu) | (uint64_t)1 << 16 | (uint64_t)((8 * kRow) >> 4) << 32 | (uint64_t)1 << 46 | layout << 61;
}

// Four K steps of 32; descriptors advance by kA and kB 16-byte units.
template <int kA, int kB>
__device__ __forceinline__ void mma4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p0, pt;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.u32 p0, %4, 0;\n\t"
        "setp.eq.u32 pt, %0, %0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p0;\n\t"
        "add.s64 da, %1, %5;\n\tadd.s64 db, %2, %6;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %3, pt;\n\t"
        "add.s64 da, da, %5;\n\tadd.s64 db, db, %6;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %3, pt;\n\t"
        "add.s64 da, da, %5;\n\tadd.s64 db, db, %6;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %3, pt;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "n"(kA), "n"(kB) : "memory");
}

// Two numbers as e4m3, the first in the low byte.
__device__ __forceinline__ uint32_t to_e4m3(float2 x)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(x.y), "f"(x.x));
    return r;
}
// The part of x that e4m3 takes (returned), and 16 times the rest.
__device__ __forceinline__ uint32_t take_e4m3(float2 &x)
{
    const uint32_t r = to_e4m3(x);
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)r));
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
    x = __fmul2_rn(__fadd2_rn(x, make_float2(-f.x, -f.y)), make_float2(16.f, 16.f));
    return r;
}
// Four numbers, as fp16, to four parts of e5m2 each (a word of four bytes a part).  e5m2 is the upper byte of fp16: a part is what is left
// cut to its first three bits, and the eleven bits of an fp16 are 3 + 3 + 3 + 2.
__device__ __forceinline__ void split_e5m2(float2 lo, float2 hi, uint32_t (&part)[4])
{
    __half2 a = __float22half2_rn(lo), b = __float22half2_rn(hi);
    const __half2 eight = __half2half2(__ushort_as_half(0x4800));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t ua = *reinterpret_cast<const uint32_t *>(&a), ub = *reinterpret_cast<const uint32_t *>(&b);
        part[i] = __byte_perm(ua, ub, 0x7531);
        if (i == 3) break;
        const uint32_t ta = ua & 0xff00ff00u, tb = ub & 0xff00ff00u;
        a = __hmul2(__hsub2(a, *reinterpret_cast<const __half2 *>(&ta)), eight);
        b = __hmul2(__hsub2(b, *reinterpret_cast<const __half2 *>(&tb)), eight);
    }
}

template <int kRows>
__global__ void __launch_bounds__(kThreads, kFewCtasQ4)
paged_few_q4_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const Params p, const int box,
                    const int scales_by_four, const int skip_last)
{
    typedef Cfg<kRows> C;
    constexpr int kSlots = C::kSlots;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t *const smem = smem_raw + (base - raw);
    const uint32_t sQ = base + C::kOffQ, sP = base + C::kOffP, sRing = base + C::kOffRing;
    Shared *sh = reinterpret_cast<Shared *>(smem + C::kOffRing + kSlots * kCodeTile);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    // The loader, query and scale warps each find this CTA's piece of the line, and go on to their first loads while the others gather.
    Walk walk;
    int32_t first = 0, n_tiles = 0;
    if (warp >= kLoadWarp) {
        if (warp == kLoadWarp && lane == 0) {
            griddep_launch_dependents();                   // the combining kernel may be launched; it waits for this one's end
            sh->abort_flag = 0;
            for (int g = 0; g < 2; ++g) {
                mbar_init(smem_u32(&sh->q_full[g]), 1);
                mbar_init(smem_u32(&sh->q_empty[g]), 5);   // four softmax warps, the issuer's commit
                mbar_init(smem_u32(&sh->s_full[g]), 1);
                mbar_init(smem_u32(&sh->p_ready[g]), 4);
            }
            for (int s = 0; s < kSlots; ++s) { mbar_init(smem_u32(&sh->kv_full[s]), 1); mbar_init(smem_u32(&sh->kv_empty[s]), 1); }
            for (int s = 0; s < kScaleSlots; ++s) { mbar_init(smem_u32(&sh->sc_full[s]), 1); mbar_init(smem_u32(&sh->sc_empty[s]), 4); }
            mbar_init(smem_u32(&sh->pv_done), 1);
            mbar_init(smem_u32(&sh->drained), 1);
            mbar_init_fence();
        }
        const int32_t all = walk_tiles(p, walk, lane), piece = few_piece(p, all);
        first = (int32_t)blockIdx.x * piece;
        n_tiles = min(max(all - first, 0), piece);
        if (n_tiles > 0) walk_to(p, walk, first, lane);
        if (warp == kLoadWarp && lane == 0) sh->count = n_tiles;
    } else if (warp == kMmaWarp) {
        tmem_alloc(smem_u32(&sh->tmem_base), C::kTmemCols);
        tmem_relinquish();
        if (lane == 0) { prefetch_tmap(&tm_k); prefetch_tmap(&tm_v); }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const int32_t count = sh->count;
    const uint32_t tmem = sh->tmem_base;

    if (count == 0) {
    } else if (warp == kLoadWarp) {
        // ------------------------------------------------------------------ loader of the codes
        reg_dealloc<kLightRegs>();
        const BoxLane bl = {lane * box, (uint32_t)(lane * box) * 128u, lane * box < kKeyTile};
        const int32_t end = first + count;
        const BoxStep step = box_step(p.c.page_size);
        BoxPlace at = box_place(p.c.page_size, walk.tile * kKeyTile, bl);      // this lane's box of the current tile, and its page
        int32_t page = box_page(p, walk.b, walk.tile * kKeyTile, walk.r.kv, bl, at);
        int n = 0;
        uint32_t issued = 0;
        bool ok = true;
        while (n < count && ok) {
            const int32_t tiles = min(walk.u0 + walk.r.tiles(), end) - max(walk.u0, first);
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
                const uint32_t bytes = tile_bytes(k0, kv, box) / 4;            // 64 bytes a token
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
                        tma_load_4d(sRing + (uint32_t)slot * kCodeTile + bl.offset, which ? (const void *)&tm_v : (const void *)&tm_k, bar, 0, at.row, kvh, page);
                    ++issued;
                }
                page = page_next;
                at = at_next;
            }
        }
        if (!ok && lane == 0) {
            // Given up: the copies under way must land before the CTA may leave.
            for (uint32_t i = issued > kSlots ? issued - kSlots : 0; i < issued; ++i) wait_quietly(&sh->kv_full[i % kSlots], (i / kSlots) & 1, p);
        }
        __syncwarp();
    } else if (warp == kQueryWarp) {
        // ------------------------------------------------------------------ segments and their queries
        reg_dealloc<kLightRegs>();
        // An earlier CTA's wait has run out: the launch is lost, every wait of this CTA gives up at its next try.
        if (lane == 0 && *reinterpret_cast<volatile int32_t *>(p.status) == PEC_ERR_TIMEOUT) sh->abort_flag = 1;
        const int32_t end = first + count;
        int segs = 0, n = 0;
        bool ok = true;
        while (n < count && ok) {
            const int g = segs & 1;
            const int32_t tiles = min(walk.u0 + walk.r.tiles(), end) - max(walk.u0, first), rows = walk.r.n * p.g;
            // A lane has four channels of every row.
            uint2 raw_q[kRows];
            const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(p.q) + (int64_t)walk.r.start * p.q_st + (int64_t)walk.kvh * p.g * p.q_sh + 4 * lane;
            int h = 0;
#pragma unroll
            for (int c = 0; c < kRows; ++c) {
                raw_q[c] = make_uint2(0u, 0u);
                if (c < rows) raw_q[c] = *reinterpret_cast<const uint2 *>(q + h * p.q_sh);
                if (++h == p.g) { h = 0; q += p.q_st; }
            }
            float most[kRows];
            float2 x[kRows][2];
#pragma unroll
            for (int c = 0; c < kRows; ++c) {
                x[c][0] = make_float2(__uint_as_float(raw_q[c].x << 16), __uint_as_float(raw_q[c].x & 0xffff0000u));
                x[c][1] = make_float2(__uint_as_float(raw_q[c].y << 16), __uint_as_float(raw_q[c].y & 0xffff0000u));
                // As whole numbers magnitudes compare as they do as numbers, NaN above all.
                const uint32_t a = max(__float_as_uint(x[c][0].x) & 0x7fffffffu, __float_as_uint(x[c][0].y) & 0x7fffffffu);
                const uint32_t b = max(__float_as_uint(x[c][1].x) & 0x7fffffffu, __float_as_uint(x[c][1].y) & 0x7fffffffu);
                most[c] = __uint_as_float(max(a, b));
            }
            const float top = warp_reduce(most, lane, [](float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); });
            // Lane c: 2^(7 - exponent) of row c's largest channel, at most 2^107; NaN for a row that is not finite.
            const uint32_t e = max(__float_as_uint(top) >> 23, 27u);
            float f_row = e == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float((261u - e) << 23);
            if (segs >= 2) ok = wait_all(&sh->q_empty[g], ((segs >> 1) - 1) & 1, sh, p);
            if (!ok) break;
            if (lane < kRows) sh->q_factor[g][lane] = p.scale_log2 / f_row;
            uint8_t *dst = smem + C::kOffQ + (uint32_t)g * C::kQBytes + (lane & 3) * 4;
#pragma unroll
            for (int c = 0; c < kRows; ++c) {
                const float f = __shfl_sync(0xffffffffu, f_row, c);
                float2 lo = __fmul2_rn(x[c][0], make_float2(f, f)), hi = __fmul2_rn(x[c][1], make_float2(f, f));
                const uint32_t one = take_e4m3(lo) | take_e4m3(hi) << 16, two = to_e4m3(lo) | to_e4m3(hi) << 16;
                const uint32_t to = (uint32_t)c * 128u + (((uint32_t)(lane >> 2) ^ (uint32_t)(c & 7)) << 4);
                *reinterpret_cast<uint32_t *>(dst + to) = one;
                const uint32_t to2 = (uint32_t)(kRows + c) * 128u + (((uint32_t)(lane >> 2) ^ (uint32_t)((kRows + c) & 7)) << 4);
                *reinterpret_cast<uint32_t *>(dst + to2) = two;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            if (lane == 0) {
                Segment s;
                s.tiles = tiles;
                s.key0 = walk.tile * kKeyTile;
                s.kv = walk.r.kv; s.pos0 = walk.r.pos0(); s.rows = rows;
                s.whole = tiles == walk.r.tiles();
                s.out = s.whole ? (int64_t)walk.r.start * p.Hq + (int64_t)walk.kvh * p.g
                                : (2 * (int64_t)blockIdx.x + (walk.u0 > first ? 1 : 0)) * p.few_rows;
                sh->seg[g] = s;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->q_full[g]));
            ++segs;
            n += tiles;
            if (n < count) walk_next(p, walk, lane);
        }
        // No more segments, in either buffer.
        for (int e = 0; e < 2 && ok; ++e, ++segs) {
            const int g = segs & 1;
            if (segs >= 2) ok = wait_all(&sh->q_empty[g], ((segs >> 1) - 1) & 1, sh, p);
            if (ok && lane == 0) { sh->seg[g].tiles = 0; mbar_arrive(smem_u32(&sh->q_full[g])); }
        }
        __syncwarp();
    } else if (warp == kMmaWarp) {
        // ------------------------------------------------------------------ MMA issuer (the whole warp walks, one lane issues)
        reg_dealloc<kLightRegs>();
        const bool leader = elect_one();
        constexpr uint32_t idesc_qk = idesc_f8f6f4_f32(128, C::kColsS, kE2M1, kE4M3, 0, 0);
        constexpr uint32_t idesc_pv = idesc_f8f6f4_f32(kHeadDim, C::kColsO, kE2M1, kE5M2, 1, 1);
        const uint64_t ring = smem_desc_sw128(sRing, 16, 1024);
        auto kv_wait = [&](int item) { return wait_all(&sh->kv_full[item % kSlots], (item / kSlots) & 1, sh, p); };
        auto kv_release = [&](int item) { if (leader) tc_commit(smem_u32(&sh->kv_empty[item % kSlots])); };
        // S(n) of a segment of Q buffer g; `last`: the segment's Q is not needed after it
        auto issue_qk = [&](int n, int g, bool last) {
            if (!kv_wait(2 * n)) return false;
            if (leader) {
                mma4<2, 2>(tmem + (uint32_t)(n & 1) * C::kColsS, ring + (uint32_t)(((2 * n) % kSlots) * (kCodeTile >> 4)),
                           smem_desc_sw128(sQ + (uint32_t)g * C::kQBytes, 16, 1024), idesc_qk, 0u);
                tc_commit(smem_u32(&sh->s_full[n & 1]));
                if (last) tc_commit(smem_u32(&sh->q_empty[g]));
            }
            kv_release(2 * n);
            return true;
        };
        int segs = 0, n = 0;
        bool ok = wait_all(&sh->q_full[0], 0, sh, p);
        int32_t tiles = ok ? sh->seg[0].tiles : 0;
        if (ok) ok = issue_qk(0, 0, tiles == 1);
        while (ok) {
            const int g = segs & 1;
            int32_t next = 0;
            for (int j = 0; j < tiles && ok; ++j, ++n) {
                if (j + 1 < tiles) {
                    ok = issue_qk(n + 1, g, j + 2 == tiles);
                } else if (n + 1 < count) {
                    ok = wait_all(&sh->q_full[g ^ 1], ((segs + 1) >> 1) & 1, sh, p);
                    if (!ok) break;
                    next = sh->seg[g ^ 1].tiles;
                    ok = issue_qk(n + 1, g ^ 1, next == 1);
                }
                if (ok) ok = kv_wait(2 * n + 1);
                if (ok) ok = wait_all(&sh->p_ready[n & 1], (n >> 1) & 1, sh, p);
                if (!ok) break;
                tc_fence_after();
                if (leader) {
                    mma4<256, (32 * C::kPRow >> 4)>(tmem + C::kColO, ring + (uint32_t)(((2 * n + 1) % kSlots) * (kCodeTile >> 4)),
                                                    desc_rows<C::kPRow>(sP + (uint32_t)(n & 1) * C::kPBytes), idesc_pv, j > 0 ? 1u : 0u);
                    tc_commit(smem_u32(&sh->pv_done));
                }
                kv_release(2 * n + 1);
            }
            if (next == 0) break;
            tiles = next;
            ++segs;
        }
        if (!ok) drain_products(&sh->drained, leader, p);
        __syncwarp();
    } else if (warp == kScaleWarp) {
        // ------------------------------------------------------------------ scales: a lane has keys 4 lane .. + 3 of each tile
        // They lie in one page (boxes are eight keys at least).  Loads run two tiles ahead of the stores, the page's number one more.
        reg_dealloc<kLightRegs>();
        const int32_t end = first + count;
        const BoxStep step = box_step(p.c.page_size);
        const BoxLane bl = {4 * lane, 0u, true};
        int32_t left = min(walk.u0 + walk.r.tiles(), end) - max(walk.u0, first), k0 = walk.tile * kKeyTile, seen = 0;
        BoxPlace at = box_place(p.c.page_size, k0, bl);
        int32_t page = -1, row = 0, keys = 0, kvh = 0;     // of the next tile to load: its keys before the request's end
        auto look_up = [&] {                               // of the walk's tile; then to the next one
            row = at.row; kvh = walk.kvh;
            keys = min(max(walk.r.kv - k0 - 4 * lane, 0), 4);
            page = keys > 0 ? __ldg(p.c.table + walk.b * p.c.table_stride + at.nth) : -1;
            if (++seen >= count) return;
            if (--left > 0) {
                k0 += kKeyTile;
                at = box_next(at, step);
            } else {
                walk_next(p, walk, lane);
                left = min(walk.u0 + walk.r.tiles(), end) - walk.u0;
                k0 = 0;
                at = box_place(p.c.page_size, 0, bl);
            }
        };
        struct Four { uint32_t k01, k23, v01, v23; };      // bf16 bits
        Four set[3];
        auto load = [&](Four &x) {                         // keys past the end, and pages out of range (the loader reports them): 0
            x = {0u, 0u, 0u, 0u};
            if (page < 0 || page >= p.c.num_pages) return;
            const uint16_t *k = p.k_scales + page * p.ks_sp + row * p.ks_st + kvh * p.ks_sh, *v = p.v_scales + page * p.vs_sp + row * p.vs_st + kvh * p.vs_sh;
            if (scales_by_four) {                          // (a page holds all four, whatever is in those past the end)
                const uint2 a = __ldg(reinterpret_cast<const uint2 *>(k)), b = __ldg(reinterpret_cast<const uint2 *>(v));
                x = {a.x, a.y, b.x, b.y};
            } else {
                x.k01 = __ldg(k) | (uint32_t)__ldg(k + p.ks_st) << 16;
                x.k23 = __ldg(k + 2 * p.ks_st) | (uint32_t)__ldg(k + 3 * p.ks_st) << 16;
                x.v01 = __ldg(v) | (uint32_t)__ldg(v + p.vs_st) << 16;
                x.v23 = __ldg(v + 2 * p.vs_st) | (uint32_t)__ldg(v + 3 * p.vs_st) << 16;
            }
        };
        int32_t valid[3];                                  // keys of each set
        look_up();
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            valid[u] = 0;
            if (u < count) {
                load(set[u]);
                valid[u] = keys;
                if (u + 1 < count) look_up();
            }
        }
        bool ok = true;
        for (int n0 = 0; n0 < count && ok; n0 += 3) {
#pragma unroll
            for (int u = 0; u < 3; ++u) {
                const int n = n0 + u;
                if (n >= count || !ok) break;
                if (n + 2 < count) {
                    load(set[(u + 2) % 3]);
                    valid[(u + 2) % 3] = keys;
                    if (n + 3 < count) look_up();
                }
                const int slot = n % kScaleSlots;
                if (n >= kScaleSlots) ok = wait_all(&sh->sc_empty[slot], (n / kScaleSlots - 1) & 1, sh, p);
                if (!ok) break;
                const Four x = set[u];
                const int have = valid[u];
                uint4 w = make_uint4(__byte_perm(x.k01, x.v01, 0x5410), __byte_perm(x.k01, x.v01, 0x7632),
                                     __byte_perm(x.k23, x.v23, 0x5410), __byte_perm(x.k23, x.v23, 0x7632));
                if (have < 4) {
                    if (have < 1) w.x = 0u;
                    if (have < 2) w.y = 0u;
                    if (have < 3) w.z = 0u;
                    w.w = 0u;
                }
                *reinterpret_cast<uint4 *>(&sh->scale[slot][4 * lane]) = w;
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->sc_full[slot]));
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------------ softmax and epilogue
        reg_alloc<kSoftmaxRegs>();
        const int quarter = warp, key = tid;               // and channel `key` of the accumulator
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const uint32_t tO = tmem + lane_base + C::kColO;
        // P'^T: a row of kPRow bytes per key, its 16-byte chunks XOR-swizzled by bits of the key.
        const uint32_t p_row = (uint32_t)key * C::kPRow, p_swizzle = (C::kPRow == 32 ? (uint32_t)(key >> 2) & 1u : (uint32_t)(key >> 1) & 3u) << 4;
        constexpr int kPairs = kRows / 2;
        int n = 0, turn = 0;                               // tiles so far; exchanges take turns in two buffers (see pec_paged_few.cu)
        for (int k = 0;; ++k) {
            bool ok = wait_all(&sh->q_full[k & 1], (k >> 1) & 1, sh, p);
            if (group_any(0, !ok)) break;
            const Segment s = sh->seg[k & 1];
            float2 factor[kPairs];
#pragma unroll
            for (int c = 0; c < kPairs; ++c) factor[c] = make_float2(sh->q_factor[k & 1][2 * c], sh->q_factor[k & 1][2 * c + 1]);
            __syncwarp();
            if (s.tiles == 0) break;
            if (lane == 0) mbar_arrive(smem_u32(&sh->q_empty[k & 1]));
            const int32_t see_all = (p.causal && s.pos0 + 1 < s.kv) ? s.pos0 + 1 : s.kv;           // keys below it are visible to every row
            // Per row: minus the reference maximum (log2 units, the same in all threads; rows past the segment's: -inf, and all their
            // probabilities 0), this thread's sum.
            float2 neg_m[kPairs], l[kPairs];
            float m_row = (lane & (kRows - 1)) < s.rows ? kNoKey : INFINITY;   // reference of row lane % kRows
#pragma unroll
            for (int c = 0; c < kPairs; ++c) {
                neg_m[c] = make_float2(2 * c < s.rows ? -kNoKey : -INFINITY, 2 * c + 1 < s.rows ? -kNoKey : -INFINITY);
                l[c] = make_float2(0.f, 0.f);
            }
            float v_ref = 0.f, v_factor = 0.f;             // a power of two that no scale of V passes four times; kBase / v_ref
            int32_t k0 = s.key0;
            bool stop = false;
            for (int j = 0; j < s.tiles; ++j, ++n, k0 += kKeyTile) {
                const int buf = n & 1, slot = n % kScaleSlots;
                ok = wait_all(&sh->sc_full[slot], (n / kScaleSlots) & 1, sh, p);
                const uint32_t scales = sh->scale[slot][key];
                const float2 scale = make_float2(__uint_as_float(scales << 16), __uint_as_float(scales & 0xffff0000u));   // K, V
                if (ok) ok = wait_all(&sh->s_full[buf], (n >> 1) & 1, sh, p);
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->sc_empty[slot]));
                tc_fence_after();
                uint32_t r[C::kColsS];
                if constexpr (C::kColsS == 16) tmem_ld16(tmem + lane_base + (uint32_t)buf * C::kColsS, r);
                else tmem_ld32(tmem + lane_base + (uint32_t)buf * C::kColsS, r);
                tc_fence_before();
                float2 x[kPairs];
#pragma unroll
                for (int c = 0; c < kPairs; ++c) {
                    const float2 hi = make_float2(__uint_as_float(r[2 * c]), __uint_as_float(r[2 * c + 1]));
                    const float2 lo = make_float2(__uint_as_float(r[kRows + 2 * c]), __uint_as_float(r[kRows + 2 * c + 1]));
                    x[c] = __fmul2_rn(__ffma2_rn(lo, make_float2(1.f / 16.f, 1.f / 16.f), hi), __fmul2_rn(factor[c], make_float2(scale.x, scale.x)));
                }
                const bool border = k0 + kKeyTile > see_all;
                if (border) {                              // by choice, not by arithmetic: a masked score may be anything
                    int t = 0, h = 0;                      // token and head of the row
#pragma unroll
                    for (int c = 0; c < kRows; ++c) {
                        const int32_t see = p.causal ? min(s.kv, s.pos0 + t + 1) : s.kv;
                        float &y = c & 1 ? x[c / 2].y : x[c / 2].x;
                        y = k0 + key < see ? y : -INFINITY;
                        if (++h == p.g) { h = 0; ++t; }
                    }
                }
                float2 d[kPairs];                          // over the reference maxima
                float most_d = -INFINITY;
#pragma unroll
                for (int c = 0; c < kPairs; ++c) {
                    d[c] = __fadd2_rn(x[c], neg_m[c]);
                    most_d = fmax3(most_d, d[c].x, d[c].y);
                }
                const bool grow = most_d > kGrow || scale.y > 4.f * v_ref;
                // The references move only when one is outgrown (and at first); O then waits for its product in flight.  (S(n) is
                // complete, and with it PV(n - 2), issued before it; PV(n) needs this P(n): the parity tells PV(n - 1)'s phase.)
                if (j == 0 || group_any(0, grow || !ok)) {
                    if (j > 0 && ok) ok = wait_all(&sh->pv_done, (n - 1) & 1, sh, p);
                    stop = group_any(0, !ok);
                    if (stop) break;
                    float y[kRows];
#pragma unroll
                    for (int c = 0; c < kPairs; ++c) { y[2 * c] = x[c].x; y[2 * c + 1] = x[c].y; }
                    const float most = warp_reduce(y, lane, [](float a, float b) { return fmaxf(a, b); });
                    float v_most = fmaxf(scale.y, 0.f);
#pragma unroll
                    for (int i = 16; i > 0; i >>= 1) v_most = fmaxf(v_most, __shfl_xor_sync(0xffffffffu, v_most, i));
                    float4 *red = sh->red[turn ^= 1];
                    if (lane < kRows) reinterpret_cast<float *>(red + lane)[quarter] = most;
                    if (lane == 0) reinterpret_cast<float *>(red + 16)[quarter] = v_most;
                    group_any(0, false);
                    // Lane c works out row c's new reference; the others get it by shuffle.
                    const float4 t = red[lane & (kRows - 1)], tv = red[16];
                    const float v_top = fmaxf(fmaxf(fmaxf(tv.x, tv.y), fmaxf(tv.z, tv.w)), 0x1p-100f);
                    float v_alpha = 1.f;
                    if (v_top > 4.f * v_ref) {             // the power of two above it
                        const float ref = __uint_as_float((__float_as_uint(v_top) & 0x7f800000u) + 0x00800000u);
                        v_alpha = v_ref / ref;             // 0 at first
                        v_ref = ref;
                        v_factor = kBase / ref;
                    }
                    const float top = fmaxf(fmaxf(t.x, t.y), fmaxf(t.z, t.w));
                    const bool move = top > m_row + kGrow;
                    const float a_row = move ? ex2(m_row - top) : 1.f;     // 0 when the row had no key so far
                    if (move) m_row = top;
                    float alpha[kRows];
#pragma unroll
                    for (int c = 0; c < kRows; ++c) {
                        const float m = __shfl_sync(0xffffffffu, m_row, c);
                        alpha[c] = __shfl_sync(0xffffffffu, a_row, c);
                        float &lc = c & 1 ? l[c / 2].y : l[c / 2].x, &nm = c & 1 ? neg_m[c / 2].y : neg_m[c / 2].x;
                        lc *= alpha[c];
                        nm = -m;
                        alpha[c] *= v_alpha;
                    }
#pragma unroll
                    for (int c = 0; c < kPairs; ++c) d[c] = __fadd2_rn(x[c], neg_m[c]);
                    if (j > 0) {
                        tc_fence_after();
                        if constexpr (kRows == 4) {
                            uint32_t o[16];
                            tmem_ld16(tO, o);
#pragma unroll
                            for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * alpha[c % kRows]);
                            tmem_st16(tO, o);
                        } else {
#pragma unroll
                            for (int i = 0; i < C::kColsO; i += 32) {
                                uint32_t o[32];
                                tmem_ld32(tO + i, o);
#pragma unroll
                                for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * alpha[c % kRows]);
                                tmem_st32(tO + i, o);
                            }
                        }
                        tmem_st_wait();
                        tc_fence_before();
                    }
                }
                // p = 2^(x - m); the row's sum takes p itself, the product p sv / v_ref in four parts.
                const float f = scale.y * v_factor;
#pragma unroll
                for (int c = 0; c < kPairs; ++c) {
                    d[c] = make_float2(ex2(d[c].x), ex2(d[c].y));
                    l[c] = __fadd2_rn(l[c], d[c]);
                    d[c] = __fmul2_rn(d[c], make_float2(f, f));
                }
                if (border && !(f < INFINITY)) {           // a value that is not finite spoils no row that does not see it
#pragma unroll
                    for (int c = 0; c < kPairs; ++c) {
                        if (x[c].x == -INFINITY) d[c].x = 0.f;
                        if (x[c].y == -INFINITY) d[c].y = 0.f;
                    }
                }
                uint32_t parts[kRows / 4][4];
#pragma unroll
                for (int c = 0; c < kRows / 4; ++c) split_e5m2(d[2 * c], d[2 * c + 1], parts[c]);
                // (S(n) is complete, and with it PV(n - 2), which read this buffer.)
                uint8_t *dst = smem + C::kOffP + (uint32_t)buf * C::kPBytes + p_row;
                if constexpr (kRows == 4) {
                    *reinterpret_cast<uint4 *>(dst + p_swizzle) = make_uint4(parts[0][0], parts[0][1], parts[0][2], parts[0][3]);
                } else if constexpr (kRows == 8) {
                    *reinterpret_cast<uint4 *>(dst + p_swizzle) = make_uint4(parts[0][0], parts[1][0], parts[0][1], parts[1][1]);
                    *reinterpret_cast<uint4 *>(dst + (16u ^ p_swizzle)) = make_uint4(parts[0][2], parts[1][2], parts[0][3], parts[1][3]);
                } else {
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i)
                        *reinterpret_cast<uint4 *>(dst + ((i << 4) ^ p_swizzle)) = make_uint4(parts[0][i], parts[1][i], parts[2][i], parts[3][i]);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->p_ready[buf]));
            }
            if (stop) break;
            ok = wait_all(&sh->pv_done, (n - 1) & 1, sh, p);
            float y[kRows];
#pragma unroll
            for (int c = 0; c < kPairs; ++c) { y[2 * c] = l[c].x; y[2 * c + 1] = l[c].y; }
            const float part = warp_reduce(y, lane, [](float a, float b) { return a + b; });
            float4 *red = sh->red[turn ^= 1];
            if (lane < kRows) reinterpret_cast<float *>(red + lane)[quarter] = part;
            if (group_any(0, !ok)) break;
            tc_fence_after();
            uint32_t o[C::kColsO];
            if constexpr (kRows == 4) {
                tmem_ld16(tO, o);
            } else {
                tmem_ld32(tO, *reinterpret_cast<uint32_t (*)[32]>(o));
                if constexpr (kRows == 16) tmem_ld32(tO + 32, *reinterpret_cast<uint32_t (*)[32]>(o + 32));
            }
            tc_fence_before();
            // Lane c works out row c's factor, place and LSE.
            const int row = lane & (kRows - 1);
            const float4 t = red[row];
            const float sum = (t.x + t.y) + (t.z + t.w);
            const int64_t at = s.whole ? s.out + (int64_t)(row / p.g) * p.Hq + row % p.g : s.out + row;
            const float f_row = sum == 0.f ? 0.f : v_ref / kBase / sum;
            if (quarter == 0 && lane < s.rows && lane < kRows)
                (s.whole ? p.lse : p.few_lse)[at] = sum == 0.f ? -INFINITY : m_row * 0.6931471805599453f + logf(sum);
#pragma unroll
            for (int c = 0; c < kRows; ++c) {
                if (c >= s.rows) break;
                const float f = __shfl_sync(0xffffffffu, f_row, c);
                const int64_t to = __shfl_sync(0xffffffffu, at, c) * kHeadDim + key;
                float sum_o = __uint_as_float(o[3 * kRows + c]);
#pragma unroll
                for (int i = 2; i >= 0; --i) sum_o = fmaf(sum_o, 0.125f, __uint_as_float(o[i * kRows + c]));
                const float y = f == 0.f ? 0.f : sum_o * f;
                if (s.whole && p.o_is_bf16) static_cast<__nv_bfloat16 *>(p.o)[to] = __float2bfloat16_rn(y);
                else (s.whole ? static_cast<float *>(p.o) : p.few_o)[to] = y;
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) tmem_dealloc(tmem, C::kTmemCols);
    // Beside the last CTAs of the kernel for many rows, which write other rows; but whoever waits for this kernel waits for that one.
    griddep_wait();
}

// Whether the scales of four tokens can be loaded at once.
static bool by_four(const uint16_t *s, int64_t sp, int64_t st, int64_t sh) { return st == 1 && sp % 4 == 0 && sh % 4 == 0 && reinterpret_cast<uintptr_t>(s) % 8 == 0; }

template <int kRows>
static cudaError_t launch(const Params &p, const CUtensorMap &tm_k, const CUtensorMap &tm_v, int box, bool after_many, cudaStream_t stream)
{
    return launch_dependent(paged_few_q4_kernel<kRows>, dim3((unsigned)p.few_ctas), kThreads, smem_bytes<kRows>(), stream, after_many, tm_k, tm_v, p, box,
                            by_four(p.k_scales, p.ks_sp, p.ks_st, p.ks_sh) && by_four(p.v_scales, p.vs_sp, p.vs_st, p.vs_sh), (int)test_skip_last_load());
}

}  // namespace few_q4
}  // namespace paged

int launch_paged_few_q4(const paged::Params &p, bool after_many, cudaStream_t stream)
{
    using namespace paged;
    const int box = host_map::box_rows(p.c.page_size);
    CUtensorMap tm_k, tm_v;
    if (!host_map::pages_q4(&tm_k, p, p.k_pages, p.c.k_sp, p.c.k_st, p.c.k_sh, box) ||
        !host_map::pages_q4(&tm_v, p, p.v_pages, p.c.v_sp, p.c.v_st, p.c.v_sh, box)) {
        set_error("%s: cuTensorMapEncodeTiled failed (driver too old, or strides/addresses not encodable)", p.who);
        return PEC_ERR_CUDA;
    }
    static unsigned char ready[host::kMaxDevices] = {};
    static std::mutex ready_mutex;
    if (!host::once_per_device(ready, ready_mutex, [] {
            return cudaFuncSetAttribute(few_q4::paged_few_q4_kernel<4>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)few_q4::smem_bytes<4>()) == cudaSuccess &&
                   cudaFuncSetAttribute(few_q4::paged_few_q4_kernel<8>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)few_q4::smem_bytes<8>()) == cudaSuccess &&
                   cudaFuncSetAttribute(few_q4::paged_few_q4_kernel<16>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)few_q4::smem_bytes<16>()) == cudaSuccess; })) {
        (void)cudaGetLastError();
        set_error("%s: cannot raise the shared-memory limit", p.who);
        return PEC_ERR_CUDA;
    }
    // The form for as many rows as a request can have (p.few_rows).
    cudaError_t err = p.few_rows <= 4 ? few_q4::launch<4>(p, tm_k, tm_v, box, after_many, stream)
                    : p.few_rows <= 8 ? few_q4::launch<8>(p, tm_k, tm_v, box, after_many, stream) : few_q4::launch<16>(p, tm_k, tm_v, box, after_many, stream);
    if (err == cudaSuccess) err = cudaGetLastError();
    if (err != cudaSuccess) { set_error("%s: launch failed: %s", p.who, cudaGetErrorString(err)); return PEC_ERR_CUDA; }
    return PEC_OK;
}

}  // namespace pec
