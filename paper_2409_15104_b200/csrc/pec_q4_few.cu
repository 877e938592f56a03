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
//         bf16's eight; channels under 2^-13 of the row's largest are held to 2^-21 of it (half of e4m3's last step, 2^-9 / 16)
//     P'  four parts of e5m2: rounded to fp16, 2^-11 of itself down to 2^-24 v_ref and 2^-35 v_ref below, so that a bf16 result errs by
//         its own rounding alone.  (Parts of e4m3, three for as many bits, end at 2^-21: a hundred thousand keys behind one that takes
//         most of the weight, which long prompts have, would be held to two bits.)
// Products of such numbers are exact and their sums are kept in fp32.
//
// The split of the work is that of pec_paged_few.cu: the key tiles of all (request, KV head) units on one line, an equal piece of it
// for each CTA, units that cross a cut merged by the combining kernel.
//
// A tile has 750 cycles at the rate of HBM, and every warp of the chain (where it lies, its copies, products, softmax, products) spends
// most of its time on hand-overs.  So two CTAs per SM, and a step takes 256 keys where shared memory has room for it (up to 8 rows).
//
// Measured: 64 requests of 2400 keys, 32 heads on 8: 47 us (3.4 TB/s); three of 102000, 64 on 8: 72 us (4.5 TB/s, 5.5 without the 12 us of
// start and combine); one of 4100: 14 us; 16 requests of 4 tokens (16 rows) and 9000 keys: 74 us, 2000 cycles a tile, which the
// softmax warps take with 16 rows a key and four parts of each probability.
//
// Warp roles:
//   warps 0-3  softmax and epilogue
//   warp 4     MMA issuer (one thread)
//   warp 5, 7  loaders of K and V: codes by the copy unit, scales (rings of steps).  Two, because a copy of 128 rows of 64 bytes keeps the
//              warp that starts it for 400 to 600 cycles
//   warp 6     walks the line: where each step lies, for the loaders; descriptor and Q of each segment (two buffers)
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <cstddef>
#include "pec_paged_tma.cuh"
#include "pec_q4.cuh"

namespace pec {
using namespace sm100;
namespace paged {
namespace few_q4 {

constexpr int kThreads = 256;
constexpr int kMmaWarp = 4, kKeyWarp = 5, kPlanWarp = 6, kValueWarp = 7;
constexpr int kSoftmaxRegs = 176, kLightRegs = 80;         // 128 * (176 + 80) = 256 * 128 (the launch allocation)
constexpr uint32_t kCodeTile = 128 * 128;                  // 128 tokens, their 64 bytes spread over 128
constexpr int kScaleSlots = 2, kPlanSlots = 3;
constexpr float kNoKey = -3.0e38f;                         // reference maximum of a row that has seen no key
constexpr float kGrow = 3.0f;                              // log2 units: a row's reference maximum moves when outgrown by 2^3
constexpr float kBase = 1024.0f;                           // p * sv / v_ref is at most 2^3 * 4; times 2^10 it stays below e5m2's 57344

template <int kRows> struct Cfg {
    static constexpr int kSub = kRows == 16 ? 1 : 2;       // tiles of 128 keys in a step
    // Rings of steps.  K's is the longer one: its products make the scores that the softmax waits for, those of V may run a step late.
    static constexpr int kKeys = kSub * kKeyTile, kSlotsK = kRows == 16 ? 3 : 2, kSlotsV = kRows == 16 ? 2 : 1;
    static constexpr uint32_t kSlotBytes = kSub * kCodeTile;
    static constexpr int kColsS = kRows == 4 ? 16 : 2 * kRows, kColsO = 4 * kRows;      // (a product has 16 columns at least)
    static constexpr uint32_t kQBytes = kColsS * 128, kPRow = kRows == 16 ? 64 : 32, kPBytes = kKeys * kPRow;
    static constexpr uint32_t kColO = 2 * kSub * kColsS, kTmemCols = kColO + kColsO <= 128 ? 128 : 256;
    static constexpr uint32_t kOffQ = 0, kOffP = 2 * kQBytes, kOffK = kOffP + kPBytes, kOffV = kOffK + kSlotsK * kSlotBytes, kOffEnd = kOffV + kSlotsV * kSlotBytes;
};

struct Segment {
    int32_t tiles;                                         // of 128 keys; 0: no more segments
    int32_t key0, key_end;                                 // positions of its keys: a request's, or a piece of them
    int32_t pos0, rows;
    int64_t out;                                           // whole unit: (first token row * Hq + first head); else partial slot * few_rows
    int32_t whole;
};
struct Plan { int32_t page[32], row[32], kvh, valid, last; };          // of a step: where each eight keys lie; its keys, < 0: no more steps
struct Shared {
    uint64_t q_full[2], q_empty[2];                        // descriptor and Q of every other segment
    uint64_t kv_full[2][3], kv_empty[2][3];                // K, V
    uint64_t sc_full[kScaleSlots], sc_empty[kScaleSlots], plan_full[kPlanSlots], plan_empty[kPlanSlots];
    uint64_t s_full[2], p_ready;                           // [TMEM buffer]
    uint64_t pv_done, drained;
    Segment seg[2];
    Plan plan[kPlanSlots];
    float q_factor[2][16];                                 // of a row's scores: log2 units of the scaled score over that of the product
    float4 red[2][17];                                     // every other exchange: rows, the scales of V; one component per warp
    __align__(16) uint16_t scale[kScaleSlots][2][2 * kKeyTile];           // K, V; bf16 bits
    int32_t any;                                           // 0: the CTA's piece of the line is empty
    uint32_t tmem_base;
    volatile int abort_flag;
};
static_assert(offsetof(Shared, scale) % 16 == 0 && offsetof(Shared, red) % 16 == 0, "written four at a time");
template <int kRows> constexpr size_t smem_bytes()
{
    return Cfg<kRows>::kOffEnd + 1024 /*alignment slack*/ + sizeof(Shared);
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

// Slot and parity of a ring's successive items: wait for the slot's full barrier with `phase`, for its empty one, from the second round
// on, with phase ^ 1.  One reader and one writer each: a writer a round ahead of another would take a phase's parity for an older one's.
struct Ring {
    uint32_t slot, phase;
    __device__ __forceinline__ void next(uint32_t slots)
    {
        if (++slot == slots) { slot = 0; phase ^= 1u; }
    }
};

template <int kRows>
__global__ void __launch_bounds__(kThreads, kFewCtasQ4)
paged_few_q4_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const Params p, const int box,
                    const int scales_by_eight, const int skip_last)
{
    typedef Cfg<kRows> C;
    constexpr int kSub = C::kSub;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t *const smem = smem_raw + (base - raw);
    const uint32_t sQ = base + C::kOffQ, sP = base + C::kOffP;
    Shared *sh = reinterpret_cast<Shared *>(smem + C::kOffEnd);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    Walk walk;
    int32_t first = 0, count = 0;                          // this CTA's piece of the line (plan warp)
    if (warp == kPlanWarp) {
        if (lane == 0) {
            griddep_launch_dependents();                   // the combining kernel may be launched; it waits for this one's end
            sh->abort_flag = 0;
            for (int g = 0; g < 2; ++g) {
                mbar_init(smem_u32(&sh->q_full[g]), 1);
                mbar_init(smem_u32(&sh->q_empty[g]), 5);   // four softmax warps, the issuer's commit
                mbar_init(smem_u32(&sh->s_full[g]), 1);
            }
            for (int w = 0; w < 2; ++w)
                for (int s = 0; s < 3; ++s) { mbar_init(smem_u32(&sh->kv_full[w][s]), 1); mbar_init(smem_u32(&sh->kv_empty[w][s]), 1); }
            for (int s = 0; s < kScaleSlots; ++s) { mbar_init(smem_u32(&sh->sc_full[s]), 2); mbar_init(smem_u32(&sh->sc_empty[s]), 4); }
            for (int s = 0; s < kPlanSlots; ++s) { mbar_init(smem_u32(&sh->plan_full[s]), 1); mbar_init(smem_u32(&sh->plan_empty[s]), 2); }
            mbar_init(smem_u32(&sh->p_ready), 4);
            mbar_init(smem_u32(&sh->pv_done), 1);
            mbar_init(smem_u32(&sh->drained), 1);
            mbar_init_fence();
        }
        const int32_t all = walk_tiles(p, walk, lane), piece = few_piece(p, all);
        first = (int32_t)blockIdx.x * piece;
        count = min(max(all - first, 0), piece);
        if (count > 0) walk_to(p, walk, first, lane);
        if (lane == 0) sh->any = count > 0;
    } else if (warp == kMmaWarp) {
        tmem_alloc(smem_u32(&sh->tmem_base), C::kTmemCols);
        tmem_relinquish();
    } else if (warp == kKeyWarp && lane == 0) {
        prefetch_tmap(&tm_k); prefetch_tmap(&tm_v);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh->tmem_base;

    if (!sh->any) {
    } else if (warp == kKeyWarp || warp == kValueWarp) {
        // ------------------------------------------------------------------ loader of K or V
        // Codes: a lane has a box of one page.  Scales: a lane has eight keys; they go a step ahead of the codes, whose slot may be taken.
        reg_dealloc<kLightRegs>();
        const int which = warp == kValueWarp;
        const CUtensorMap *map = which ? &tm_v : &tm_k;
        const uint16_t *scales = which ? p.v_scales : p.k_scales;
        const int64_t s_p = which ? p.vs_sp : p.ks_sp, s_t = which ? p.vs_st : p.ks_st, s_h = which ? p.vs_sh : p.ks_sh;
        const int32_t mine = lane * box;                   // this lane's first key of each step
        const int slots = which ? C::kSlotsV : C::kSlotsK;
        const uint32_t sRing = base + (which ? C::kOffV : C::kOffK);
        Ring ring = {0u, 0u}, sc = {0u, 0u}, pl = {0u, 0u};
        struct Step { int32_t page, row, kvh, valid, last; } now, next = {};
        uint4 x;                                           // the next step's scales
        int32_t own = 0;                                   // of this lane's eight keys, those before the end
        bool ok = true;
        auto take_plan = [&] {                             // into `next`; starts the load of its scales
            ok = wait_all(&sh->plan_full[pl.slot], pl.phase, sh, p);
            const Plan &plan = sh->plan[pl.slot];
            const int group = (mine >> 3) & 31;
            next = {plan.page[group], plan.row[group], plan.kvh, plan.valid, plan.last};
            const int32_t sc_page = plan.page[lane], sc_row = plan.row[lane];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->plan_empty[pl.slot]));
            pl.next(kPlanSlots);
            // (Keys past the end have scale 0: what is in their place may be anything.  A page holds all eight, whatever is in those.)
            x = make_uint4(0u, 0u, 0u, 0u);
            own = next.valid - 8 * lane;
            if (!ok || own <= 0) return;
            const uint16_t *at = scales + sc_page * s_p + sc_row * s_t + next.kvh * s_h;
            if (scales_by_eight) {
                x = __ldg(reinterpret_cast<const uint4 *>(at));
            } else {
                auto two = [&](int i) { return __ldg(at + i * s_t) | (uint32_t)__ldg(at + (i + 1) * s_t) << 16; };
                x = make_uint4(two(0), two(2), two(4), two(6));
            }
        };
        auto store_scales = [&](int m) {                   // of step m, taken last
            if (m >= kScaleSlots) ok = wait_all(&sh->sc_empty[sc.slot], sc.phase ^ 1u, sh, p);
            if (!ok) return;
            if (own < 8) {
                uint32_t *w = &x.x;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = own > 2 * i + 1 ? w[i] : own > 2 * i ? w[i] & 0xffffu : 0u;
            }
            if (8 * lane < C::kKeys) *reinterpret_cast<uint4 *>(&sh->scale[sc.slot][which][8 * lane]) = x;
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->sc_full[sc.slot]));
            sc.next(kScaleSlots);
        };
        int n = 0;
        take_plan();
        if (ok) store_scales(0);
        for (; ok; ++n) {
            now = next;
            if (now.valid < 0) break;
            take_plan();
            if (ok && n >= slots) ok = wait_all(&sh->kv_empty[which][ring.slot], ring.phase ^ 1u, sh, p);
            if (skip_last && which && n > 0 && now.last) ok = false;       // test hook: the wait for it runs out
            if (!ok) break;
            const int32_t keys = (now.valid + box - 1) & -box;             // whole boxes (box is a power of two)
            const uint32_t bar = smem_u32(&sh->kv_full[which][ring.slot]);
            if (lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)keys * 64u);
            __syncwarp();
            if (mine < keys) tma_load_4d(sRing + ring.slot * C::kSlotBytes + (uint32_t)mine * 128u, map, bar, 0, now.row, now.kvh, now.page);
            ring.next(slots);
            if (next.valid >= 0) store_scales(n + 1);
        }
        // Given up: the copies under way must land before the CTA may leave.
        if (!ok && lane == 0)
            for (int i = max(n - slots, 0); i < n; ++i) wait_quietly(&sh->kv_full[which][i % slots], (i / slots) & 1, p);
        __syncwarp();
    } else if (warp == kPlanWarp) {
        // ------------------------------------------------------------------ walk along the line, two steps ahead of the plans
        reg_dealloc<kLightRegs>();
        // An earlier CTA's wait has run out: the launch is lost, every wait of this CTA gives up at its next try.
        if (lane == 0 && *reinterpret_cast<volatile int32_t *>(p.status) == PEC_ERR_TIMEOUT) sh->abort_flag = 1;
        const int32_t end = first + count;
        const BoxStep step = {C::kKeys / p.c.page_size, C::kKeys % p.c.page_size, p.c.page_size};
        const BoxLane bl = {8 * lane, 0u, true};            // eight keys: one page, as boxes are eight at least
        int32_t k0 = walk.tile * kKeyTile, left = min(walk.u0 + walk.r.tiles(), end) - max(walk.u0, first);    // of the walk's step; of its segment, in tiles
        int32_t key_end = min(walk.r.kv, k0 + left * kKeyTile);
        count -= left;                                     // tiles of later segments
        BoxPlace at = box_place(p.c.page_size, k0, bl);
        int segs = 0;
        // The walk's segment begins: descriptor and Q.
        auto begin = [&] {
            const int g = segs & 1, rows = walk.r.n * p.g;
            if (segs >= 2 && !wait_all(&sh->q_empty[g], ((segs >> 1) - 1) & 1, sh, p)) return false;
            // Four rows at a time, a lane with four channels of each.
            const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(p.q) + (int64_t)walk.r.start * p.q_st + (int64_t)walk.kvh * p.g * p.q_sh + 4 * lane;
            int h = 0;
            uint2 raw_q[4];
            auto fetch = [&](int c0) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    raw_q[c] = make_uint2(0u, 0u);
                    if (c0 + c < rows) raw_q[c] = *reinterpret_cast<const uint2 *>(q + h * p.q_sh);
                    if (++h == p.g) { h = 0; q += p.q_st; }
                }
            };
            fetch(0);
#pragma unroll 1
            for (int c0 = 0; c0 < kRows; c0 += 4) {
                float2 x[4][2];
                float most[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    x[c][0] = make_float2(__uint_as_float(raw_q[c].x << 16), __uint_as_float(raw_q[c].x & 0xffff0000u));
                    x[c][1] = make_float2(__uint_as_float(raw_q[c].y << 16), __uint_as_float(raw_q[c].y & 0xffff0000u));
                    // As whole numbers magnitudes compare as they do as numbers, NaN above all.
                    const uint32_t a = max(__float_as_uint(x[c][0].x) & 0x7fffffffu, __float_as_uint(x[c][0].y) & 0x7fffffffu);
                    const uint32_t b = max(__float_as_uint(x[c][1].x) & 0x7fffffffu, __float_as_uint(x[c][1].y) & 0x7fffffffu);
                    most[c] = __uint_as_float(max(a, b));
                }
                if (c0 + 4 < kRows) fetch(c0 + 4);
                const float top = warp_reduce(most, lane, [](float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); });
                // Lane c: 2^(7 - exponent) of row c's largest channel, at most 2^107; NaN for a row that is not finite.
                const uint32_t e = max(__float_as_uint(top) >> 23, 27u);
                const float f_row = e == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float((261u - e) << 23);
                if (lane < 4) sh->q_factor[g][c0 + lane] = p.scale_log2 / f_row;
                uint8_t *dst = smem + C::kOffQ + (uint32_t)g * C::kQBytes + (lane & 3) * 4;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float f = __shfl_sync(0xffffffffu, f_row, c);
                    float2 lo = __fmul2_rn(x[c][0], make_float2(f, f)), hi = __fmul2_rn(x[c][1], make_float2(f, f));
                    const uint32_t one = take_e4m3(lo) | take_e4m3(hi) << 16, two = to_e4m3(lo) | to_e4m3(hi) << 16;
                    const uint32_t r1 = (uint32_t)(c0 + c), r2 = r1 + kRows;
                    *reinterpret_cast<uint32_t *>(dst + r1 * 128u + (((uint32_t)(lane >> 2) ^ (r1 & 7u)) << 4)) = one;
                    *reinterpret_cast<uint32_t *>(dst + r2 * 128u + (((uint32_t)(lane >> 2) ^ (r2 & 7u)) << 4)) = two;
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            if (lane == 0) {
                Segment s;
                s.tiles = left;
                s.key0 = k0; s.key_end = key_end;
                s.pos0 = walk.r.pos0(); s.rows = rows;
                s.whole = left == walk.r.tiles();
                s.out = s.whole ? (int64_t)walk.r.start * p.Hq + (int64_t)walk.kvh * p.g
                                : (2 * (int64_t)blockIdx.x + (walk.u0 > first ? 1 : 0)) * p.few_rows;
                sh->seg[g] = s;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->q_full[g]));
            ++segs;
            return true;
        };
        struct Spot { int32_t page, row, kvh, valid; };
        auto spot = [&] {                                  // of the walk's step; the page's number is looked at two steps later
            Spot x = {-1, at.row, walk.kvh, max(min(key_end - k0, C::kKeys), 0)};
            if (bl.first < x.valid) x.page = __ldg(p.c.table + walk.b * p.c.table_stride + at.nth);
            return x;
        };
        bool fresh = false;                                // the walk's step is the first of a segment that is to begin
        auto advance = [&] {                               // to the next step; false: there is none
            left -= kSub;
            if (left > 0) {
                k0 += C::kKeys;
                at = box_next(at, step);
                return true;
            }
            if (count <= 0) return false;
            walk_next(p, walk, lane);
            left = min(walk.r.tiles(), count);
            count -= left;
            k0 = 0;
            key_end = min(walk.r.kv, left * kKeyTile);
            at = box_place(p.c.page_size, 0, bl);
            return fresh = true;
        };
        const Spot none = {-1, 0, 0, -1};
        bool ok = begin();
        Spot now = spot(), after = none;
        bool more = ok && advance();
        if (more) after = spot();
        Ring pl = {0u, 0u};
        for (int n = 0; ok; ++n) {
            if (n >= kPlanSlots) ok = wait_all(&sh->plan_empty[pl.slot], pl.phase ^ 1u, sh, p);
            if (!ok) break;
            // A page number out of range is reported, and page 0 read in its place.
            if (bl.first < now.valid && (now.page < 0 || now.page >= p.c.num_pages)) {
                raise_status(p.status, PEC_ERR_BAD_INDEX);
                now.page = 0;
            }
            Plan &plan = sh->plan[pl.slot];
            plan.page[lane] = now.page;
            plan.row[lane] = now.row;
            if (lane == 0) { plan.kvh = now.kvh; plan.valid = now.valid; plan.last = after.valid < 0; }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->plan_full[pl.slot]));
            pl.next(kPlanSlots);
            if (now.valid < 0) break;
            now = after;
            after = none;
            // Not before the plan of the step before has been handed over: a segment begins in the place of the one before the last, whose
            // last keys are loaded when the step after them is known.
            if (fresh) ok = begin();
            fresh = false;
            if (ok && more) {
                more = advance();
                if (more) after = spot();
            }
        }
        // No more segments, in either buffer.
        for (int e = 0; e < 2 && ok; ++e, ++segs) {
            const int g = segs & 1;
            if (segs >= 2) ok = wait_all(&sh->q_empty[g], ((segs >> 1) - 1) & 1, sh, p);
            if (ok && lane == 0) { sh->seg[g].tiles = 0; mbar_arrive(smem_u32(&sh->q_full[g])); }
        }
        __syncwarp();
    } else if (warp == kMmaWarp) {
        // ------------------------------------------------------------------ MMA issuer, one thread
        reg_dealloc<kLightRegs>();
        const bool leader = elect_one();
        bool ok = true;
        if (leader) {
            constexpr uint32_t idesc_qk = idesc_f8f6f4_f32(128, C::kColsS, kE2M1, kE4M3, 0, 0);
            constexpr uint32_t idesc_pv = idesc_f8f6f4_f32(kHeadDim, C::kColsO, kE2M1, kE5M2, 1, 1);
            const uint64_t k_desc = smem_desc_sw128(base + C::kOffK, 16, 1024), v_desc = smem_desc_sw128(base + C::kOffV, 16, 1024), q_desc = smem_desc_sw128(sQ, 16, 1024), p_desc = desc_rows<C::kPRow>(sP);
            auto wait = [&](uint64_t *bar, uint32_t parity) {
                return mbar_wait_bounded(smem_u32(bar), parity, &sh->abort_flag, p.status, p.wait_cycles, (int)PEC_ERR_TIMEOUT);
            };
            Ring k_ring = {0u, 0u}, v_ring = {0u, 0u};
            // S(n) of a segment of Q buffer g; `last`: the segment's Q is not needed after it.  (A step of one tile has a second one of
            // whatever codes lie there: its keys are masked.)
            auto issue_qk = [&](int n, int g, bool last) {
                if (!wait(&sh->kv_full[0][k_ring.slot], k_ring.phase)) return false;
#pragma unroll
                for (int i = 0; i < kSub; ++i)
                    mma4<2, 2>(tmem + (uint32_t)((n & 1) * kSub + i) * C::kColsS, k_desc + ((k_ring.slot * C::kSlotBytes + i * kCodeTile) >> 4),
                               q_desc + (uint32_t)g * (C::kQBytes >> 4), idesc_qk, 0u);
                tc_commit(smem_u32(&sh->s_full[n & 1]));
                tc_commit(smem_u32(&sh->kv_empty[0][k_ring.slot]));
                if (last) tc_commit(smem_u32(&sh->q_empty[g]));
                k_ring.next(C::kSlotsK);
                return true;
            };
            auto steps_of = [&](int g) { return (sh->seg[g].tiles + kSub - 1) / kSub; };
            int segs = 0, n = 0;
            ok = wait(&sh->q_full[0], 0);
            int32_t steps = ok ? steps_of(0) : 0;
            if (ok) ok = issue_qk(0, 0, steps == 1);
            while (ok) {
                const int g = segs & 1;
                int32_t next = 0;
                for (int j = 0; j < steps && ok; ++j, ++n) {
                    if (j + 1 < steps) {
                        ok = issue_qk(n + 1, g, j + 2 == steps);
                    } else {
                        ok = wait(&sh->q_full[g ^ 1], ((segs + 1) >> 1) & 1);
                        if (!ok) break;
                        next = steps_of(g ^ 1);
                        if (next > 0) ok = issue_qk(n + 1, g ^ 1, next == 1);
                    }
                    if (ok) ok = wait(&sh->kv_full[1][v_ring.slot], v_ring.phase);
                    if (ok) ok = wait(&sh->p_ready, n & 1);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int i = 0; i < kSub; ++i)
                        mma4<256, (32 * C::kPRow >> 4)>(tmem + C::kColO, v_desc + ((v_ring.slot * C::kSlotBytes + i * kCodeTile) >> 4),
                                                        p_desc + (uint32_t)i * (128 * C::kPRow >> 4), idesc_pv, j > 0 || i > 0 ? 1u : 0u);
                    tc_commit(smem_u32(&sh->pv_done));
                    tc_commit(smem_u32(&sh->kv_empty[1][v_ring.slot]));
                    v_ring.next(C::kSlotsV);
                }
                if (next == 0) break;
                steps = next;
                ++segs;
            }
        }
        __syncwarp();
        if (!__all_sync(0xffffffffu, ok)) drain_products(&sh->drained, leader, p);
        __syncwarp();
    } else {
        // ------------------------------------------------------------------ softmax and epilogue
        reg_alloc<kSoftmaxRegs>();
        const int quarter = warp, key = tid;               // key of each tile, and channel `key` of the accumulator
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const uint32_t tO = tmem + lane_base + C::kColO;
        // P'^T: a row of kPRow bytes per key, its 16-byte chunks XOR-swizzled by bits of the key.
        uint8_t *const p_row = smem + C::kOffP + (uint32_t)key * C::kPRow;
        const uint32_t p_swizzle = (C::kPRow == 32 ? (uint32_t)(key >> 2) & 1u : (uint32_t)(key >> 1) & 3u) << 4;
        constexpr int kPairs = kRows / 2;
        Ring sc = {0u, 0u};
        int n = 0, turn = 0;                               // steps so far; exchanges take turns in two buffers (see pec_paged_few.cu)
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
            const int32_t see_all = (p.causal && s.pos0 + 1 < s.key_end) ? s.pos0 + 1 : s.key_end;   // keys below it are visible to every row
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
            for (int j = 0; j < s.tiles; j += kSub, ++n, k0 += C::kKeys) {
                const int buf = n & 1;
                ok = wait_all(&sh->sc_full[sc.slot], sc.phase, sh, p);
                float ks[kSub], vs[kSub];
#pragma unroll
                for (int i = 0; i < kSub; ++i) {
                    ks[i] = __uint_as_float((uint32_t)sh->scale[sc.slot][0][i * kKeyTile + key] << 16);
                    vs[i] = __uint_as_float((uint32_t)sh->scale[sc.slot][1][i * kKeyTile + key] << 16);
                }
                if (ok) ok = wait_all(&sh->s_full[buf], (n >> 1) & 1, sh, p);
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->sc_empty[sc.slot]));
                sc.next(kScaleSlots);
                tc_fence_after();
                uint32_t r[kSub * C::kColsS];
                static_assert(kSub * C::kColsS == 32, "a step's scores");
                tmem_ld32(tmem + lane_base + (uint32_t)buf * 32u, r);
                tc_fence_before();
                float2 x[kSub][kPairs];
#pragma unroll
                for (int i = 0; i < kSub; ++i)
#pragma unroll
                    for (int c = 0; c < kPairs; ++c) {
                        const uint32_t *q = r + i * C::kColsS + 2 * c;
                        const float2 hi = make_float2(__uint_as_float(q[0]), __uint_as_float(q[1]));
                        const float2 lo = make_float2(__uint_as_float(q[kRows]), __uint_as_float(q[kRows + 1]));
                        x[i][c] = __fmul2_rn(__ffma2_rn(lo, make_float2(1.f / 16.f, 1.f / 16.f), hi), __fmul2_rn(factor[c], make_float2(ks[i], ks[i])));
                    }
                const bool border = k0 + C::kKeys > see_all;
                if (border) {                              // by choice, not by arithmetic: a masked score may be anything
                    int t = 0, h = 0;                      // token and head of the row
#pragma unroll
                    for (int c = 0; c < kRows; ++c) {
                        const int32_t see = (p.causal ? min(s.key_end, s.pos0 + t + 1) : s.key_end) - k0 - key;
#pragma unroll
                        for (int i = 0; i < kSub; ++i) {
                            float &y = c & 1 ? x[i][c / 2].y : x[i][c / 2].x;
                            y = i * kKeyTile < see ? y : -INFINITY;
                        }
                        if (++h == p.g) { h = 0; ++t; }
                    }
                }
                float2 d[kSub][kPairs];                    // over the reference maxima
                float most_d = -INFINITY, most_v = 0.f;
#pragma unroll
                for (int i = 0; i < kSub; ++i) {
                    most_v = fmaxf(most_v, vs[i]);
#pragma unroll
                    for (int c = 0; c < kPairs; ++c) {
                        d[i][c] = __fadd2_rn(x[i][c], neg_m[c]);
                        most_d = fmax3(most_d, d[i][c].x, d[i][c].y);
                    }
                }
                // The references move only when one is outgrown (and at first); O then waits for its product in flight, PV(n - 1).  (PV(n)
                // needs this P(n), and PV(n - 2) was waited for before P(n - 1) was stored: the parity tells the one phase between.)
                if (j == 0 || group_any(0, most_d > kGrow || most_v > 4.f * v_ref || !ok)) {
                    if (j > 0 && ok) ok = wait_all(&sh->pv_done, (n - 1) & 1, sh, p);
                    stop = group_any(0, !ok);
                    if (stop) break;
                    float y[kRows];
#pragma unroll
                    for (int c = 0; c < kPairs; ++c) {
                        y[2 * c] = x[0][c].x; y[2 * c + 1] = x[0][c].y;
                        if constexpr (kSub == 2) { y[2 * c] = fmaxf(y[2 * c], x[1][c].x); y[2 * c + 1] = fmaxf(y[2 * c + 1], x[1][c].y); }
                    }
                    const float most = warp_reduce(y, lane, [](float a, float b) { return fmaxf(a, b); });
#pragma unroll
                    for (int i = 16; i > 0; i >>= 1) most_v = fmaxf(most_v, __shfl_xor_sync(0xffffffffu, most_v, i));
                    float4 *red = sh->red[turn ^= 1];
                    if (lane < kRows) reinterpret_cast<float *>(red + lane)[quarter] = most;
                    if (lane == 0) reinterpret_cast<float *>(red + 16)[quarter] = most_v;
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
                    for (int i = 0; i < kSub; ++i)
#pragma unroll
                        for (int c = 0; c < kPairs; ++c) d[i][c] = __fadd2_rn(x[i][c], neg_m[c]);
                    if (j > 0) {
                        tc_fence_after();
#pragma unroll
                        for (int i = 0; i < C::kColsO; i += 16) {
                            uint32_t o[16];
                            tmem_ld16(tO + i, o);
#pragma unroll
                            for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * alpha[c % kRows]);
                            tmem_st16(tO + i, o);
                        }
                        tc_fence_before();
                    }
                } else if (j > 0) {
                    // P(n - 1) is read by its product until that is done.
                    if (!wait_all(&sh->pv_done, (n - 1) & 1, sh, p)) sh->abort_flag = 1;       // (voted on with the next step)
                }
                // p = 2^(x - m); the row's sum takes p itself, the product p sv / v_ref in four parts.
#pragma unroll
                for (int i = 0; i < kSub; ++i) {
                    const float f = vs[i] * v_factor;
#pragma unroll
                    for (int c = 0; c < kPairs; ++c) {
                        d[i][c] = make_float2(ex2(d[i][c].x), ex2(d[i][c].y));
                        l[c] = __fadd2_rn(l[c], d[i][c]);
                        d[i][c] = __fmul2_rn(d[i][c], make_float2(f, f));
                    }
                    if (border && !(f < INFINITY)) {       // a value that is not finite spoils no row that does not see it
#pragma unroll
                        for (int c = 0; c < kPairs; ++c) {
                            if (x[i][c].x == -INFINITY) d[i][c].x = 0.f;
                            if (x[i][c].y == -INFINITY) d[i][c].y = 0.f;
                        }
                    }
                    uint32_t parts[kRows / 4][4];
#pragma unroll
                    for (int c = 0; c < kRows / 4; ++c) split_e5m2(d[i][2 * c], d[i][2 * c + 1], parts[c]);
                    uint8_t *dst = p_row + i * kKeyTile * C::kPRow;
                    if constexpr (kRows == 4) {
                        *reinterpret_cast<uint4 *>(dst + p_swizzle) = make_uint4(parts[0][0], parts[0][1], parts[0][2], parts[0][3]);
                    } else if constexpr (kRows == 8) {
                        *reinterpret_cast<uint4 *>(dst + p_swizzle) = make_uint4(parts[0][0], parts[1][0], parts[0][1], parts[1][1]);
                        *reinterpret_cast<uint4 *>(dst + (16u ^ p_swizzle)) = make_uint4(parts[0][2], parts[1][2], parts[0][3], parts[1][3]);
                    } else {
#pragma unroll
                        for (uint32_t q = 0; q < 4; ++q)
                            *reinterpret_cast<uint4 *>(dst + ((q << 4) ^ p_swizzle)) = make_uint4(parts[0][q], parts[1][q], parts[2][q], parts[3][q]);
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->p_ready));
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
                const float out = f == 0.f ? 0.f : sum_o * f;
                if (s.whole && p.o_is_bf16) static_cast<__nv_bfloat16 *>(p.o)[to] = __float2bfloat16_rn(out);
                else (s.whole ? static_cast<float *>(p.o) : p.few_o)[to] = out;
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) tmem_dealloc(tmem, C::kTmemCols);
    // Beside the last CTAs of the kernel for many rows, which write other rows; but whoever waits for this kernel waits for that one.
    griddep_wait();
}

// Whether the scales of eight tokens can be loaded at once.
static bool by_eight(const uint16_t *s, int64_t sp, int64_t st, int64_t sh) { return st == 1 && sp % 8 == 0 && sh % 8 == 0 && reinterpret_cast<uintptr_t>(s) % 16 == 0; }

template <int kRows>
static cudaError_t launch(const Params &p, const CUtensorMap &tm_k, const CUtensorMap &tm_v, int box, bool after_many, cudaStream_t stream)
{
    return launch_dependent(paged_few_q4_kernel<kRows>, dim3((unsigned)p.few_ctas), kThreads, smem_bytes<kRows>(), stream, after_many, tm_k, tm_v, p, box,
                            by_eight(p.k_scales, p.ks_sp, p.ks_st, p.ks_sh) && by_eight(p.v_scales, p.vs_sp, p.vs_st, p.vs_sh), (int)test_skip_last_load());
}

template <int kRows>
static bool set_up()
{
    cudaFuncAttributes attr;
    return cudaFuncSetAttribute(paged_few_q4_kernel<kRows>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<kRows>()) == cudaSuccess &&
           cudaFuncGetAttributes(&attr, paged_few_q4_kernel<kRows>) == cudaSuccess && attr.numRegs * kThreads >= 128 * (kSoftmaxRegs + kLightRegs);
}

}  // namespace few_q4
}  // namespace paged

int launch_paged_few_q4(const paged::Params &p, bool after_many, cudaStream_t stream)
{
    using namespace paged;
    const int box = host_map::box_rows(p.c.page_size);
    CUtensorMap tm_k, tm_v;
    if (!host_map::pages_q4(&tm_k, p, p.k_pages, p.c.k_sp, p.c.k_st, p.c.k_sh, box, true) ||
        !host_map::pages_q4(&tm_v, p, p.v_pages, p.c.v_sp, p.c.v_st, p.c.v_sh, box, true)) {
        set_error("%s: cuTensorMapEncodeTiled failed (driver too old, or strides/addresses not encodable)", p.who);
        return PEC_ERR_CUDA;
    }
    static unsigned char ready[host::kMaxDevices] = {};
    static std::mutex ready_mutex;
    if (!host::once_per_device(ready, ready_mutex, [] { return few_q4::set_up<4>() && few_q4::set_up<8>() && few_q4::set_up<16>(); })) {
        (void)cudaGetLastError();
        set_error("%s: kernel set-up failed (shared-memory limit, or the register allocation does not cover the warp-role split)", p.who);
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
