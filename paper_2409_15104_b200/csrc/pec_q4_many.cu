// Attention of bf16 queries with more than 16 packed rows over keys and values held in 4 bits, on the sm_100a tensor cores.
//
// Tensor-bound by its operations, 4 * 128 per visible (row, key) pair; in practice by 2^x of every pair (16 a cycle and SM).  One CTA =
// one item of the plan: up to 256 packed rows (two stages of 128 / g whole tokens each) of one KV head against one slice of the keys.
//   warps 0-3, 4-7  softmax and epilogue of stage 0 and 1 (a thread = a packed row = a TMEM lane)
//   warps 8, 10     MMA issuers of stage 0 and 1       warp 9  loader of Q and codes       warp 11  idle
//   warps 12-15     K and V: codes decoded into a ring of four tiles of 128 keys, 32 keys each
// Measured, 32 heads on 8: 2048 tokens on 30720 1120 us, 32 requests of 8 tokens and 4000 keys 145, one of 32 tokens and 60000 110.  What
// follows gives for each choice the first of these with it and without, everything else as it was at that time.
// The codes come ahead of their decoding, in a ring of their own: with 16 bytes a lane in flight instead few rows waited for memory (1261
// with it, 1323 without; 32 requests of 8 tokens 169 and 206).
// The tiles are decoded to fp16, to which the hardware converts codes (two an instruction).  fp16 has no range to hold scales, so what
// is multiplied is in units, powers of two that the other side makes up for:
//     K   of one for each 32 keys of a tile, such that scales are below 2^13 of it: a factor of those scores
//     V   of one for all, which moves when a tile's scales pass 2^13 of it: a factor of O
//     Q   of one for each row (its largest channel in [2^14, 2^15)), in place, before the first product
// A code times its scale has eight bits at most and is exact down to scales of 2^-30 (V: 2^-27) of the largest; below, the scale is a
// multiple of 2^-24 units, off by 2^-25, and the product by six times that at most: 6 * 2^-37 (V: 6 * 2^-34) of the largest scale.  A channel
// of Q is exact to 2^-31 of its row's largest, and off by 2^-39 of it below.  Probabilities are rounded to fp16, to 2^-11 of themselves: the largest of a row is held in [2^10, 2^15], and
// those below 2^-24 of it, in fp16's subnormals, are off by at most 2^-35 of it.
// Scores stay in tensor memory until probabilities take their place; S(j + 1) of a stage begins when PV(j) is done, some 2000 cycles in
// which the other stage has the unit of 2^x to itself: the stages take turns (1195 with, 1263 without) and hand P over by halves.  A
// row's 128 scores are in registers from its maximum on (1121; read a second time, by halves, 1195), which leaves the other warps 64.
// With the score buffer of the bf16 cache's kernel, one that both stages use in turns, and tiles decoded to bf16 it was 1493.
// A block that has rows for one stage only gives them to both, even tiles to one and odd tiles to the other, and merges what they have
// added up at its end (32 requests of 8 tokens 145 with, 169 without; one of 32 tokens and 60000 keys 110 and 119).
// TMEM columns: S_s [128 s, +128), P_s its first 64; O_s [256 + 128 s, +128).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include "pec_paged_tma.cuh"
#include "pec_q4.cuh"

namespace pec {
using namespace sm100;
namespace paged {
namespace many_q4 {

constexpr int kTile = 128;
constexpr int kSlots = 4;                                  // K/V ring
constexpr int kCodeSlots = 4;                              // ring of the tiles' codes
constexpr uint32_t kCodeBytes = kTile * q4::kHeadBytes;
constexpr int kMmaWarp0 = 8, kLoadWarp = 9, kMmaWarp1 = 10, kDecodeWarp = 12;
constexpr int kThreads = 512;
constexpr int kSoftmaxRegs = 192, kLightRegs = 64;         // 256 * 192 + 256 * 64 = 512 * 128 (the launch allocation)
constexpr uint32_t kTmemCols = 512, kColS = 0, kColO = 256;
// The largest probability of a row lies in [2^kLift, 2^(kLift + kGrow)].
constexpr float kLift = 10.f, kGrow = 5.f;

struct Geom {
    int32_t found;
    int32_t b, kv, key_lo, key_hi;
    int32_t tok_row;                                       // token row of the block's first token in q
    int32_t rows[2];                                       // valid packed rows per stage
    int32_t pos0[2];                                       // position of each stage's first token
    int32_t n[2], n_max;                                   // key tiles of each stage (a prefix of the CTA's walk)
    int32_t shared;                                        // both stages have the first one's rows: even tiles and odd ones
    int32_t slices;
    int64_t slot;                                          // partial slot, where slices > 1
};
struct Shared {
    uint64_t bar_q[2];
    uint64_t code_full[kCodeSlots], code_empty[kCodeSlots];
    uint64_t kv_full[kSlots], kv_empty[kSlots];
    uint64_t s_full[2], p_ready[2][2], pv_done[2];         // [stage], one phase per key tile; P by halves
    uint64_t drained[2];
    uint64_t turn[2][4];                                   // [stage][warp]: 2^x of a tile done
    uint64_t merged;                                       // (shared) the second stage's sums are complete
    uint64_t q_ready[2];                                   // [stage]: Q is in fp16
    struct { float4 k; float v; } unit[4];                 // of every fourth tile: K's for each 32 keys, V's
    float v_most[4];
    float v_units[4];
    float2 sums[kTile];                                    // (shared) of the second stage's rows: reference maximum, sum
    Geom g;
    uint32_t tmem_base;
    volatile int abort_flag;
};
constexpr size_t kSmemBytes = (2 + kSlots) * kTileBytes + kCodeSlots * kCodeBytes + 1024 /*alignment slack*/ + sizeof(Shared);
static_assert(kSmemBytes <= 227 * 1024, "");

__device__ __forceinline__ bool wait_all(uint64_t *bar, uint32_t parity, Shared *sh, const Params &p)   // warp-uniform
{
    return __all_sync(0xffffffffu, mbar_wait_bounded(smem_u32(bar), parity, &sh->abort_flag, p.status, p.wait_cycles, (int)PEC_ERR_TIMEOUT));
}

// A row of Q in its two swizzled half tiles, bf16 to fp16 in place, times a power of two that brings its largest channel to [2^14, 2^15)
// (at most 2^107; NaN for a row that is not finite), which is returned.
__device__ __forceinline__ float row_to_f16(uint8_t *at, int row)
{
    auto place = [&](int c) { return reinterpret_cast<uint4 *>(at + (c >> 3) * kHalfTileBytes + (((c ^ row) & 7) << 4)); };
    uint32_t most = 0;                                     // as whole numbers magnitudes compare as they do as numbers, NaN above all
#pragma unroll
    for (int c = 0; c < 16; ++c) {
        const uint4 u = *place(c);
        most = __vmaxu2(most, __vmaxu2(__vmaxu2(u.x & 0x7fff7fffu, u.y & 0x7fff7fffu), __vmaxu2(u.z & 0x7fff7fffu, u.w & 0x7fff7fffu)));
    }
    const uint32_t e = max(max(most & 0xffffu, most >> 16) >> 7, 34u);
    const float f = e == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float((268u - e) << 23);
#pragma unroll
    for (int c = 0; c < 16; ++c) {
        uint4 u = *place(c);
        uint32_t *w = &u.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_f16(__uint_as_float(w[i] << 16) * f, __uint_as_float(w[i] & 0xffff0000u) * f);
        *place(c) = u;
    }
    return f;
}

__global__ void __launch_bounds__(kThreads, 1)
paged_many_q4_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                     const Params p, const int box, const int skip_last)
{
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t sQ = (raw + 1023u) & ~1023u, sRing = sQ + 2 * kTileBytes, sCodes = sRing + kSlots * kTileBytes;
    Shared *sh = reinterpret_cast<Shared *>(smem_raw + (sQ - raw) + (2 + kSlots) * kTileBytes + kCodeSlots * kCodeBytes);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, kvh = blockIdx.x % p.Hkv;
    const int tps = kTile / p.g, srows = tps * p.g;        // tokens and packed rows of a stage

    // The loader warp reads the CTA's item, works out the geometry and starts the first loads (Q, codes of K(0), V(0)) before the CTA-wide
    // sync; meanwhile others set up the remaining barriers and the tensor memory.
    const BoxLane bl = box_lane(box, lane);
    const BoxStep box_by = box_step(p.c.page_size);
    BoxPlace box_at = {0, 0};                              // this lane's box of the next tile, and its page
    int32_t page = 0;
    bool found = false;
    // This lane's box (if it is one to load) of the codes of K (which = 0) or V of the tile at position k0.
    auto load_codes = [&](int which, int slot, int32_t k0, int32_t kv) {
        const uint32_t bar = smem_u32(&sh->code_full[slot]);
        if (lane == 0) mbar_arrive_expect_tx(bar, tile_bytes(k0, kv, box) / (2 * kHeadDim) * q4::kHeadBytes);
        __syncwarp();
        if (bl.used && k0 + bl.first < kv)
            tma_load_4d(sCodes + (uint32_t)slot * kCodeBytes + (uint32_t)bl.first * q4::kHeadBytes, which ? (const void *)&tm_v : (const void *)&tm_k, bar, 0, box_at.row, kvh, page);
    };
    if (warp == kLoadWarp) {
        // The kernel for few rows may start on SMs that this grid leaves.  The plan has to be complete before its list is read.
        if (lane == 0) {
            griddep_launch_dependents();
            sh->abort_flag = 0;
            for (int st = 0; st < 2; ++st) mbar_init(smem_u32(&sh->bar_q[st]), 1);
            for (int s = 0; s < kCodeSlots; ++s) { mbar_init(smem_u32(&sh->code_full[s]), 1); mbar_init(smem_u32(&sh->code_empty[s]), 4); }
            for (int s = 0; s < kSlots; ++s) { mbar_init(smem_u32(&sh->kv_full[s]), 4); mbar_init(smem_u32(&sh->kv_empty[s]), 2); }
        }
        griddep_wait();
        const Item it = p.many_items[blockIdx.x / p.Hkv];  // (inside the list's room, filled or not)
        found = (int)(blockIdx.x / p.Hkv) < p.many_count[0];
        Geom g = {};
        if (found) {
            const int32_t tok0 = it.block * 2 * tps;
            g.b = it.b; g.kv = it.r.kv; g.key_lo = it.key_lo; g.key_hi = it.key_hi;
            g.tok_row = it.r.start + tok0;
            g.slices = it.slices;
            g.slot = (int64_t)it.slot * p.Hkv + kvh;
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                int32_t nt = it.r.n - tok0 - st * tps;
                nt = nt < 0 ? 0 : (nt > tps ? tps : nt);
                g.rows[st] = nt * p.g;
                g.pos0[st] = it.r.pos0() + tok0 + st * tps;
                int32_t end = it.key_hi;
                if (p.causal && end > g.pos0[st] + nt) end = g.pos0[st] + nt;
                g.n[st] = (nt > 0 && end > it.key_lo) ? (end - it.key_lo + kTile - 1) / kTile : 0;
            }
            g.n_max = g.n[0] > g.n[1] ? g.n[0] : g.n[1];
            g.shared = g.rows[1] == 0 && g.n[0] > 1;
            if (g.shared) { g.rows[1] = g.rows[0]; g.pos0[1] = g.pos0[0]; g.n[1] = g.n[0]; }
            if (g.slices > 1 && g.slot >= p.many_cap) found = false;       // cannot happen (see the plan); never write past the scratch
        }
        g.found = found;
        if (lane == 0) {
            sh->g = g;
            // P is handed over by the warps that have rows only.
            for (int i = 0; i < 4; ++i) mbar_init(smem_u32(&sh->p_ready[i >> 1][i & 1]), g.rows[i >> 1] > 32 ? (uint32_t)(g.rows[i >> 1] + 31) / 32 : 1);
            mbar_init_fence();
        }
        __syncwarp();
        if (found && g.n_max > 0) {
            box_at = box_place(p.c.page_size, g.key_lo, bl);
            page = box_page(p, g.b, g.key_lo, g.kv, bl, box_at);
            if (lane == 0) {
                // The second stage's tokens may lie past the request's, or past q (zero fill): those rows are not used.
                for (int st = 0; st < 2; ++st) {
                    const uint32_t bar = smem_u32(&sh->bar_q[st]), dst = sQ + st * kTileBytes;
                    mbar_arrive_expect_tx(bar, (uint32_t)srows * 256u);
                    const int32_t row = g.tok_row + (g.shared ? 0 : st * tps);
                    tma_load_4d(dst, &tm_q, bar, 0, 0, kvh, row);
                    tma_load_4d(dst + kHalfTileBytes, &tm_q, bar, 64, 0, kvh, row);
                }
            }
            load_codes(0, 0, g.key_lo, g.kv);
            load_codes(1, 1, g.key_lo, g.kv);
            box_at = box_next(box_at, box_by);
            if (g.n_max > 1) page = box_page(p, g.b, g.key_lo + kTile, g.kv, bl, box_at);
        }
    } else if (tid == kMmaWarp0 * 32) {
        for (int st = 0; st < 2; ++st) {
            mbar_init(smem_u32(&sh->s_full[st]), 1);
            mbar_init(smem_u32(&sh->pv_done[st]), 1);
            mbar_init(smem_u32(&sh->drained[st]), 1);
            if (st == 0) mbar_init(smem_u32(&sh->merged), 4);
            for (int i = 0; i < 4; ++i) mbar_init(smem_u32(&sh->turn[st][i]), 1);
            mbar_init(smem_u32(&sh->q_ready[st]), 4);      // one arrival per softmax warp
        }
        mbar_init_fence();
        prefetch_tmap(&tm_q); prefetch_tmap(&tm_k); prefetch_tmap(&tm_v);
    } else if (warp == 4) {
        tmem_alloc(smem_u32(&sh->tmem_base), kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const int n_max = sh->g.n_max;
    const uint32_t tmem = sh->tmem_base;
    if (!sh->g.found) {
        if (warp == 4) tmem_dealloc(tmem, kTmemCols);
        return;
    }

    if (warp >= 8) reg_dealloc<kLightRegs>();
    if (warp == kLoadWarp) {
        // ------------------------------------------------------------------ loader of codes (one box per lane); tile 0 is under way
        if (n_max > 0) {
            const int32_t b = sh->g.b, kv = sh->g.kv;
            int32_t k0 = sh->g.key_lo + kTile;
            int issued = 2;
            bool ok = true;
            for (int j = 1; j < n_max && ok; ++j, k0 += kTile) {
                const BoxPlace at_next = box_next(box_at, box_by);
                const int32_t page_next = j + 1 < n_max ? box_page(p, b, k0 + kTile, kv, bl, at_next) : 0;
#pragma unroll
                for (int which = 0; which < 2; ++which) {  // K, V
                    const int item = 2 * j + which, slot = item % kCodeSlots, fill = item / kCodeSlots;
                    if (skip_last && item == 2 * n_max - 1) { ok = false; break; }   // test hook: the wait for it runs out
                    if (fill > 0) ok = wait_all(&sh->code_empty[slot], (fill - 1) & 1, sh, p);
                    if (!ok) break;
                    load_codes(which, slot, k0, kv);
                    ++issued;
                }
                page = page_next;
                box_at = at_next;
            }
            if (lane == 0) {
                // Copies must land before the CTA may leave; those that give up do not wait for them.
                wait_quietly(&sh->bar_q[0], 0, p); wait_quietly(&sh->bar_q[1], 0, p);
                for (int i = issued > kCodeSlots ? issued - kCodeSlots : 0; i < issued; ++i) wait_quietly(&sh->code_full[i % kCodeSlots], (i / kCodeSlots) & 1, p);
            }
        }
        __syncwarp();
    } else if (warp == kMmaWarp0 || warp == kMmaWarp1) {
        // ------------------------------------------------------------------ MMA issuers, one warp per stage
        if (n_max > 0) {
            const int st = (warp == kMmaWarp0) ? 0 : 1;
            const bool leader = elect_one();
            constexpr uint32_t idesc_qk = idesc_f16_f32(kTile, kTile, 0, 0);
            constexpr uint32_t idesc_pv = idesc_f16_f32(kTile, kHeadDim, 0, 1);
            auto kv_wait = [&](int item) { return wait_all(&sh->kv_full[item % kSlots], (item / kSlots) & 1, sh, p); };
            auto kv_release = [&](int item) { if (leader) tc_commit(smem_u32(&sh->kv_empty[item % kSlots])); };
            const uint32_t tS = tmem + kColS + st * kTile, tO = tmem + kColO + st * kTile;
            uint64_t a_desc[8];
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
                a_desc[ks] = smem_desc_sw128(sQ + st * kTileBytes + (uint32_t)(ks >> 2) * kHalfTileBytes + (uint32_t)(ks & 3) * 32u, 16, 1024);
            const uint64_t k_ring = smem_desc_sw128(sRing, 16, kGroupBytes), v_ring = smem_desc_sw128(sRing, kGroupHalf, kGroupBytes);
            const int n_st = sh->g.n[st], shared = sh->g.shared;
            auto issue_qk = [&](int j) {
                const uint64_t k0 = k_ring + (uint32_t)((((2 * j) % kSlots) * kTileBytes) >> 4);
                if (leader) mma_ss_k128_commit<(kGroupHalf >> 4)>(tS, a_desc, k0, idesc_qk, smem_u32(&sh->s_full[st]));
            };
            auto issue_pv = [&](int j, int m, int half) {
                const uint64_t v0 = v_ring + (uint32_t)((((2 * j + 1) % kSlots) * kTileBytes + half * 8 * kGroupBytes) >> 4);
                if (leader) {
                    mma_pv_k64(tO, tS + 32 * half, v0, idesc_pv, m > 0 || half ? 1u : 0u);
                    if (half) tc_commit(smem_u32(&sh->pv_done[st]));
                }
            };
            bool ok = wait_all(&sh->q_ready[st], 0, sh, p);
            int m = 0;                                             // this stage's tiles so far
            for (int j = 0; j < n_max && ok; ++j) {
                const bool mine = shared ? (j & 1) == st : j < n_st;
                ok = kv_wait(2 * j);                               // K(j)
                if (!ok) break;
                if (mine) {
                    // P(m - 1) lies where S(m) goes.  (Two products into different accumulators need not run in the order of their issue.)
                    if (m > 0) ok = wait_all(&sh->pv_done[st], (m - 1) & 1, sh, p);
                    if (!ok) break;
                    issue_qk(j);
                }
                kv_release(2 * j);
                ok = kv_wait(2 * j + 1);                           // V(j)
                if (!ok) break;
                if (mine) {
                    for (int half = 0; half < 2 && ok; ++half) {
                        ok = wait_all(&sh->p_ready[st][half], m & 1, sh, p);
                        if (!ok) break;
                        tc_fence_after();
                        issue_pv(j, m, half);
                    }
                    if (!ok) break;
                    ++m;
                }
                kv_release(2 * j + 1);
            }
            if (!ok) drain_products(&sh->drained[st], leader, p);
        }
        __syncwarp();
    } else if (warp >= kDecodeWarp) {
        // ------------------------------------------------------------------ tiles of a cache held in 4 bits
        // This warp: keys 32 w .. + 31 of each tile, eight at a time; a lane has 32 channels of one of the eight.  The scale of key 32 w + i is
        // loaded by lane i, two tiles ahead, the number of its page three, and looked at a tile later: nothing here waits for memory.
        const int w = warp - kDecodeWarp, row8 = lane >> 2, quarter = lane & 3;
        const int32_t b = sh->g.b, kv = sh->g.kv, key_lo = sh->g.key_lo;
        const BoxLane own = {32 * w + lane, 0u, true};
        const BoxStep step = box_step(p.c.page_size);
        BoxPlace at = box_place(p.c.page_size, key_lo, own);
        auto valid = [&](int j) { return j < n_max && key_lo + j * kTile + own.first < kv; };
        auto look_up = [&](int j) { return valid(j) ? __ldg(p.c.table + b * p.c.table_stride + at.nth) : 0; };
        const uint16_t *k_scales = p.k_scales + kvh * p.ks_sh, *v_scales = p.v_scales + kvh * p.vs_sh;
        struct Scales { uint32_t k, v; };                  // (keys past the end: 0, so that nothing there meets a product)
        auto fetch = [&](int j, int32_t pg, int32_t row) {
            if (!valid(j)) return Scales{0u, 0u};
            if (pg < 0 || pg >= p.c.num_pages) { raise_status(p.status, PEC_ERR_BAD_INDEX); pg = 0; }
            return Scales{__ldg(k_scales + pg * p.ks_sp + row * p.ks_st), __ldg(v_scales + pg * p.vs_sp + row * p.vs_st)};
        };
        // A lane's place in the group of eight keys: its half of the channels, and from which chunk of 16 bytes on.  Lanes of either half
        // store their four chunks in another order, which keeps eight lanes out of one another's banks.
        const uint32_t to = (uint32_t)(quarter >> 1) * kGroupHalf + (uint32_t)row8 * 128u, chunk = (uint32_t)(quarter & 1) * 4u, turned = (uint32_t)(quarter >> 1) * 2u;
        const uint32_t from = sCodes + (uint32_t)(32 * w + row8) * q4::kHeadBytes + (uint32_t)quarter * 16u;
        bool ok = true;
        // K (which = 0) or V of tile j into the ring in units of 1 / inverse.
        auto decode = [&](int j, int which, uint32_t scales, float inverse) {
            const int item = 2 * j + which, slot = item % kSlots, fill = item / kSlots, code_slot = item % kCodeSlots;
            ok = wait_all(&sh->code_full[code_slot], (item / kCodeSlots) & 1, sh, p);
            if (!ok) return;
            uint4 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[i].x), "=r"(x[i].y), "=r"(x[i].z), "=r"(x[i].w)
                             : "r"(from + (uint32_t)code_slot * kCodeBytes + (uint32_t)i * 8u * q4::kHeadBytes) : "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->code_empty[code_slot]));
            if (fill > 0) ok = wait_all(&sh->kv_empty[slot], (fill - 1) & 1, sh, p);
            if (!ok) return;
            const uint32_t dst = sRing + (uint32_t)slot * kTileBytes + (uint32_t)w * 4u * kGroupBytes + to;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t bits = __shfl_sync(0xffffffffu, scales, 8 * i + row8);
                const __half2 s2 = __float2half2_rn(__uint_as_float(bits << 16) * inverse);
                const uint32_t words[4] = {turned ? x[i].z : x[i].x, turned ? x[i].w : x[i].y, turned ? x[i].x : x[i].z, turned ? x[i].y : x[i].w};
#pragma unroll
                for (uint32_t c = 0; c < 4; ++c) {
                    uint32_t r[4];
                    q4::decode8_f16(words[c], s2, r);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                                 ::"r"(dst + (uint32_t)i * kGroupBytes + (((chunk + (c ^ turned)) ^ (uint32_t)row8) << 4)), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->kv_full[slot]));
        };
        // The largest of the warp's scales (bf16 bits; NaN left out).
        auto most_of = [&](uint32_t x) { return __uint_as_float(__reduce_max_sync(0xffffffffu, x > 0x7f80u ? 0u : x) << 16); };
        // m's power of two or the next, times 2^less: what brings scales up to m below 2^-less.
        auto unit_of = [](float m, int less) { return __uint_as_float((__float_as_uint(fmaxf(m, 0x1p-100f)) & 0x7f800000u) + ((uint32_t)(1 + less) << 23)); };
        auto inverse_of = [](float power) { return __uint_as_float((254u << 23) - __float_as_uint(power)); };
        const int32_t page0 = look_up(0), row0 = at.row;   // (the first three at once)
        at = box_next(at, step);
        const int32_t page1 = look_up(1), row1 = at.row;
        at = box_next(at, step);
        int32_t raw_page = look_up(2);                     // of the tile that `at` is at
        Scales now = fetch(0, page0, row0), next = fetch(1, page1, row1);
        float v_unit = 0.f;
        for (int j = 0; j < n_max; ++j) {
            const Scales after = fetch(j + 2, raw_page, at.row);
            at = box_next(at, step);
            raw_page = look_up(j + 3);
            // The four warps go on, and move V's unit, by common votes alone.
            const float k_unit = unit_of(most_of(now.k), -13), v_most = most_of(now.v);
            if (group_any(0, v_most >= 0x1p13f * v_unit || !ok)) {
                if (group_any(0, !ok)) break;
                if (lane == 0) sh->v_most[w] = v_most;
                group_any(0, false);
                v_unit = unit_of(fmaxf(fmaxf(sh->v_most[0], sh->v_most[1]), fmaxf(sh->v_most[2], sh->v_most[3])), -10);
                group_any(0, false);
            }
            // (V of three tiles ago is in the ring, so its product before is done and the softmax through with that tile's units.)
            if (lane == 0) {
                reinterpret_cast<float *>(&sh->unit[j & 3].k)[w] = k_unit;
                if (w == 0) sh->unit[j & 3].v = v_unit;
            }
            __syncwarp();
            decode(j, 0, now.k, inverse_of(k_unit));
            if (ok) decode(j, 1, now.v, inverse_of(v_unit));
            now = next;
            next = after;
        }
        __syncwarp();
    } else if (warp > kMmaWarp1) {
        // An earlier CTA's wait has run out: the launch is lost, every wait of this CTA gives up at its next try.
        if (lane == 0 && *reinterpret_cast<volatile int32_t *>(p.status) == PEC_ERR_TIMEOUT) sh->abort_flag = 1;
    } else {
        // ------------------------------------------------------------------ softmax + epilogue
        reg_alloc<kSoftmaxRegs>();
        const int st = warp >> 2, quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const uint32_t tS = tmem + lane_base + kColS + st * kTile;
        const uint32_t tO = tmem + lane_base + kColO + st * kTile;
        const int shared = sh->g.shared, n_all = sh->g.n[st];
        const int n_t = shared ? (n_all + 1 - st) / 2 : n_all, rows_valid = sh->g.rows[st] - quarter * 32;   // of this warp's 32 rows
        const bool works = rows_valid > 0;                 // a warp without rows only gives its share of the score buffer back
        const int32_t tok = row / p.g, head = row - tok * p.g;
        const int32_t pos0 = sh->g.pos0[st], my_pos = pos0 + tok, key_hi = sh->g.key_hi;
        const int32_t see_all = (p.causal && pos0 + 1 < key_hi) ? pos0 + 1 : key_hi;       // keys below it are visible to every row
        const int32_t see = (p.causal && my_pos + 1 < key_hi) ? my_pos + 1 : key_hi;       // ... to this row
        int32_t k0 = sh->g.key_lo + (shared ? st * kTile : 0);
        const int n_other = shared ? (n_all + st) / 2 : sh->g.n[st ^ 1];       // of the other stage
        const bool paired = sh->g.rows[st ^ 1] > quarter * 32;

        float m_ref = -INFINITY, l_run = 0.f;              // log2 units; a probability of 1 is 2^kLift at least
        float row_scale = 0.f, v_unit = 1.f;               // log2 units of a score over its product's; what O is in units of
        bool ok = n_max > 0 ? wait_all(&sh->bar_q[st], 0, sh, p) : true;
        if (ok && n_max > 0) {
            row_scale = p.scale_log2 / row_to_f16(smem_raw + (sQ - raw) + st * kTileBytes + row * 128, row);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->q_ready[st]));
        }
        for (int j = 0; j < n_t && ok && works; ++j, k0 += shared ? 2 * kTile : kTile) {      // this stage's tiles
            ok = wait_all(&sh->s_full[st], j & 1, sh, p);  // (PV(j - 1) is done as well)
            if (!ok) break;
            tc_fence_after();
            const int tile = shared ? 2 * j + st : j;
            const float4 k_unit = sh->unit[tile & 3].k;
            const float v_now = sh->unit[tile & 3].v;
            // (never 0, by which a masked score would be NaN)
            const float factor[4] = {fmaxf(row_scale * k_unit.x, 0x1p-126f), fmaxf(row_scale * k_unit.y, 0x1p-126f),
                                     fmaxf(row_scale * k_unit.z, 0x1p-126f), fmaxf(row_scale * k_unit.w, 0x1p-126f)};
            const bool masked = k0 + kTile > see_all;
            int n_vis = see - k0;
            n_vis = n_vis < 0 ? 0 : (n_vis > kTile ? kTile : n_vis);
            uint32_t r[kTile];
            tmem_ld128(tS, r);
            if (masked) {                                  // by choice, not by arithmetic: a masked score may be anything
#pragma unroll
                for (int c = 0; c < kTile; ++c) r[c] = c < n_vis ? r[c] : 0xff800000u;
            }
            float top[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll
                for (int c = 32 * q; c < 32 * q + 32; c += 4) {
                    m0 = fmax3(m0, __uint_as_float(r[c]), __uint_as_float(r[c + 1]));
                    m1 = fmax3(m1, __uint_as_float(r[c + 2]), __uint_as_float(r[c + 3]));
                }
                top[q] = fmaxf(m0, m1) * factor[q];
            }
            const float m_new = fmax3(top[0], top[1], fmaxf(top[2], top[3]));
            float alpha = 1.f;
            bool grow = m_new > m_ref + (kLift + kGrow);
            if (grow) {
                const float m_old = m_ref;
                m_ref = m_new - kLift;
                alpha = ex2(m_old - m_ref);                // 0 when the row had no key so far
                l_run *= alpha;
            }
            if (v_now != v_unit) { alpha *= v_unit / v_now; grow = true; v_unit = v_now; }
            if (j > 0 && __any_sync(0xffffffffu, grow)) {
                const float2 a2 = make_float2(alpha, alpha);
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t o[32];
                    tmem_ld32(tO + c * 32, o);
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        const float2 x = __fmul2_rn(make_float2(__uint_as_float(o[i]), __uint_as_float(o[i + 1])), a2);
                        o[i] = __float_as_uint(x.x); o[i + 1] = __float_as_uint(x.y);
                    }
                    tmem_st32(tO + c * 32, o);
                }
            }
            const float neg_m = (m_ref == -INFINITY) ? 0.f : -m_ref;
            const float2 nm2 = make_float2(neg_m, neg_m);
            float2 sum[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = make_float2(0.f, 0.f);
            // The two stages' warps of a scheduler take turns here (one waits for its products while the other has the unit of 2^x).
            if (paired && j - (st ^ 1) >= 0 && j - (st ^ 1) < n_other) {
                ok = wait_all(&sh->turn[st ^ 1][quarter], (j - (st ^ 1)) & 1, sh, p);
                if (!ok) break;
            }
            // p = 2^(s - m), rounded to fp16 as the product's operand; the row's sum takes p before it is rounded.
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const float f = factor[2 * half + (i >> 4)];
                    const float2 x = __ffma2_rn(make_float2(__uint_as_float(r[64 * half + 2 * i]), __uint_as_float(r[64 * half + 2 * i + 1])), make_float2(f, f), nm2);
                    const float2 e = make_float2(ex2(x.x), ex2(x.y));
                    sum[i & 3] = __fadd2_rn(sum[i & 3], e);
                    r[64 * half + i] = pack_f16(e.x, e.y);
                }
                if (half && lane == 0) mbar_arrive(smem_u32(&sh->turn[st][quarter]));
                tmem_st32(tS + half * 32, r + 64 * half);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->p_ready[st][half]));
            }
            const float2 s01 = __fadd2_rn(__fadd2_rn(sum[0], sum[1]), __fadd2_rn(sum[2], sum[3]));
            l_run += s01.x + s01.y;
        }

        // Epilogue: O / l and LSE = ln2 * m + ln l; rows without any visible key give 0 and -inf.  A warp stages its rows in its
        // quarter of the stage's Q tile (no longer read: the stage's last product is done) and writes them out two rows per
        // instruction, 256 contiguous bytes each; where a row goes is fetched by shuffle from the lane that owns it.
        if (ok && works && n_t > 0) ok = wait_all(&sh->pv_done[st], (n_t - 1) & 1, sh, p);
        // A stage without keys has no product to wait for: its four warps must be done with their rows of Q, which lie in one another's
        // quarters, before any of them reuses the tile.  The other stage's products do not read it.
        if (ok && n_t == 0 && n_max > 0) ok = wait_all(&sh->q_ready[st], 0, sh, p);
        // Stages that share rows: the first one writes them, with what the second has added up.
        float mine = v_unit, others = 0.f;                 // what either stage's O counts
        if (shared && st == 1) {
            sh->sums[row] = make_float2(m_ref, l_run);
            sh->v_units[row >> 5] = v_unit;
            __syncwarp();
            if (ok && lane == 0) mbar_arrive(smem_u32(&sh->merged));
        }
        if (shared && st == 0 && ok) {
            ok = wait_all(&sh->merged, 0, sh, p) && wait_all(&sh->pv_done[1], (n_other - 1) & 1, sh, p);
            const float2 o = sh->sums[row];
            const float top = fmaxf(m_ref, o.x), base = top == -INFINITY ? 0.f : top, a = ex2(m_ref - base), b = ex2(o.x - base);
            mine *= a;
            others = sh->v_units[row >> 5] * b;
            l_run = l_run * a + o.y * b;
            m_ref = top;
        }
        if (ok && works && !(shared && st == 1)) {
            tc_fence_after();
            const bool empty = (l_run == 0.f);
            const float inv = empty ? 0.f : 1.f / l_run;
            const bool whole = sh->g.slices <= 1;
            const int64_t at = whole ? (int64_t)(sh->g.tok_row + st * tps + tok) * p.Hq + kvh * p.g + head
                                     : sh->g.slot * p.many_rows + st * srows + row;
            const bool bf16_out = whole && p.o_is_bf16;
            float *out_f = whole ? static_cast<float *>(p.o) : p.many_o;
            const int sub = lane >> 4, chunk = lane & 15;
            uint8_t *stage_buf = smem_raw + (sQ - raw) + st * kTileBytes + quarter * 8192;
            uint8_t *my_row = stage_buf + lane * 256;
            const int passes = bf16_out ? 1 : 2;           // a row is 256 bytes of bf16, or two halves of 256 bytes of fp32
#pragma unroll 1
            for (int pass = 0; pass < passes; ++pass) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if (!bf16_out && half) break;
                    uint32_t r[64];
                    if (n_t == 0) {
#pragma unroll
                        for (int i = 0; i < 64; ++i) r[i] = 0u;
                    } else {
                        tmem_ld64(tO + (bf16_out ? half : pass) * 64, r);
                    }
                    float f[64];
#pragma unroll
                    for (int i = 0; i < 64; ++i) f[i] = empty ? 0.f : __uint_as_float(r[i]) * inv * mine;
                    if (shared) {
                        tmem_ld64(tmem + lane_base + kColO + kTile + (bf16_out ? half : pass) * 64, r);
#pragma unroll
                        for (int i = 0; i < 64; ++i) f[i] = empty ? 0.f : fmaf(__uint_as_float(r[i]) * inv, others, f[i]);
                    }
                    if (bf16_out) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            *reinterpret_cast<uint4 *>(my_row + (((half * 8 + i) ^ (lane & 15)) << 4)) =
                                make_uint4(pack_bf16(f[8 * i], f[8 * i + 1]), pack_bf16(f[8 * i + 2], f[8 * i + 3]),
                                           pack_bf16(f[8 * i + 4], f[8 * i + 5]), pack_bf16(f[8 * i + 6], f[8 * i + 7]));
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            *reinterpret_cast<float4 *>(my_row + ((i ^ (lane & 15)) << 4)) = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
                    }
                }
                __syncwarp();
                uint4 val[16];
#pragma unroll
                for (int rr = 0; rr < 16; ++rr) {
                    const int x = 2 * rr + sub;
                    val[rr] = *reinterpret_cast<const uint4 *>(stage_buf + x * 256 + ((chunk ^ (x & 15)) << 4));
                }
#pragma unroll
                for (int rr = 0; rr < 16; ++rr) {
                    const int x = 2 * rr + sub;
                    const int64_t to = __shfl_sync(0xffffffffu, at, x);
                    if (x < rows_valid) {
                        uint8_t *dst = bf16_out ? static_cast<uint8_t *>(p.o) + to * 256 + chunk * 16
                                                : reinterpret_cast<uint8_t *>(out_f + to * kHeadDim + pass * 64) + chunk * 16;
                        *reinterpret_cast<uint4 *>(dst) = val[rr];
                    }
                }
                __syncwarp();
            }
            if (lane < rows_valid) (whole ? p.lse : p.many_lse)[at] = empty ? -INFINITY : m_ref * 0.6931471805599453f + logf(l_run);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 4) tmem_dealloc(tmem, kTmemCols);
}

}  // namespace many_q4
}  // namespace paged

int launch_paged_many_q4(const paged::Params &p, int64_t items, cudaStream_t stream)
{
    using namespace paged;
    const int box = host_map::box_rows(p.c.page_size);
    CUtensorMap tm_q, tm_k, tm_v;
    if (!host_map::queries(&tm_q, p, kFewRows / p.g) || !host_map::pages_q4(&tm_k, p, p.k_pages, p.c.k_sp, p.c.k_st, p.c.k_sh, box, false) ||
        !host_map::pages_q4(&tm_v, p, p.v_pages, p.c.v_sp, p.c.v_st, p.c.v_sh, box, false)) {
        set_error("%s: cuTensorMapEncodeTiled failed (driver too old, or strides/addresses not encodable)", p.who);
        return PEC_ERR_CUDA;
    }
    static unsigned char ready[host::kMaxDevices] = {};
    static std::mutex ready_mutex;
    if (!host::once_per_device(ready, ready_mutex, [] {
            cudaFuncAttributes attr;
            return cudaFuncSetAttribute(many_q4::paged_many_q4_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)many_q4::kSmemBytes) == cudaSuccess &&
                   cudaFuncGetAttributes(&attr, many_q4::paged_many_q4_kernel) == cudaSuccess &&
                   attr.numRegs * many_q4::kThreads >= 256 * many_q4::kSoftmaxRegs + (many_q4::kThreads - 256) * many_q4::kLightRegs; })) {
        (void)cudaGetLastError();
        set_error("%s: kernel set-up failed (shared-memory limit, or the register allocation does not cover the warp-role split)", p.who);
        return PEC_ERR_CUDA;
    }
    if (items * p.Hkv > 0x7fffffff) { set_error("%s: grid too large", p.who); return PEC_ERR_UNSUPPORTED; }
    cudaError_t err = launch_dependent(many_q4::paged_many_q4_kernel, dim3((unsigned)(items * p.Hkv)), many_q4::kThreads, many_q4::kSmemBytes, stream, true,
                                       tm_q, tm_k, tm_v, p, box, (int)test_skip_last_load());
    if (err == cudaSuccess) err = cudaGetLastError();
    if (err != cudaSuccess) { set_error("%s: launch failed: %s", p.who, cudaGetErrorString(err)); return PEC_ERR_CUDA; }
    return PEC_OK;
}

}  // namespace pec
