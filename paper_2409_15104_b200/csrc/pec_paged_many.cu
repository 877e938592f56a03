// Paged attention of requests with many packed rows (prefill chunks) on the sm_100a tensor cores.
//
// Tensor-bound: 4 * 128 operations per visible (row, key) pair.  One CTA = one item of the plan: up to 256 packed rows (two
// stages of 128 / g whole tokens each) of one KV head against one slice of the request's keys.  Packing the heads of a KV group
// makes full tiles of short chunks and lets a key tile serve g heads.  The structure is that of the contiguous prefill kernel:
//   warps 0-3, 4-7  softmax and epilogue of stage 0 and 1 (a thread = a packed row = a TMEM lane)
//   warps 8, 10     MMA issuers of stage 0 and 1       warp 9  TMA loader       warp 11  idle (completes the warpgroup)
// One 128-column score buffer that both stages use in turns, a P region per stage, K and V tiles of 128 keys through a ring of
// four slots; per stage the issue order is S(j + 1), PV(j).  The tiles come page by page (see pec_paged_tma.cuh).
// TMEM columns: scores [0, 128); P_s [128 + 64 s, +64); O_s [256 + 128 s, +128).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include "pec_paged_tma.cuh"

namespace pec {
using namespace sm100;
namespace paged {
namespace many {

constexpr int kTile = 128;
constexpr int kSlots = 4;                                  // K/V ring
constexpr int kThreads = 384;
constexpr int kMmaWarp0 = 8, kLoadWarp = 9, kMmaWarp1 = 10;
constexpr int kLightRegs = 56, kSoftmaxRegs = 224;         // 256 * 224 + 128 * 56 = 384 * 168 (the launch allocation)
constexpr uint32_t kTmemCols = 512, kColS = 0, kColP = 128, kColO = 256;
constexpr float kRescaleThreshold = 8.0f;                  // log2 units

struct Geom {
    int32_t found;
    int32_t b, kv, key_lo, key_hi;
    int32_t tok_row;                                       // token row of the block's first token in q
    int32_t rows[2];                                       // valid packed rows per stage
    int32_t pos0[2];                                       // position of each stage's first token
    int32_t n[2], n_max;                                   // key tiles of each stage (a prefix of the CTA's walk)
    int32_t slices;
    int64_t slot;                                          // partial slot, where slices > 1
};
struct Shared {
    uint64_t bar_q[2];
    uint64_t kv_full[kSlots], kv_empty[kSlots];
    uint64_t s_full[2], s_taken[2], p_ready[2];            // [stage], one phase per key tile
    uint64_t pv_done[2];
    uint64_t drained[2];
    Geom g;
    uint32_t tmem_base;
    volatile int abort_flag;
};
constexpr size_t kSmemBytes = (2 + kSlots) * kTileBytes + 1024 /*alignment slack*/ + sizeof(Shared);

__device__ __forceinline__ bool wait_all(uint64_t *bar, uint32_t parity, Shared *sh, const Params &p)   // warp-uniform
{
    return __all_sync(0xffffffffu, mbar_wait_bounded(smem_u32(bar), parity, &sh->abort_flag, p.status, p.wait_cycles, (int)PEC_ERR_TIMEOUT));
}

__global__ void __launch_bounds__(kThreads, 1)
paged_many_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                  const __grid_constant__ CUtensorMap tm_v, const Params p, const int box, const int skip_last)
{
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t sQ = (raw + 1023u) & ~1023u, sRing = sQ + 2 * kTileBytes;
    Shared *sh = reinterpret_cast<Shared *>(smem_raw + (sQ - raw) + (2 + kSlots) * kTileBytes);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, kvh = blockIdx.x % p.Hkv;
    const int tps = kTile / p.g, srows = tps * p.g;        // tokens and packed rows of a stage

    // The loader warp reads the CTA's item, works out the geometry and starts the first loads (Q, K(0), V(0)) before the CTA-wide
    // sync; meanwhile others set up the remaining barriers and the tensor memory.
    const BoxLane bl = box_lane(box, lane);
    const BoxStep step = box_step(p.c.page_size);
    BoxPlace at = {0, 0};                                  // this lane's box of the next tile, and its page
    int32_t page = 0;
    bool found = false;
    // This lane's box (if it is one to load) of K (which = 0) or V into the ring's slot.
    auto load_tile = [&](int which, int slot, uint32_t bytes, bool mine) {
        const uint32_t bar = smem_u32(&sh->kv_full[slot]);
        if (lane == 0) mbar_arrive_expect_tx(bar, bytes);
        __syncwarp();
        if (mine)
            load_box(sRing + (uint32_t)slot * kTileBytes, which ? (const void *)&tm_v : (const void *)&tm_k, bar, bl, which ? p.fv : p.fk, kvh, at.row, page);
    };
    if (warp == kLoadWarp) {
        // The kernel for few rows may start on SMs that this grid leaves.  The plan has to be complete before its list is read.
        if (lane == 0) {
            griddep_launch_dependents();
            sh->abort_flag = 0;
            for (int st = 0; st < 2; ++st) mbar_init(smem_u32(&sh->bar_q[st]), 1);
            for (int s = 0; s < kSlots; ++s) { mbar_init(smem_u32(&sh->kv_full[s]), 1); mbar_init(smem_u32(&sh->kv_empty[s]), 2); }
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
            if (g.slices > 1 && g.slot >= p.many_cap) found = false;       // cannot happen (see the plan); never write past the scratch
        }
        g.found = found;
        if (lane == 0) {
            sh->g = g;
            // P is handed over by the warps that have rows only.  (Those without would run ahead: S(j + 1) may be complete before
            // P(j) is, and their arrivals for j + 1 would then complete phase j.)
            for (int st = 0; st < 2; ++st) mbar_init(smem_u32(&sh->p_ready[st]), g.rows[st] > 32 ? (uint32_t)(g.rows[st] + 31) / 32 : 1);
            mbar_init_fence();
        }
        __syncwarp();
        if (found && g.n_max > 0) {

            at = box_place(p.c.page_size, g.key_lo, bl);
            page = box_page(p, g.b, g.key_lo, g.kv, bl, at);
            if (lane == 0) {
                // The second stage's tokens may lie past the request's, or past q (zero fill): those rows are not used.
                for (int st = 0; st < 2; ++st) {
                    const uint32_t bar = smem_u32(&sh->bar_q[st]), dst = sQ + st * kTileBytes;
                    mbar_arrive_expect_tx(bar, (uint32_t)srows * 256u);
                    tma_load_4d(dst, &tm_q, bar, 0, 0, kvh, g.tok_row + st * tps);
                    tma_load_4d(dst + kHalfTileBytes, &tm_q, bar, 64, 0, kvh, g.tok_row + st * tps);
                }
            }
            const uint32_t bytes = tile_bytes(g.key_lo, g.kv, box);
            const bool mine = bl.used && g.key_lo + bl.first < g.kv;
            load_tile(0, 0, bytes, mine);
            load_tile(1, 1, bytes, mine);
            at = box_next(at, step);
            if (g.n_max > 1) page = box_page(p, g.b, g.key_lo + kTile, g.kv, bl, at);
        }
    } else if (tid == kMmaWarp0 * 32) {
        for (int st = 0; st < 2; ++st) {
            mbar_init(smem_u32(&sh->s_full[st]), 1);
            mbar_init(smem_u32(&sh->s_taken[st]), 4);      // one arrival per softmax warp
            mbar_init(smem_u32(&sh->pv_done[st]), 1);
            mbar_init(smem_u32(&sh->drained[st]), 1);
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

    if (warp == kLoadWarp) {
        // ------------------------------------------------------------------ TMA loader (one box per lane); tile 0 is under way
        reg_dealloc<kLightRegs>();
        if (n_max > 0) {
            const int32_t b = sh->g.b, kv = sh->g.kv;
            int32_t k0 = sh->g.key_lo + kTile;
            int issued = 2;
            bool ok = true;
            for (int j = 1; j < n_max && ok; ++j, k0 += kTile) {
                const BoxPlace at_next = box_next(at, step);
                const int32_t page_next = j + 1 < n_max ? box_page(p, b, k0 + kTile, kv, bl, at_next) : 0;
                const uint32_t bytes = tile_bytes(k0, kv, box);
                const bool mine = bl.used && k0 + bl.first < kv;
#pragma unroll
                for (int which = 0; which < 2; ++which) {  // K, V
                    const int item = 2 * j + which, slot = item % kSlots, fill = item / kSlots;
                    if (skip_last && item == 2 * n_max - 1) { ok = false; break; }   // test hook: the wait for it runs out
                    if (fill > 0) ok = wait_all(&sh->kv_empty[slot], (fill - 1) & 1, sh, p);
                    if (!ok) break;
                    load_tile(which, slot, bytes, mine);
                    ++issued;
                }
                page = page_next;
                at = at_next;
            }
            if (!ok && lane == 0) {
                // Given up: the copies under way must land before the CTA may leave.
                auto landed = [&](uint64_t *bar, uint32_t parity) { wait_quietly(bar, parity, p); };
                landed(&sh->bar_q[0], 0); landed(&sh->bar_q[1], 0);
                for (int i = issued > kSlots ? issued - kSlots : 0; i < issued; ++i) landed(&sh->kv_full[i % kSlots], (i / kSlots) & 1);
            }
        }
        __syncwarp();
    } else if (warp == kMmaWarp0 || warp == kMmaWarp1) {
        // ------------------------------------------------------------------ MMA issuers, one warp per stage
        reg_dealloc<kLightRegs>();
        if (n_max > 0) {
            const int st = (warp == kMmaWarp0) ? 0 : 1;
            const bool leader = elect_one();
            constexpr uint32_t idesc_qk = idesc_bf16_f32(kTile, kTile, 0, 0), idesc_pv = idesc_bf16_f32(kTile, kHeadDim, 0, 1);
            auto kv_wait = [&](int item) { return wait_all(&sh->kv_full[item % kSlots], (item / kSlots) & 1, sh, p); };
            auto kv_release = [&](int item) { if (leader) tc_commit(smem_u32(&sh->kv_empty[item % kSlots])); };
            const uint32_t tS = tmem + kColS, tP = tmem + kColP + st * 64, tO = tmem + kColO + st * kTile;
            uint64_t a_desc[8];
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
                a_desc[ks] = smem_desc_sw128(sQ + st * kTileBytes + (uint32_t)(ks >> 2) * kHalfTileBytes + (uint32_t)(ks & 3) * 32u, 16, 1024);
            const uint64_t k_ring = smem_desc_sw128(sRing, 16, kGroupBytes), v_ring = smem_desc_sw128(sRing, kGroupHalf, kGroupBytes);
            const int n_st = sh->g.n[st], n_ot = sh->g.n[st ^ 1];
            const int32_t key_lo = sh->g.key_lo, kv = sh->g.kv;
            auto issue_qk = [&](int j) {
                const uint64_t k0 = k_ring + (uint32_t)((((2 * j) % kSlots) * kTileBytes) >> 4);
                if (leader) mma_ss_k128_commit<(kGroupHalf >> 4)>(tS, a_desc, k0, idesc_qk, smem_u32(&sh->s_full[st]));
            };
            auto issue_pv = [&](int j) {
                const uint64_t v0 = v_ring + (uint32_t)((((2 * j + 1) % kSlots) * kTileBytes) >> 4);
                if (leader) {
                    mma_pv_k64(tO, tP, v0, idesc_pv, j > 0 ? 1u : 0u);
                    mma_pv_k64(tO, tP + 32, v0 + (8 * kGroupBytes >> 4), idesc_pv, 1u);
                    tc_commit(smem_u32(&sh->pv_done[st]));
                }
            };
            // The score buffer is used in the order (0,0), (1,0), (0,1), (1,1), ... (stage, tile), a stage that has run out of
            // tiles dropping out; S(j) may be issued once the previous user's softmax warps hold their scores.
            auto wait_buffer = [&](int j) {
                int pst, pj;
                if (st == 0) {
                    if (j == 0) return true;
                    pst = (j - 1 < n_ot) ? 1 : 0; pj = j - 1;
                } else {
                    if (j < n_ot) { pst = 0; pj = j; }
                    else if (j > 0) { pst = 1; pj = j - 1; }
                    else return true;
                }
                const bool got = wait_all(&sh->s_taken[pst], pj & 1, sh, p);
                if (got) tc_fence_after();
                return got;
            };

            bool ok = wait_all(&sh->bar_q[st], 0, sh, p) && kv_wait(0);
            if (ok) {
                if (n_st > 0) { ok = wait_buffer(0); if (ok) issue_qk(0); }
                kv_release(0);
            }
            for (int j = 0; j < n_max && ok; ++j) {
                if (j + 1 < n_max) {
                    ok = kv_wait(2 * j + 2);                       // K(j+1)
                    if (!ok) break;
                    if (j + 1 < n_st) {
                        ok = wait_buffer(j + 1);
                        if (!ok) break;
                        issue_qk(j + 1);
                    }
                    kv_release(2 * j + 2);
                }
                ok = kv_wait(2 * j + 1);                           // V(j)
                if (!ok) break;
                if (j < n_st) {
                    const int32_t valid = kv - key_lo - j * kTile;
                    // (both issuers write the same zeros; neither's product reads anything else there)
                    if (valid < kTile) clear_tail(sRing + (uint32_t)((2 * j + 1) % kSlots) * kTileBytes, valid, lane);
                    ok = wait_all(&sh->p_ready[st], j & 1, sh, p);
                    if (!ok) break;
                    tc_fence_after();
                    issue_pv(j);
                }
                kv_release(2 * j + 1);
            }
            if (!ok) drain_products(&sh->drained[st], leader, p);
        }
        __syncwarp();
    } else if (warp > kMmaWarp1) {
        reg_dealloc<kLightRegs>();
        // An earlier CTA's wait has run out: the launch is lost, every wait of this CTA gives up at its next try.
        if (lane == 0 && *reinterpret_cast<volatile int32_t *>(p.status) == PEC_ERR_TIMEOUT) sh->abort_flag = 1;
    } else {
        // ------------------------------------------------------------------ softmax + epilogue
        reg_alloc<kSoftmaxRegs>();
        const int st = warp >> 2, quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const uint32_t tS = tmem + lane_base + kColS;
        const uint32_t tP = tmem + lane_base + kColP + st * 64;
        const uint32_t tO = tmem + lane_base + kColO + st * kTile;
        const int n_t = sh->g.n[st], rows_valid = sh->g.rows[st] - quarter * 32;   // of this warp's 32 rows
        const bool works = rows_valid > 0;                 // a warp without rows only gives its share of the score buffer back
        const int32_t tok = row / p.g, head = row - tok * p.g;
        const int32_t pos0 = sh->g.pos0[st], my_pos = pos0 + tok, key_hi = sh->g.key_hi;
        const int32_t see_all = (p.causal && pos0 + 1 < key_hi) ? pos0 + 1 : key_hi;       // keys below it are visible to every row
        const int32_t see = (p.causal && my_pos + 1 < key_hi) ? my_pos + 1 : key_hi;       // ... to this row
        int32_t k0 = sh->g.key_lo;

        float m_ref = -INFINITY, l_run = 0.f;              // m_ref in log2 units of the scaled scores
        bool ok = true;
        for (int j = 0; j < n_t && ok; ++j, k0 += kTile) {
            ok = wait_all(&sh->s_full[st], j & 1, sh, p);
            if (!ok) break;
            uint32_t r[kTile];
            if (works) {
                tc_fence_after();
                tmem_ld128(tS, r);
                tc_fence_before();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->s_taken[st]));        // the buffer may take the other stage's next tile
            if (works) {
                if (k0 + kTile > see_all) {                // by choice, not by arithmetic: a masked score may be anything
                    int n_vis = see - k0;
                    n_vis = n_vis < 0 ? 0 : (n_vis > kTile ? kTile : n_vis);
#pragma unroll
                    for (int c = 0; c < kTile; ++c) r[c] = (c < n_vis) ? r[c] : 0xff800000u;
                }
                float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
#pragma unroll
                for (int c = 0; c < kTile; c += 8) {
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
                    alpha = ex2(m_ref - m_new);            // 0 when the row had no key so far
                    m_ref = m_new;
                    l_run *= alpha;
                }
                bool pv_waited = (j == 0);
                if (j > 0 && __any_sync(0xffffffffu, grow)) {
                    ok = wait_all(&sh->pv_done[st], (j - 1) & 1, sh, p);   // PV(j) needs this warp's P(j): the phase is unambiguous
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
                // p = 2^(s scale - m), rounded to bf16 as the product's operand; the row's sum takes p before it is rounded.  A second
                // part of p (as the form for at most 16 rows has) would be a third product for every two in a kernel that the tensor
                // pipe bounds, and 64 more columns for either stage of a tensor memory that is full: scores 128, P 2 x 64, O 2 x 128.
#pragma unroll
                for (int i = 0; i < kTile / 2; ++i) {
                    const float2 x = __ffma2_rn(make_float2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])), sc2, nm2);
                    const float2 e = make_float2(ex2(x.x), ex2(x.y));
                    sum[i & 3] = __fadd2_rn(sum[i & 3], e);
                    r[i] = pack_bf16(e.x, e.y);
                }
                const float2 s01 = __fadd2_rn(__fadd2_rn(sum[0], sum[1]), __fadd2_rn(sum[2], sum[3]));
                l_run += s01.x + s01.y;
                if (!pv_waited) {                          // P(j-1) is read by its product until that is done
                    ok = wait_all(&sh->pv_done[st], (j - 1) & 1, sh, p);
                    if (!ok) break;
                    tc_fence_after();
                }
                tmem_st32(tP, r);
                tmem_st32(tP + 32, r + 32);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->p_ready[st]));
            }
        }

        // Epilogue: O / l and LSE = ln2 * m + ln l; rows without any visible key give 0 and -inf.  A warp stages its rows in its
        // quarter of the stage's Q tile (no longer read: the stage's last product is done) and writes them out two rows per
        // instruction, 256 contiguous bytes each; where a row goes is fetched by shuffle from the lane that owns it.
        if (ok && works && n_t > 0) ok = wait_all(&sh->pv_done[st], (n_t - 1) & 1, sh, p);
        // A stage without keys never waited for its Q tile: the load must have landed before the tile is reused.  The other
        // stage's products do not read it.
        if (ok && n_t == 0 && n_max > 0) ok = wait_all(&sh->bar_q[st], 0, sh, p);
        if (ok && works) {
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
                    for (int i = 0; i < 64; ++i) f[i] = empty ? 0.f : __uint_as_float(r[i]) * inv;
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

}  // namespace many
}  // namespace paged

int launch_paged_many(const paged::Params &p, int64_t items, cudaStream_t stream)
{
    using namespace paged;
    const int box = host_map::box_rows(p.c.page_size);
    CUtensorMap tm_q, tm_k, tm_v;
    if (!host_map::queries(&tm_q, p, kFewRows / p.g) || !host_map::pages(&tm_k, p, p.k_pages, p.c.k_st, p.fk, box) ||
        !host_map::pages(&tm_v, p, p.v_pages, p.c.v_st, p.fv, box)) {
        set_error("pec_paged_attn: cuTensorMapEncodeTiled failed (driver too old, or strides/addresses not encodable)");
        return PEC_ERR_CUDA;
    }
    static unsigned char ready[host::kMaxDevices] = {};
    static std::mutex ready_mutex;
    if (!host::once_per_device(ready, ready_mutex, [] {
            cudaFuncAttributes attr;
            return cudaFuncSetAttribute(many::paged_many_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)many::kSmemBytes) == cudaSuccess &&
                   cudaFuncGetAttributes(&attr, many::paged_many_kernel) == cudaSuccess &&
                   attr.numRegs * many::kThreads >= 256 * many::kSoftmaxRegs + 128 * many::kLightRegs; })) {
        (void)cudaGetLastError();
        set_error("pec_paged_attn: kernel set-up failed (shared-memory limit, or the register allocation does not cover the warp-role split)");
        return PEC_ERR_CUDA;
    }
    if (items * p.Hkv > 0x7fffffff) { set_error("pec_paged_attn: grid too large"); return PEC_ERR_UNSUPPORTED; }
    cudaError_t err = launch_dependent(many::paged_many_kernel, dim3((unsigned)(items * p.Hkv)), many::kThreads, many::kSmemBytes, stream, true,
                                       tm_q, tm_k, tm_v, p, box, (int)test_skip_last_load());
    if (err == cudaSuccess) err = cudaGetLastError();
    if (err != cudaSuccess) { set_error("pec_paged_attn: launch failed: %s", cudaGetErrorString(err)); return PEC_ERR_CUDA; }
    return PEC_OK;
}

}  // namespace pec
