// Attention of a ragged batch over a KV cache in pages: prompts, and drafted tokens of many heads, on the 5th-generation tensor cores (sm_100a).
//
// A CTA of eight warps owns 128 rows of one (sequence, KV head): neighbouring tokens x the query heads of the group, token by token, so that keys and values are fetched once for the whole
// group and a few drafted tokens fill a tile.  The roles and their hand-over are those of the prefill over KV tiles (tgp_attn_sm100.cu):
//   warps 0-3  softmax: thread t is row t and TMEM lane t;
//   warp 4     issues S_j = Q K_j^T;  warp 6  issues O += P_j V_j;  warp 5  issues every TMA load;  warp 7  idle (completes the second warpgroup for setmaxnreg).
// K and V blocks of 64 keys arrive as pieces of up to 64 rows, none of which crosses a page; one tensor map covers all rows of the key pages and one all of the value pages, and
// a piece behind the sequence, or of a page that is none, is asked for outside the map, which fills it with zeros.  The table's entries are read 32 pieces at a time, a lane each,
// ahead of their loads.  Q is one box of [tokens][heads of the group][64].
// Which blocks are visited: those of the first `sinks` positions, then those from the first row's window to the last row's position; the mask is applied in blocks that some row does not see whole.
// A value that some rows see and others do not, and that is no number, would reach the others as 0 x inf: in such blocks it is put to zero in shared memory, and added at the
// end to the rows that see it.
// P is rounded to bf16 for the second product.  Every mbarrier wait is bounded; a wait that runs out sets an error word (tgp_k_attn_status), every role leaves its loop, loads in flight are waited for, TMEM
// is freed and nothing is stored.
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <algorithm>
#include <cfloat>
#include <cstdint>
#include "tgp.h"
#include "tgp_kernels.h"
#include "tgp_launch.cuh"
#include "tgp_sm100.cuh"
#include "tgp_attn_paged.cuh"

namespace {

using namespace tgp_sm100;
typedef __nv_bfloat16 bf16;
constexpr uint32_t BQ = 128, BKV = 64, THREADS = 256;

__device__ int g_attn_paged_error = 0;   // as g_attn_tc_error of the prefill over KV tiles

__device__ __forceinline__ void tma_load_3d(void *dst, const CUtensorMap *map, int x, int y, int z, uint64_t *bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar)) : "memory");
}

struct ManyArgs { TgpPagedAttn a; uint32_t tokens, piece; int none; };       // tokens of a CTA, rows of a piece, a row outside the maps

template <int DH>
__global__ void __launch_bounds__(THREADS, 2) tgp_attn_paged_many_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                                                                         const ManyArgs args) {
    extern __shared__ __align__(1024) uint8_t smem[];
    constexpr int KB = DH / 64;                          // 64-wide blocks of the head dimension
    constexpr uint32_t Q_BYTES = KB * BQ * 128, KV_BYTES = KB * BKV * 128;
    uint8_t *Qs = smem, *Ks = Qs + Q_BYTES, *Vs = Ks + 2 * KV_BYTES;                            // K and V: two stages each
    uint64_t *bar_k = reinterpret_cast<uint64_t *>(Vs + 2 * KV_BYTES);      // [2] K stage landed (stage 0's first use also carries Q)
    uint64_t *bar_v = bar_k + 2;                                       // [2] V stage landed
    uint64_t *bar_s = bar_v + 2;                                       // S complete in TMEM (tensor core)
    uint64_t *bar_sfree = bar_s + 1;                                   // all 128 rows of S are in registers
    uint64_t *bar_p = bar_sfree + 1;                                   // [2] all 128 rows of P_j (buffer j & 1) written, O rescaled where needed
    uint64_t *bar_o = bar_p + 2;                                       // [2] P V_j complete (tensor core): P buffer j & 1 and the V stage are free
    uint64_t *bar_kfree = bar_o + 2;                                   // [2] S_j complete: K stage j & 1 is free
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bar_kfree + 2);
    volatile uint32_t *failed = tmem_slot + 1;                         // [0] a wait ran out; [1] never set
    volatile uint32_t *odd = failed + 2;                               // a value that is no number was put to zero
    uint32_t *place = tmem_slot + 4;                                   // this CTA's sequence and tile
    const TgpPagedAttn &a = args.a;

    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (smem_u32(smem) & 1023u) {                            // the swizzle assumes 1024-byte aligned tiles
        if (tid == 0) atomicCAS(&g_attn_paged_error, 0, 5);
        return;
    }
    // Set-up and the TMEM allocation overlap the previous kernel, which wrote what is read below.
    if (warp == 5 && elect_one()) {
        mbar_init(bar_k, 1); mbar_init(bar_k + 1, 1); mbar_init(bar_v, 1); mbar_init(bar_v + 1, 1);
        mbar_init(bar_s, 1); mbar_init(bar_sfree, 128); mbar_init(bar_p, 128); mbar_init(bar_p + 1, 128); mbar_init(bar_o, 1); mbar_init(bar_o + 1, 1); mbar_init(bar_kfree, 1); mbar_init(bar_kfree + 1, 1);
        failed[0] = 0;
        failed[1] = 0;
        *odd = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmQ) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmK) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmV) : "memory");
    }
    if (warp == 4) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(256u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");     // not before the allocation: see tgp_sm100.cuh
    }
    if (warp == 7) {
        // ---- which tile: blockIdx.x counts the tiles of all sequences that are this kernel's, a sequence's last tile (the longest) first ----
        asm volatile("griddepcontrol.wait;" ::: "memory");
        uint32_t before = 0, b = 0xffffffffu, tile = 0;
        for (uint32_t i0 = 0; i0 < a.B && b == 0xffffffffu; i0 += 32) {
            const uint32_t i = i0 + lane;
            uint32_t mine = 0;
            if (i < a.B) {
                const TgpPagedSeq s = tgp_paged_seq(a, i);
                if (s.n && !s.idle && s.n * a.G > a.few) mine = (s.n + args.tokens - 1) / args.tokens;
            }
            uint32_t x = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const uint32_t y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
            const uint32_t hit = __ballot_sync(0xffffffffu, before + x > blockIdx.x);
            if (hit) {
                const int at = __ffs(hit) - 1;
                b = i0 + at;
                tile = before + __shfl_sync(0xffffffffu, x, at) - 1 - blockIdx.x;
            }
            before += __shfl_sync(0xffffffffu, x, 31);
        }
        if (lane == 0) { place[0] = b; place[1] = tile; }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = *tmem_slot;
    const uint32_t tmem_S = tmem_base, tmem_O = tmem_base + 64, tmem_P = tmem_base + 192;     // P: two buffers of 32 columns (bf16 pairs)
    const uint32_t b = place[0], hk = blockIdx.y;
    const bool live = b != 0xffffffffu;
    const TgpPagedSeq seq = live ? tgp_paged_seq(a, b) : TgpPagedSeq{0, 1, 1, false};
    const uint32_t t0 = place[1] * args.tokens, first_pos = seq.end - seq.n + t0, last_pos = min(first_pos + args.tokens, seq.end) - 1;      // tokens of the tile
    const uint32_t tokens = last_pos - first_pos + 1, rows = tokens * a.G;
    const TgpPagedKeys keys = tgp_paged_keys<BKV>(a, first_pos, last_pos);
    const uint32_t nblk = live ? keys.chunks : 0, pieces = BKV / args.piece;
    const int32_t *table = a.table + (size_t)(live ? b : 0) * a.W;
    auto page_at = [&](uint32_t key) { const uint32_t i = key / a.P; return i < a.W ? (uint32_t)table[i] : 0xffffffffu; };

    // is a page missing?  And rows behind the box's: zeros, so that they do not slow the softmax down
    bool missing = false;
    for (uint32_t i = tid; i < nblk * pieces; i += THREADS) {
        const uint32_t key = keys.chunk(i / pieces) * BKV + i % pieces * args.piece;
        missing |= key <= last_pos && page_at(key) >= a.n_pages;
    }
    for (uint32_t i = args.tokens * a.G * KB * 8 + tid; i < BQ * KB * 8; i += THREADS)
        *reinterpret_cast<uint4 *>(Qs + (i / 8 % KB) * (BQ * 128) + (i / (8 * KB)) * 128 + (i % 8) * 16) = make_uint4(0, 0, 0, 0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    missing = __syncthreads_or(missing);
    auto give_up = [&](int code) { if (!*failed) { *failed = 1; atomicCAS(&g_attn_paged_error, 0, code); } };
    // whole: every row sees every key of the block
    auto whole = [&](uint32_t key0) { return key0 + BKV - 1 <= first_pos && (!a.window || last_pos - key0 < a.window || key0 + BKV <= a.sinks); };
    // Registers move from the second warpgroup (three single-thread roles and an idle warp) to the softmax warpgroup:
    // 128 * 64 + 128 * 192 is the 128 per thread the CTA is launched with.
    if (warp >= 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;" ::: "memory");
        if (warp == 5 && nblk) {
            // ======================= TMA warp =======================
            // Two windows of 32 pieces each, a lane's piece in either: rows of the maps (args.none: zeros)
            uint32_t nk = 0, nv = 0, window = 0;                             // K and V blocks asked for; the first window, which V is in
            auto row_of = [&](uint32_t piece) {
                const uint32_t j = piece / pieces;
                if (j >= nblk) return args.none;
                const uint32_t key = keys.chunk(j) * BKV + piece % pieces * args.piece;
                if (key > last_pos) return args.none;
                const uint32_t page = page_at(key);
                return page < a.n_pages ? (int)((page * a.Hkv + hk) * a.P + key % a.P) : args.none;
            };
            int here = row_of(lane), there = row_of(32 + lane);
            auto load = [&](uint8_t *dst, const CUtensorMap *map, uint32_t j, uint64_t *bar, uint32_t more_bytes) {
                if (elect_one()) mbar_expect_tx(bar, KV_BYTES + more_bytes);
                for (uint32_t i = 0; i < pieces; ++i) {
                    const uint32_t p = j * pieces + i;
                    const int y = __shfl_sync(0xffffffffu, p / 32 == window ? here : there, p & 31);
                    if (elect_one())
#pragma unroll
                        for (uint32_t kb = 0; kb < KB; ++kb) tma_load_2d(dst + kb * (BKV * 128) + i * args.piece * 128, map, kb * 64, y, bar);
                }
            };
            auto next_k = [&](uint32_t more_bytes) { load(Ks + (nk & 1) * KV_BYTES, &tmK, nk, bar_k + (nk & 1), more_bytes); nk += 1; };
            auto next_v = [&]() {
                if (nv * pieces / 32 != window) { window += 1; here = there; there = row_of((window + 1) * 32 + lane); }
                load(Vs + (nv & 1) * KV_BYTES, &tmV, nv, bar_v + (nv & 1), 0);
                nv += 1;
            };
            next_k(KB * args.tokens * a.G * 128);                            // K_0 and, on the same barrier, Q
            if (elect_one())
#pragma unroll
                for (uint32_t kb = 0; kb < KB; ++kb) tma_load_3d(Qs + kb * (BQ * 128), &tmQ, kb * 64, hk * a.G, seq.first + t0, bar_k);
            if (1 < nblk) next_k(0);
            next_v();
            auto wait = [&](uint64_t *bar, uint32_t parity, int code) {
                const bool ok = mbar_wait(bar, parity, failed);
                if (!ok) give_up(code);
                return __all_sync(0xffffffffu, ok);
            };
            // test hook: the first CTA of the grid never loads this V block, so the wait for it runs out
            const uint32_t withhold = (blockIdx.x | blockIdx.y) == 0 ? (uint32_t)g_withhold_step : 0xffffffffu;
            for (uint32_t jb = 0; jb + 1 < nblk; ++jb) {
                const uint32_t st = jb & 1;
                if (jb + 1 == withhold) break;
                if (jb + 2 < nblk) {                                         // K_jb+2 goes where K_jb is, once S_jb is complete
                    if (!wait(bar_kfree + st, (jb >> 1) & 1, 1)) break;
                    next_k(0);
                }
                if (jb >= 1 && !wait(bar_o + (st ^ 1), ((jb - 1) >> 1) & 1, 2)) break;                 // V_jb+1 goes where V_jb-1 is
                next_v();
            }
            // every load asked for must have landed before the CTA may exit (bounded; `never` is never set)
            volatile uint32_t *never = failed + 1;
            for (uint32_t st = 0; st < 2; ++st) {
                const uint32_t ck = (nk + 1 - st) >> 1, cv = (nv + 1 - st) >> 1;     // loads asked for into this stage
                if (ck) mbar_wait(bar_k + st, (ck - 1) & 1, never);
                if (cv) mbar_wait(bar_v + st, (cv - 1) & 1, never);
            }
        } else if (warp == 4) {
            // ======================= S warp: one thread issues S_j = Q K_j^T =======================
            constexpr uint32_t idesc_s = umma_idesc(BKV);
            auto wait = [&](uint64_t *bar, uint32_t parity, int code) {
                bool ok = mbar_wait(bar, parity, failed);
                if (!ok) give_up(code);
                return __all_sync(0xffffffffu, ok);
            };
            for (uint32_t jb = 0; jb < nblk; ++jb) {
                if (jb >= 1 && !wait(bar_sfree, (jb - 1) & 1, 4)) break;         // S_jb-1 is in registers
                if (!wait(bar_k + (jb & 1), (jb >> 1) & 1, 3)) break;            // K_jb (and Q with K_0) has landed
                if (elect_one()) {
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint8_t *Kj = Ks + (jb & 1) * KV_BYTES;
#pragma unroll
                    for (uint32_t kb = 0; kb < KB; ++kb) {
                        const uint64_t dq = umma_desc(smem_u32(Qs + kb * (BQ * 128))), dk = umma_desc(smem_u32(Kj + kb * (BKV * 128)));
#pragma unroll
                        for (uint32_t k = 0; k < 4; ++k) umma(tmem_S, dq + 2 * k, dk + 2 * k, idesc_s, (kb | k) != 0);
                    }
                    umma_commit(bar_s);
                    umma_commit(bar_kfree + (jb & 1));                           // its completion also frees the K stage
                }
                __syncwarp();
            }
        } else if (warp == 6) {
            // ======================= P V warp: one thread issues O += P_j V_j =======================
            constexpr uint32_t idesc_o = umma_idesc(DH) | (1u << 16);           // bit 16: B operand is MN-major
            auto wait = [&](uint64_t *bar, uint32_t parity, int code) {
                bool ok = mbar_wait(bar, parity, failed);
                if (!ok) give_up(code);
                return __all_sync(0xffffffffu, ok);
            };
            for (uint32_t jb = 0; jb < nblk; ++jb) {
                const uint32_t st = jb & 1, key0 = keys.chunk(jb) * BKV;
                if (!wait(bar_v + st, (jb >> 1) & 1, 3)) break;
                if (!whole(key0)) {
                    // Values that no row sees, whatever the page holds there, are zeros; those that some rows see and that are no numbers too, and remembered.
                    for (uint32_t i = lane; i < BKV * KB * 8; i += 32) {
                        const uint32_t r = i / (KB * 8), kb = (i / 8) % KB, c = i % 8, key = key0 + r;
                        const bool none = key > last_pos || (a.window && key < keys.low && key >= a.sinks);
                        const bool every = key <= first_pos && (!a.window || last_pos - key < a.window || key < a.sinks);
                        if (every) continue;
                        uint4 *at = reinterpret_cast<uint4 *>(Vs + st * KV_BYTES + kb * (BKV * 128) + r * 128 + c * 16);
                        uint32_t w[4] = {0u, 0u, 0u, 0u};
                        if (!none) {
                            const uint4 v = *at;
                            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
                            bool found = false;
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if ((w[e] & 0x7f80u) == 0x7f80u) { w[e] &= 0xffff0000u; found = true; }
                                if ((w[e] & 0x7f800000u) == 0x7f800000u) { w[e] &= 0xffffu; found = true; }
                            }
                            if (!found) continue;
                            *odd = 1;
                        }
                        *at = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
                if (!wait(bar_p + st, (jb >> 1) & 1, 4)) break;
                if (elect_one()) {
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t dv = umma_desc_mn(smem_u32(Vs + st * KV_BYTES), BKV * 128);
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k)                             // 16 keys per step: 8 columns of P, 2048 B of V rows
                        umma_ts(tmem_O, tmem_P + st * 32 + 8 * k, dv + 128 * k, idesc_o, (jb | k) != 0);
                    umma_commit(bar_o + st);
                }
                __syncwarp();
            }
            __syncwarp();
            asm volatile("bar.arrive 1, 160;" ::: "memory");                 // `odd` is what it is going to be
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;" ::: "memory");
        // ======================= softmax warps: thread = row = TMEM lane =======================
        const uint32_t tok = tid / a.G;
        const bool row_ok = tid < rows;
        const uint32_t qpos = first_pos + min(tok, tokens - 1);              // padding rows take the last token's mask
        const uint32_t lane_addr = (warp * 32u) << 16;                       // this warp's quarter of the TMEM lanes
        float m_ref = -FLT_MAX, lrow = 0.f;                                  // exponent reference and running sum of this row
        auto wait = [&](uint64_t *bar, uint32_t parity, int code) {
            bool ok = mbar_wait(bar, parity, failed);
            if (!ok) give_up(code);
            return __all_sync(0xffffffffu, ok);
        };
        bool ok = true;
        for (uint32_t jb = 0; jb < nblk; ++jb) {
            const uint32_t key0 = keys.chunk(jb) * BKV;
            if (!(ok = wait(bar_s, jb & 1, 1))) break;
            float s[BKV];
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            tmem_ld64(tmem_S + lane_addr, s);
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            mbar_arrive(bar_sfree);
            if (!whole(key0)) {
                // hidden: behind the row, or before its window and none of the first positions
                const uint32_t low = a.window && qpos >= a.window ? qpos - a.window + 1 : 0;
#pragma unroll
                for (uint32_t i = 0; i < BKV; ++i)
                    if (key0 + i > qpos || (key0 + i < low && key0 + i >= a.sinks)) s[i] = -INFINITY;
            }
            if (missing) {
                uint32_t there = 0;                                          // a bit per 16 keys (no page begins inside them)
                for (uint32_t i = 0; i < 4; ++i) there |= (page_at(key0 + i * 16) < a.n_pages ? 1u : 0u) << i;
#pragma unroll
                for (uint32_t i = 0; i < BKV; ++i)
                    if (!(there >> (i / 16) & 1)) s[i] = -INFINITY;
            }
            auto row_max = [&]() {                                           // of the scaled scores (scale > 0: max commutes with it)
                float m0 = max3(s[0], s[1], s[2]), m1 = max3(s[3], s[4], s[5]);
#pragma unroll
                for (uint32_t i = 6; i + 3 < BKV; i += 4) { m0 = max3(m0, s[i], s[i + 1]); m1 = max3(m1, s[i + 2], s[i + 3]); }
                return max3(m0, m1, fmaxf(s[BKV - 2], s[BKV - 1])) * a.sl2;
            };
            uint32_t w[BKV / 2];
            auto exps = [&](float m) {                                       // w = exp2(S * scale - m) as bf16 pairs; returns their fp32 sum
                const uint64_t sc2 = pack2(a.sl2, a.sl2), nm2 = pack2(-m, -m);
                uint64_t acc0 = pack2(0.f, 0.f), acc1 = acc0;
#pragma unroll
                for (uint32_t i = 0; i < BKV / 2; ++i) {
                    float x0, x1;
                    unpack2(fma2(pack2(s[2 * i], s[2 * i + 1]), sc2, nm2), x0, x1);
                    const float p0 = ex2(x0), p1 = ex2(x1);                  // a masked score is -inf: p = 0
                    if (i & 1) acc1 = add2(acc1, pack2(p0, p1)); else acc0 = add2(acc0, pack2(p0, p1));
                    __nv_bfloat162 pk = __floats2bfloat162_rn(p0, p1);       // .x = p0 in the lower half
                    w[i] = *reinterpret_cast<uint32_t *>(&pk);
                }
                float l0, l1;
                unpack2(add2(acc0, acc1), l0, l1);
                return l0 + l1;
            };
            // The exponent reference m is the row max of block 0, moved only where a block's sum says that a score lies more than about 2^40 above it (or overflowed).  A row
            // that sees nothing of block 0 has the lowest finite reference: its sums are 0, and the first finite score takes the slow path.
            if (jb == 0) m_ref = fmaxf(row_max(), -FLT_MAX);
            float lblk = exps(m_ref);
            if (jb > 0 && __any_sync(0xffffffffu, !(lblk <= 0x1p40f))) {
                if (!(ok = wait(bar_o + ((jb - 1) & 1), ((jb - 1) >> 1) & 1, 2))) break;           // P V_{j-1}: nothing is accumulating into O
                const float m_new = fmaxf(m_ref, row_max()), alpha = ex2(m_ref - m_new);
                m_ref = m_new;
                lrow *= alpha;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                for (uint32_t h = 0; h < DH / 32; ++h) {
                    float v[32];
                    uint32_t u[32];
                    tmem_ld32(tmem_O + lane_addr + h * 32, v);
#pragma unroll
                    for (uint32_t i = 0; i < 32; ++i) u[i] = __float_as_uint(v[i] * alpha);
                    tmem_st32(tmem_O + lane_addr + h * 32, u);
                }
                lblk = exps(m_ref);
            }
            lrow += lblk;
            if (jb >= 2 && !(ok = wait(bar_o + (jb & 1), ((jb - 2) >> 1) & 1, 2))) break;      // P V_{j-2}: this P buffer is free
            tmem_st32(tmem_P + (jb & 1) * 32 + lane_addr, w);
            tmem_wait_st();
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            mbar_arrive(bar_p + (jb & 1));
        }
        // ---- the last P V; normalise and store this thread's row ----
        if (ok && nblk) ok = wait(bar_o + ((nblk - 1) & 1), ((nblk - 1) >> 1) & 1, 2);
        __syncwarp();
        asm volatile("bar.sync 1, 160;" ::: "memory");                       // (the P V warp has left its loop, too, however it went)
        if (ok && nblk) {
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const bool empty = lrow == 0.f;                                  // a row that sees nothing is zero
            const float inv = 1.0f / lrow;
            bf16 *dst = a.o + ((size_t)(seq.first + t0 + tok) * a.Hq + hk * a.G + (tid - tok * a.G)) * DH;
#pragma unroll
            for (uint32_t h = 0; h < DH / 32; ++h) {
                float v[32];
                __syncwarp();
                tmem_ld32(tmem_O + lane_addr + h * 32, v);
                if (*odd) {                                                  // keys that some rows see and others do not: what was put to zero
                    for (uint32_t jb = 0; jb < nblk; ++jb) {
                        const uint32_t key0 = keys.chunk(jb) * BKV;
                        if (whole(key0)) continue;
                        for (uint32_t key = key0; key < key0 + BKV && key <= qpos; ++key) {
                            const uint32_t page = page_at(key);
                            if (page >= a.n_pages || !tgp_paged_sees(a, qpos, key) || (key <= first_pos && (!a.window || last_pos - key < a.window || key < a.sinks))) continue;
                            const bf16 *from = a.v + (((size_t)page * a.Hkv + hk) * a.P + key % a.P) * DH + h * 32;
#pragma unroll
                            for (uint32_t i = 0; i < 32; ++i) {
                                const float x = __bfloat162float(from[i]);
                                if (!(fabsf(x) < INFINITY)) v[i] += x;
                            }
                        }
                    }
                }
#pragma unroll
                for (uint32_t c = 0; c < 4; ++c) {
                    uint32_t w[4];
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) {
                        __nv_bfloat162 pk = __floats2bfloat162_rn(v[c * 8 + 2 * i] * inv, v[c * 8 + 2 * i + 1] * inv);
                        w[i] = empty ? 0u : *reinterpret_cast<uint32_t *>(&pk);
                    }
                    if (row_ok) *reinterpret_cast<uint4 *>(dst + h * 32 + c * 8) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 4) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(256u) : "memory");
    }
}

template <int DH> constexpr int smem_bytes() { return (DH / 64) * (BQ + 4 * BKV) * 128 + 256; }

// bf16 map of [rows of a third dimension][heads][Dh] with boxes of [tokens][heads of a group][64] and the 128-byte swizzle
bool tensor_map_q(CUtensorMap *map, const void *base, uint64_t T, uint64_t Hq, uint64_t Dh, uint32_t G, uint32_t tokens) {
    PFN_cuTensorMapEncodeTiled_v12000 fn = tensor_map_encoder();
    if (!fn) return false;
    cuuint64_t dims[3] = {Dh, Hq, T}, strides[2] = {Dh * 2, Hq * Dh * 2};
    cuuint32_t box[3] = {64u, G, tokens}, estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DH>
int launch_many(const CUtensorMap &q, const CUtensorMap &k, const CUtensorMap &v, const ManyArgs &a, dim3 grid, cudaStream_t st) {
    if (!tgpk_allow_smem<tgp_attn_paged_many_kernel<DH>>(smem_bytes<DH>(), true)) return TGP_E_CUDA;
    return tgp_launch::launch(tgp_attn_paged_many_kernel<DH>, grid, dim3(THREADS), smem_bytes<DH>(), st, 1, q, k, v, a);
}

}  // namespace

int tgpk_attn_paged_many(const TgpPagedAttn &a, uint32_t Dh, cudaStream_t st) {
    ManyArgs args{a, BQ / a.G, BKV, 0};
    while (a.P % args.piece) args.piece /= 2;                                // (a page holds a multiple of 16 positions)
    const uint64_t rows = (uint64_t)a.n_pages * a.Hkv * a.P;
    args.none = (int)rows;
    CUtensorMap mq, mk, mv;
    if (!tensor_map_q(&mq, a.q, a.T, a.Hq, Dh, a.G, args.tokens) || !tensor_map_bf16_2d(&mk, a.k, rows, Dh, (uint64_t)Dh * 2, args.piece) ||
        !tensor_map_bf16_2d(&mv, a.v, rows, Dh, (uint64_t)Dh * 2, args.piece)) return TGP_E_CUDA;
    // tiles: of T rows, and one more for each sequence that this kernel has
    const uint32_t least = a.few / a.G + 1, tiles = a.T / args.tokens + std::min(a.B, a.T / least);
    if (a.Hkv > 65535) return TGP_E_TOO_LARGE;
    return Dh == 64 ? launch_many<64>(mq, mk, mv, args, dim3(tiles, a.Hkv), st) : launch_many<128>(mq, mk, mv, args, dim3(tiles, a.Hkv), st);
}

int tgpk_attn_paged_wait_test(unsigned long long limit_ns, int withhold_step) {
    if (cudaMemcpyToSymbol(g_wait_limit_ns, &limit_ns, sizeof(limit_ns)) != cudaSuccess) return TGP_E_CUDA;
    return cudaMemcpyToSymbol(g_withhold_step, &withhold_step, sizeof(withhold_step)) == cudaSuccess ? TGP_OK : TGP_E_CUDA;
}

int tgpk_attn_paged_status_clear() { const int z = 0; return cudaMemcpyToSymbol(g_attn_paged_error, &z, sizeof(z)) == cudaSuccess ? TGP_OK : TGP_E_CUDA; }
int tgpk_attn_paged_status(int *code) { return cudaMemcpyFromSymbol(code, g_attn_paged_error, sizeof(int)) == cudaSuccess ? TGP_OK : TGP_E_CUDA; }
