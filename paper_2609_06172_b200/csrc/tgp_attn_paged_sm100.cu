// Attention of a ragged batch over a KV cache in pages: prompts, and drafted tokens of many heads, on the 5th-generation tensor cores (sm_100a).
//
// A CTA of eight warps owns 128 rows of one (sequence, KV head): neighbouring tokens x the query heads of the group, token by token, so that keys and values are fetched once for the whole
// group and a few drafted tokens fill a tile.  CTAs stay, two to an SM, and take tiles as they become free:
//   warps 0-3  softmax: thread t is row t and TMEM lane t;  the store of O;
//   warp 4     issues S_j = Q K_j^T;  warp 6  issues O += P_j V_j, and sees to the values that not every row sees;  warp 5  issues every TMA load;
//   warp 7     finds the next tiles, up to four ahead: the first is the CTA's own, further ones are numbered by a counter.
// S has two buffers of 64 columns, and P_j, in bf16, takes the place of the first half of S_j: so S_j+1 is multiplied while S_j is exponentiated and P_j-1 V_j-1 added up.
// K and V blocks of 64 keys arrive as pieces of up to 64 rows, none of which crosses a page; one tensor map covers all rows of the key pages and one all of the value pages, and
// a piece behind the sequence, or of a page that is none, is asked for outside the map, which fills it with zeros.  The table's entries are read 32 pieces at a time, a lane each,
// ahead of their loads.  Q is one box of [tokens][heads of the group][64].
// Which blocks are visited: those of the first `sinks` positions, then those from the first row's window to the last row's position; the mask is applied in blocks that some row does not see whole.
// A value that some rows see and others do not, and that is no number, would reach the others as 0 x inf: in such blocks it is put to zero in shared memory, and added at the
// end to the rows that see it.
// P is rounded to bf16 for the second product.  Every mbarrier wait is bounded; a wait that runs out sets an error word (tgp_k_attn_status), every role leaves its loop, loads in flight are waited for, TMEM
// is freed and nothing is stored.
//
// What bounds it: a block of 64 keys takes one CTA some 1670 cycles and two on an SM 2400 together, 512 of them the tensor pipe's and as many the exponentials' for each by arithmetic; the rest is their chain within a CTA, and the
// instruction cache: loops that few rows reach are not unrolled, and a block is exponentiated in halves by the same code (together 207 -> 181 us in the case below, in turn).  A tile costs some 7600 cycles besides.  Three prompts of up to 2500 tokens, 64 heads
// of 128 over 8, a window of 1000: 189 - 196 us behind calls of its own kind, 189 - 190 between appends, 0.39 to 0.40 of what the products alone take at 1667 TFLOP/s (tensor pipe 37 %, exponentials' 38 % busy).  Without the window 218 - 237, 0.44 to 0.48.  No step bounds it by itself: copies without exponentials, most of
// S, most of P V or the loads took 2 to 6 % less, one without the softmax 12 %.  Not better: blocks of 128 keys, those shared by two tiles in one CTA an SM, all of a block's scores at a time, 16 columns of S at a time,
// exponentials of a quarter or half of the pairs by polynomials (even), eight softmax warps that share rows (198 us), a tile's keys split over several CTAs and joined where there are few tiles (even there, and 1.1 times as
// long elsewhere by its code alone).
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

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
                   "=r"(r[14]), "=r"(r[15]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
                 "r"(r[15]) : "memory");
}

struct ManyArgs { TgpPagedAttn a; unsigned long long *counter; uint32_t tokens, piece; int none; bool wide; };      // tiles begun beyond the CTAs' first ones; tokens of a tile, rows of a piece, a row outside the maps; output on 32 bytes

// what a CTA works on: `tokens` tokens of a sequence and KV head, the first at row `row` and position `pos` (no tokens: the end)
struct Tile { uint32_t row, pos, tokens, hk, b, missing; };
constexpr uint32_t TILES = 4;                              // of which so many are known ahead

template <int DH>
__global__ void __launch_bounds__(THREADS, 2) tgp_attn_paged_many_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                                                                         const ManyArgs args) {
    extern __shared__ __align__(1024) uint8_t smem[];
    constexpr int KB = DH / 64;                          // 64-wide blocks of the head dimension
    constexpr uint32_t Q_BYTES = KB * BQ * 128, KV_BYTES = KB * BKV * 128;
    uint8_t *Qs = smem, *Ks = Qs + Q_BYTES, *Vs = Ks + 2 * KV_BYTES;                            // K and V: two stages each
    uint64_t *bar_k = reinterpret_cast<uint64_t *>(Vs + 2 * KV_BYTES);      // [2] K stage landed (of a tile's first block also Q)
    uint64_t *bar_v = bar_k + 2;                                       // [2] V stage landed
    uint64_t *bar_s = bar_v + 2;                                       // [2] S_i complete in TMEM (tensor core), in buffer i & 1
    uint64_t *bar_p = bar_s + 2;                                       // [2] all 128 rows of P_i written over S_i, O rescaled where needed
    uint64_t *bar_o = bar_p + 2;                                       // [2] P V_i complete (tensor core): buffer i & 1 and the V stage are free
    uint64_t *bar_kfree = bar_o + 2;                                   // [2] S_i complete: K stage i & 1 is free, and with a tile's last block Q
    uint64_t *bar_ofree = bar_kfree + 2;                               // O of a tile is in registers
    uint64_t *bar_odd = bar_ofree + 1;                                 // `odd` of a tile is what it is going to be
    uint64_t *bar_tile = bar_odd + 1;                                  // [TILES] a tile is known
    uint64_t *bar_tfree = bar_tile + TILES;                            // [TILES] the seven warps that work on it have read it
    Tile *tiles = reinterpret_cast<Tile *>(bar_tfree + TILES);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(tiles + TILES);
    volatile uint32_t *failed = tmem_slot + 1;                         // [0] a wait ran out; [1] never set
    volatile uint32_t *odd = failed + 2;                               // [2] (of tiles in turn) a value that is no number was put to zero
    const TgpPagedAttn &a = args.a;

    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (smem_u32(smem) & 1023u) {                            // the swizzle assumes 1024-byte aligned tiles
        if (tid == 0) atomicCAS(&g_attn_paged_error, 0, 5);
        return;
    }
    // Set-up and the TMEM allocation overlap the previous kernel, which wrote what is read below.
    if (warp == 5 && elect_one()) {
        mbar_init(bar_k, 1); mbar_init(bar_k + 1, 1); mbar_init(bar_v, 1); mbar_init(bar_v + 1, 1);
        mbar_init(bar_s, 1); mbar_init(bar_s + 1, 1); mbar_init(bar_p, 128); mbar_init(bar_p + 1, 128); mbar_init(bar_o, 1); mbar_init(bar_o + 1, 1); mbar_init(bar_kfree, 1); mbar_init(bar_kfree + 1, 1);
        mbar_init(bar_ofree, 128); mbar_init(bar_odd, 1);
        for (uint32_t i = 0; i < TILES; ++i) { mbar_init(bar_tile + i, 1); mbar_init(bar_tfree + i, 7); }
        failed[0] = 0;
        failed[1] = 0;
        odd[0] = odd[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmQ) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmK) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmV) : "memory");
    }
    if (warp == 4) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(256u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        asm volatile("griddepcontrol.wait;" ::: "memory");                  // the few-rows kernel reads, without a wait of its own, what this one waits for
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");     // not before the allocation: see tgp_sm100.cuh
    }
    // rows of Q behind the box's: zeros, so that they do not slow the softmax down
    for (uint32_t i = args.tokens * a.G * KB * 8 + tid; i < BQ * KB * 8; i += THREADS)
        *reinterpret_cast<uint4 *>(Qs + (i / 8 % KB) * (BQ * 128) + (i / (8 * KB)) * 128 + (i % 8) * 16) = make_uint4(0, 0, 0, 0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = *tmem_slot;
    const uint32_t tmem_S = tmem_base, tmem_O = tmem_base + 2 * BKV;         // S: two buffers of 64 columns; P_i (32 columns of bf16 pairs) takes the first of S_i's
    const uint32_t pieces = BKV / args.piece;
    auto give_up = [&](int code) { if (!*failed) { *failed = 1; atomicCAS(&g_attn_paged_error, 0, code); } };
    auto wait = [&](uint64_t *bar, uint32_t parity, int code) {              // by a warp
        const bool ok = mbar_wait(bar, parity, failed);
        if (!ok) give_up(code);
        return __all_sync(0xffffffffu, ok);
    };
    auto page_at = [&](const Tile &t, uint32_t key) { const uint32_t i = key / a.P; return i < a.W ? (uint32_t)a.table[(size_t)t.b * a.W + i] : 0xffffffffu; };
    auto last_of = [&](const Tile &t) { return t.pos + t.tokens - 1; };
    auto keys_of = [&](const Tile &t) { return tgp_paged_keys<BKV>(a, t.pos, last_of(t)); };
    // whole: every row sees every key of the block
    auto whole = [&](const Tile &t, uint32_t key0) { return key0 + BKV - 1 <= t.pos && (!a.window || last_of(t) - key0 < a.window || key0 + BKV <= a.sinks); };
    // the n-th tile of this CTA; false at the end
    auto tile_at = [&](Tile &t, uint32_t n, bool &ok) {
        ok = wait(bar_tile + n % TILES, n / TILES & 1, 4);
        if (!ok) return false;
        t = tiles[n % TILES];
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_tfree + n % TILES);
        return t.tokens != 0;
    };
    // Registers move from the second warpgroup (three single-thread roles and the warp that finds tiles) to the softmax warpgroup:
    // 128 * 64 + 128 * 192 is the 128 per thread the CTA is launched with.
    if (warp >= 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;" ::: "memory");
        if (warp == 7) {
            // ======================= tiles: the first is the CTA's own, further ones are those that nobody has begun =======================
            uint32_t all = 0;                                                // tiles of all sequences
#pragma unroll 4
            for (uint32_t i0 = 0; i0 < a.B; i0 += 32) {
                uint32_t mine = 0;
                if (i0 + lane < a.B) { const TgpPagedSeq s = tgp_paged_seq(a, i0 + lane); if (s.n && !s.idle && s.n * a.G > a.few) mine = (s.n + args.tokens - 1) / args.tokens; }
                all += __reduce_add_sync(0xffffffffu, mine);
            }
            const uint32_t items = all * a.Hkv;
            bool ok = true;
            uint32_t i0 = 0, before = 0;                                     // 32 sequences, and the tiles before them: a CTA's items ascend, so they do, too
            for (uint32_t n = 0, item = blockIdx.x; ok; ++n) {
                Tile t{0, 0, 0, 0, 0, 0};
                const bool live = item < items;
                if (live) {
                    // A sequence's last tile (the longest) comes first, and the KV heads of a tile one after the other.
                    const uint32_t at = item / a.Hkv;
                    t.hk = item - at * a.Hkv;
                    for (; i0 < a.B; i0 += 32) {
                        TgpPagedSeq s{0, 0, 0, false};
                        uint32_t mine = 0;
                        if (i0 + lane < a.B) { s = tgp_paged_seq(a, i0 + lane); if (s.n && !s.idle && s.n * a.G > a.few) mine = (s.n + args.tokens - 1) / args.tokens; }
                        uint32_t x = mine;
#pragma unroll
                        for (int o = 1; o < 32; o <<= 1) { const uint32_t y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
                        const uint32_t hit = __ballot_sync(0xffffffffu, before + x > at);
                        if (hit) {
                            const int from = __ffs(hit) - 1;
                            const uint32_t t0 = (before + __shfl_sync(0xffffffffu, x, from) - 1 - at) * args.tokens, rows = __shfl_sync(0xffffffffu, s.n, from);
                            t.b = i0 + from;
                            t.row = __shfl_sync(0xffffffffu, s.first, from) + t0;
                            t.pos = __shfl_sync(0xffffffffu, s.end, from) - rows + t0;
                            t.tokens = min(args.tokens, rows - t0);
                            break;
                        }
                        before += __shfl_sync(0xffffffffu, x, 31);
                    }
                    const TgpPagedKeys keys = keys_of(t);                    // is a page missing?
                    uint32_t missing = 0;
                    for (uint32_t i = lane; i < keys.chunks * pieces; i += 32) {
                        const uint32_t key = keys.chunk(i / pieces) * BKV + i % pieces * args.piece;
                        missing |= key <= last_of(t) && page_at(t, key) >= a.n_pages;
                    }
                    t.missing = __any_sync(0xffffffffu, missing);
                }
                if (n >= TILES) ok = wait(bar_tfree + n % TILES, n / TILES - 1 & 1, 4);
                if (ok && lane == 0) { tiles[n % TILES] = t; mbar_arrive(bar_tile + n % TILES); }
                __syncwarp();
                if (!live) break;
                // Every item is followed by one number, so the last one is number `items`.  (A CTA that gave up takes numbers all the same, to the end: the counter has to be put back.)
                do {
                    uint32_t next = 0;
                    if (lane == 0) {
                        next = tgp_paged_arrive(args.counter);
                        if (next == items) atomicExch(args.counter, 0ull);
                    }
                    item = gridDim.x + __shfl_sync(0xffffffffu, next, 0) - 1;
                } while (!ok && item < items);
            }
        } else if (warp == 5) {
            // ======================= TMA warp =======================
            // Places in the sequence of all blocks: of K, two blocks ahead, and of V.  Either has 32 pieces' rows of the maps in its lanes (args.none: zeros).
            struct Cursor { Tile t; TgpPagedKeys keys; uint32_t n, j, i, base; int rows; bool live; };      // tile n, its block j, block i of all; lane 0's piece
            bool ok = true;
            auto fill = [&](Cursor &c) {
                c.base = c.j * pieces;
                const uint32_t piece = c.base + lane, j = piece / pieces;
                c.rows = args.none;
                if (j < c.keys.chunks) {
                    const uint32_t key = c.keys.chunk(j) * BKV + piece % pieces * args.piece;
                    if (key <= last_of(c.t)) { const uint32_t page = page_at(c.t, key); if (page < a.n_pages) c.rows = (int)((page * a.Hkv + c.t.hk) * a.P + key % a.P); }
                }
            };
            auto enter = [&](Cursor &c, bool release) {
                ok = wait(bar_tile + c.n % TILES, c.n / TILES & 1, 4);
                if (!ok) { c.live = false; return; }
                c.t = tiles[c.n % TILES];
                __syncwarp();
                if (release && lane == 0) mbar_arrive(bar_tfree + c.n % TILES);
                c.live = c.t.tokens != 0;
                c.j = 0;
                if (c.live) { c.keys = keys_of(c.t); fill(c); }
            };
            auto load = [&](Cursor &c, uint8_t *dst, const CUtensorMap *map, uint64_t *bar, uint32_t more_bytes) {
                if (elect_one()) mbar_expect_tx(bar, KV_BYTES + more_bytes);
                __syncwarp();
#pragma unroll 1
                for (uint32_t i = 0; i < pieces; ++i) {
                    const int y = __shfl_sync(0xffffffffu, c.rows, c.j * pieces + i - c.base);
                    if (elect_one())
#pragma unroll
                        for (uint32_t kb = 0; kb < KB; ++kb) tma_load_2d(dst + kb * (BKV * 128) + i * args.piece * 128, map, kb * 64, y, bar);
                    __syncwarp();
                }
                ++c.i;
            };
            auto step = [&](Cursor &c, bool release) {
                if (++c.j == c.keys.chunks) { ++c.n; enter(c, release); }
                else if ((c.j + 1) * pieces - c.base > 32) fill(c);
            };
            Cursor k{}, v{};
            enter(k, false);
            if (ok) enter(v, true);
            auto load_k = [&]() {                                            // with a tile's first block Q is waited for, too
                load(k, Ks + (k.i & 1) * KV_BYTES, &tmK, bar_k + (k.i & 1), k.j == 0 ? KB * args.tokens * a.G * 128 : 0);
            };
            auto load_q = [&](uint32_t i, const Tile &t) {
                if (elect_one())
#pragma unroll
                    for (uint32_t kb = 0; kb < KB; ++kb) tma_load_3d(Qs + kb * (BQ * 128), &tmQ, kb * 64, t.hk * a.G, t.row, bar_k + (i & 1));
                __syncwarp();
            };
            // test hook: the first CTA of the grid never loads this V block, so the wait for it runs out
            const uint32_t withhold = blockIdx.x == 0 ? (uint32_t)g_withhold_step : 0xffffffffu;
            uint32_t q_due = 0xffffffffu;                                    // the block whose Q is not asked for yet
            Tile q_tile{};
            // block i: K_i goes where K_i-2 was, once S_i-2 is complete, V_i-1 where V_i-3 was, once P V_i-3 is, and Q of block i where that of the tile before was, once S_i-1 is
            for (uint32_t i = 0; ok; ++i) {
                const bool more = k.live;
                if (more) {
                    if (i >= 2 && !(ok = wait(bar_kfree + (i & 1), (i - 2 >> 1) & 1, 1))) break;
                    if (k.j == 0) { q_due = i; q_tile = k.t; }
                    load_k();
                    if (i == 0) { load_q(0, q_tile); q_due = 0xffffffffu; }
                    step(k, false);
                    if (!ok) break;
                }
                if (i >= 1) {
                    if (!v.live) break;
                    if (v.i == withhold) break;
                    if (v.i >= 2 && !(ok = wait(bar_o + (v.i & 1), (v.i - 2 >> 1) & 1, 2))) break;
                    load(v, Vs + (v.i & 1) * KV_BYTES, &tmV, bar_v + (v.i & 1), 0);
                    step(v, true);
                    if (!ok) break;
                }
                if (q_due == i && i) {
                    if (!(ok = wait(bar_kfree + (i - 1 & 1), (i - 1 >> 1) & 1, 1))) break;
                    load_q(i, q_tile);
                    q_due = 0xffffffffu;
                }
            }
            // every load asked for must have landed before the CTA may exit (bounded; `never` is never set), and with a tile's first K that of the Q that it is waited for with
            volatile uint32_t *never = failed + 1;
            if (q_due != 0xffffffffu && __all_sync(0xffffffffu, mbar_wait(bar_kfree + (q_due - 1 & 1), (q_due - 1 >> 1) & 1, never))) load_q(q_due, q_tile);
            for (uint32_t st = 0; st < 2; ++st) {
                const uint32_t ck = (k.i + 1 - st) >> 1, cv = (v.i + 1 - st) >> 1;   // loads asked for into this stage
                if (ck) mbar_wait(bar_k + st, (ck - 1) & 1, never);
                if (cv) mbar_wait(bar_v + st, (cv - 1) & 1, never);
            }
        } else if (warp == 4) {
            // ======================= S warp: one thread issues S_i = Q K_i^T =======================
            constexpr uint32_t idesc_s = umma_idesc(BKV);
            Tile t;
            bool ok = true;
            for (uint32_t n = 0, i = 0; ok && tile_at(t, n, ok); ++n) {
                const uint32_t nblk = keys_of(t).chunks;
                for (uint32_t jb = 0; jb < nblk; ++jb, ++i) {
                    if (!(ok = wait(bar_k + (i & 1), (i >> 1) & 1, 3))) break;           // K_i (and Q with a tile's first) has landed
                    if (i >= 2 && !(ok = wait(bar_o + (i & 1), (i - 2 >> 1) & 1, 2))) break;         // P V_i-2: the buffer is free
                    if (elect_one()) {
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint8_t *Ki = Ks + (i & 1) * KV_BYTES;
#pragma unroll
                        for (uint32_t kb = 0; kb < KB; ++kb) {
                            const uint64_t dq = umma_desc(smem_u32(Qs + kb * (BQ * 128))), dk = umma_desc(smem_u32(Ki + kb * (BKV * 128)));
#pragma unroll
                            for (uint32_t k = 0; k < 4; ++k) umma(tmem_S + (i & 1) * BKV, dq + 2 * k, dk + 2 * k, idesc_s, (kb | k) != 0);
                        }
                        umma_commit(bar_s + (i & 1));
                        umma_commit(bar_kfree + (i & 1));                            // its completion also frees the K stage
                    }
                    __syncwarp();
                }
            }
        } else if (warp == 6) {
            // ======================= P V warp: one thread issues O += P_i V_i =======================
            constexpr uint32_t idesc_o = umma_idesc(DH) | (1u << 16);           // bit 16: B operand is MN-major
            Tile t;
            bool ok = true;
            for (uint32_t n = 0, i = 0; ok && tile_at(t, n, ok); ++n) {
                const TgpPagedKeys keys = keys_of(t);
                const uint32_t last_pos = last_of(t);
                if (lane == 0) odd[n & 1] = 0;                                  // (the tile before the last is done with it: its O has been waited for)
                __syncwarp();
                for (uint32_t jb = 0; jb < keys.chunks; ++jb, ++i) {
                    const uint32_t st = i & 1, key0 = keys.chunk(jb) * BKV;
                    if (!(ok = wait(bar_v + st, (i >> 1) & 1, 3))) break;
                    // Steps of 16 keys that no row sees are left out.  In the others, values that no row sees, whatever the page holds there, are zeros; those that some rows see and
                    // others do not are looked at, and what is no number becomes zero and is remembered.
                    uint32_t steps = 0xf;
                    if (!whole(t, key0)) {
                        // rows of the block: [head, from) and [past, 64) are nobody's (a window's: [0, head) are first positions).  Of the others, [near, far) are before some rows' windows and
                        // [sure, past) behind some rows.
                        auto clip = [&](uint32_t key) { return key <= key0 ? 0u : min(key - key0, BKV); };
                        const uint32_t past = clip(last_pos + 1), from = min(past, clip(keys.low)), head = min(from, clip(a.sinks)), sure = max(from, min(past, clip(t.pos + 1)));
                        const uint32_t near = max(from, min(past, clip(a.sinks))), far = a.window && last_pos >= a.window ? max(near, min(past, clip(last_pos - a.window + 1))) : near;
                        auto rows_of = [&](uint32_t r0, uint32_t r1, auto &&f) {         // f of every 16 bytes of rows [r0, r1)
#pragma unroll 1
                            for (uint32_t e = lane; e < (r1 - r0) * KB * 8 && r1 > r0; e += 32) f(reinterpret_cast<uint4 *>(Vs + st * KV_BYTES + (e / 8 % KB) * (BKV * 128) + (r0 + e / (KB * 8)) * 128 + e % 8 * 16));
                        };
                        auto zero = [&](uint4 *at) { *at = make_uint4(0u, 0u, 0u, 0u); };
                        steps = 0;
#pragma unroll 1
                        for (uint32_t k = 0; k < 4; ++k) if (16 * k < head || (16 * k + 16 > from && 16 * k < past)) steps |= 1u << k;
                        // (of steps that are left out nothing is read)
                        rows_of(past, min(BKV, (past + 15) / 16 * 16), zero);
                        rows_of(head, min(from, (head + 15) / 16 * 16), zero);
                        rows_of(max(head, from / 16 * 16), from, zero);
                        uint32_t exponents = 0;                                  // a bit where a half word's exponent is all ones
                        auto look = [&](uint4 *at) {
                            const uint4 v = *at;
                            exponents |= ((v.x & 0x7f807f80u) + 0x00800080u) | ((v.y & 0x7f807f80u) + 0x00800080u) | ((v.z & 0x7f807f80u) + 0x00800080u) | ((v.w & 0x7f807f80u) + 0x00800080u);
                        };
                        rows_of(near, far, look);
                        rows_of(sure, past, look);
                        if (__any_sync(0xffffffffu, (exponents & 0x80008000u) != 0)) {
                            auto clean = [&](uint4 *at) {
                                uint32_t w[4] = {at->x, at->y, at->z, at->w};
#pragma unroll
                                for (int h = 0; h < 4; ++h) {
                                    if ((w[h] & 0x7f80u) == 0x7f80u) w[h] &= 0xffff0000u;
                                    if ((w[h] & 0x7f800000u) == 0x7f800000u) w[h] &= 0xffffu;
                                }
                                *at = make_uint4(w[0], w[1], w[2], w[3]);
                            };
                            rows_of(near, far, clean);
                            __syncwarp();
                            rows_of(sure, past, clean);
                            if (lane == 0) odd[n & 1] = 1;
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    }
                    if (!(ok = wait(bar_p + st, (i >> 1) & 1, 4))) break;
                    if (jb == 0 && n && !(ok = wait(bar_ofree, (n - 1) & 1, 4))) break;  // O of the tile before is in registers
                    if (elect_one()) {
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint64_t dv = umma_desc_mn(smem_u32(Vs + st * KV_BYTES), BKV * 128);
#pragma unroll
                        for (uint32_t k = 0; k < 4; ++k)                             // 16 keys per step: 8 columns of P, 2048 B of V rows
                            if (steps >> k & 1) umma_ts(tmem_O, tmem_S + st * BKV + 8 * k, dv + 128 * k, idesc_o, jb != 0 || (steps & ((1u << k) - 1)) != 0);
                        umma_commit(bar_o + st);
                    }
                    __syncwarp();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_odd);
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;" ::: "memory");
        // ======================= softmax warps: thread = row = TMEM lane =======================
        const uint32_t tok = tid / a.G;
        const uint32_t lane_addr = (warp * 32u) << 16;                       // this warp's quarter of the TMEM lanes
        Tile t;
        bool ok = true;
        for (uint32_t n = 0, i0 = 0; ok && tile_at(t, n, ok); ++n) {
            const TgpPagedKeys keys = keys_of(t);
            const uint32_t nblk = keys.chunks, qpos = t.pos + min(tok, t.tokens - 1);    // padding rows take the last token's mask
            const bool row_ok = tid < t.tokens * a.G;
            float m_ref = -FLT_MAX, lrow = 0.f;                              // exponent reference and running sum of this row
            for (uint32_t jb = 0; jb < nblk; ++jb) {
                const uint32_t i = i0 + jb, key0 = keys.chunk(jb) * BKV, buffer = tmem_S + lane_addr + (i & 1) * BKV;
                if (!(ok = wait(bar_s + (i & 1), (i >> 1) & 1, 1))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                uint64_t hidden = 0;                                         // a bit per key that is: behind the row, or before its window and none of the first positions, or of no page
                if (t.missing || !whole(t, key0)) {
                    auto below = [&](int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; };       // the first n keys of the block
                    const uint32_t low = a.window && qpos >= a.window ? qpos - a.window + 1 : 0;
                    hidden = ~below((int)(qpos - key0) + 1) | (below((int)(low - key0)) & ~below((int)(min(a.sinks, 0x7fffffffu) - key0)));
                    if (t.missing)
#pragma unroll 1
                        for (uint32_t e = 0; e < 4; ++e) if (page_at(t, key0 + e * 16) >= a.n_pages) hidden |= 0xffffull << e * 16;       // (no page begins inside 16 keys)
                }
                const bool masked = __any_sync(0xffffffffu, hidden != 0);
                // Half a block at a time, by the same code: with all of a block unrolled, in several places, warps waited for instructions.
#pragma unroll 1
                for (uint32_t half = 0; half < 2; ++half) {
                    float s[32];
                    tmem_ld32(buffer + half * 32, s);
                    if (masked) {
                        const uint32_t h = half ? (uint32_t)(hidden >> 32) : (uint32_t)hidden;
#pragma unroll
                        for (uint32_t e = 0; e < 32; ++e) if (h >> e & 1) s[e] = -INFINITY;
                    }
                    // The exponent reference m_ref is the row's maximum of the tile's first keys, moved only where its own sum says that a score lies more than about 2^40 above it (or overflowed):
                    // the others of the warp keep theirs, so that a row's bits do not depend on its neighbours, and rows that nobody has (the next sequence's queries) do not ask.  A
                    // row that sees nothing of the first ones has the lowest finite reference: its sums are 0, and the first finite score moves it.
                    uint32_t w[16];
                    float sum;
                    for (bool move = (jb | half) == 0, own = move;;) {
                        if (move) {                                          // the maximum of the scaled scores (scale > 0: it commutes with it)
                            float m0 = max3(s[0], s[1], s[2]), m1 = max3(s[3], s[4], s[5]);
#pragma unroll
                            for (uint32_t e = 6; e + 3 < 32; e += 4) { m0 = max3(m0, s[e], s[e + 1]); m1 = max3(m1, s[e + 2], s[e + 3]); }
                            const float m_new = own ? fmaxf(m_ref, max3(m0, m1, fmaxf(s[30], s[31])) * a.sl2) : m_ref, alpha = ex2(m_ref - m_new);
                            m_ref = m_new;
                            lrow *= alpha;
                            if (half) {                                      // the first half's weights
                                uint32_t v[16];
                                tmem_wait_st();
                                tmem_ld16(buffer, v);
#pragma unroll
                                for (uint32_t e = 0; e < 16; ++e) { const __nv_bfloat162 two = *reinterpret_cast<__nv_bfloat162 *>(&v[e]), x = __floats2bfloat162_rn(__low2float(two) * alpha, __high2float(two) * alpha); v[e] = *reinterpret_cast<const uint32_t *>(&x); }
                                tmem_st16(buffer, v);
                            }
                            if (jb) {
                                if (!(ok = wait(bar_o + (i - 1 & 1), (i - 1 >> 1) & 1, 2))) break;   // P V_{i-1}: nothing is accumulating into O
                                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
                                for (uint32_t h = 0; h < DH / 32; ++h) {
                                    float v[32];
                                    uint32_t u[32];
                                    tmem_ld32(tmem_O + lane_addr + h * 32, v);
#pragma unroll
                                    for (uint32_t e = 0; e < 32; ++e) u[e] = __float_as_uint(v[e] * alpha);
                                    tmem_st32(tmem_O + lane_addr + h * 32, u);
                                }
                            }
                        }
                        // w = exp2(S * scale - m) as bf16 pairs, and their fp32 sum
                        const uint64_t sc2 = pack2(a.sl2, a.sl2), nm2 = pack2(-m_ref, -m_ref);
                        uint64_t acc0 = pack2(0.f, 0.f), acc1 = acc0;
#pragma unroll
                        for (uint32_t e = 0; e < 16; ++e) {
                            float x0, x1;
                            unpack2(fma2(pack2(s[2 * e], s[2 * e + 1]), sc2, nm2), x0, x1);
                            const float p0 = ex2(x0), p1 = ex2(x1);          // a masked score is -inf: p = 0
                            if (e & 1) acc1 = add2(acc1, pack2(p0, p1)); else acc0 = add2(acc0, pack2(p0, p1));
                            __nv_bfloat162 pk = __floats2bfloat162_rn(p0, p1);   // .x = p0 in the lower half
                            w[e] = *reinterpret_cast<uint32_t *>(&pk);
                        }
                        float l0, l1;
                        unpack2(add2(acc0, acc1), l0, l1);
                        sum = l0 + l1;
                        own = sum > 0x1p40f && row_ok;                       // (a NaN is one with any reference)
                        if (move || !__any_sync(0xffffffffu, own)) break;
                        move = true;
                    }
                    if (!ok) break;
                    lrow += sum;
                    tmem_st16(buffer + half * 16, w);                        // over scores that have been read
                }
                if (!ok) break;
                tmem_wait_st();
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                mbar_arrive(bar_p + (i & 1));
            }
            i0 += nblk;
            // ---- the last P V; normalise and store this thread's row ----
            ok = ok && wait(bar_o + (i0 - 1 & 1), (i0 - 1 >> 1) & 1, 2) && wait(bar_odd, n & 1, 2);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const bool empty = lrow == 0.f;                                  // a row that sees nothing is zero
            const float inv = 1.0f / lrow;
            bf16 *dst = a.o + ((size_t)(t.row + tok) * a.Hq + t.hk * a.G + (tid - tok * a.G)) * DH;
#pragma unroll 1
            for (uint32_t h = 0; h < DH / 32; ++h) {
                float v[32];
                __syncwarp();
                tmem_ld32(tmem_O + lane_addr + h * 32, v);
                uint32_t w[16];
#pragma unroll
                for (uint32_t e = 0; e < 16; ++e) {
                    __nv_bfloat162 pk = __floats2bfloat162_rn(v[2 * e] * inv, v[2 * e + 1] * inv);
                    w[e] = empty ? 0u : *reinterpret_cast<uint32_t *>(&pk);
                }
                if (!row_ok) continue;
                if (args.wide) {                                             // (whole sectors)
#pragma unroll
                    for (uint32_t c = 0; c < 2; ++c)
                        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst + h * 32 + c * 16), "r"(w[8 * c]), "r"(w[8 * c + 1]), "r"(w[8 * c + 2]), "r"(w[8 * c + 3]),
                                     "r"(w[8 * c + 4]), "r"(w[8 * c + 5]), "r"(w[8 * c + 6]), "r"(w[8 * c + 7]) : "memory");
                } else {
#pragma unroll
                    for (uint32_t c = 0; c < 4; ++c) *reinterpret_cast<uint4 *>(dst + h * 32 + c * 8) = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
                }
            }
            __syncwarp();
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            mbar_arrive(bar_ofree);
            if (odd[n & 1] && row_ok) {                                      // keys that some rows see and others do not: what was put to zero is added now
                const uint32_t last_pos = last_of(t);
#pragma unroll 1
                for (uint32_t jb = 0; jb < nblk; ++jb) {
                    const uint32_t key0 = keys.chunk(jb) * BKV;
                    if (whole(t, key0)) continue;
#pragma unroll 1
                    for (uint32_t key = key0; key < key0 + BKV && key <= qpos; ++key) {
                        const uint32_t page = page_at(t, key);
                        if (page >= a.n_pages || !tgp_paged_sees(a, qpos, key) || (key <= t.pos && (!a.window || last_pos - key < a.window || key < a.sinks))) continue;
                        const bf16 *from = a.v + (((size_t)page * a.Hkv + t.hk) * a.P + key % a.P) * DH;
#pragma unroll 1
                        for (uint32_t e = 0; e < DH; ++e) {
                            const float x = __bfloat162float(from[e]);
                            if (!(fabsf(x) < INFINITY)) dst[e] = __float2bfloat16_rn(__bfloat162float(dst[e]) + x);
                        }
                    }
                }
            }
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 4) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(256u) : "memory");
    }
}

template <int DH> constexpr int smem_bytes() { return (DH / 64) * (BQ + 4 * BKV) * 128 + 512; }

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

int tgpk_attn_paged_many(const TgpPagedAttn &a, uint32_t Dh, unsigned long long *counter, cudaStream_t st) {
    ManyArgs args{a, counter, BQ / a.G, BKV, 0, reinterpret_cast<uintptr_t>(a.o) % 32 == 0};
    while (a.P % args.piece) args.piece /= 2;                                // (a page holds a multiple of 16 positions)
    const uint64_t rows = (uint64_t)a.n_pages * a.Hkv * a.P;
    args.none = (int)rows;
    CUtensorMap mq, mk, mv;
    if (!tensor_map_q(&mq, a.q, a.T, a.Hq, Dh, a.G, args.tokens) || !tensor_map_bf16_2d(&mk, a.k, rows, Dh, (uint64_t)Dh * 2, args.piece) ||
        !tensor_map_bf16_2d(&mv, a.v, rows, Dh, (uint64_t)Dh * 2, args.piece)) return TGP_E_CUDA;
    // tiles: of T rows, and one more for each sequence that this kernel has; two CTAs fit an SM
    const uint32_t least = a.few / a.G + 1, tiles = a.T / args.tokens + std::min(a.B, a.T / least);
    const dim3 grid((uint32_t)std::min<uint64_t>((uint64_t)tiles * a.Hkv, 2 * (uint32_t)tgpk_sms()));
    return Dh == 64 ? launch_many<64>(mq, mk, mv, args, grid, st) : launch_many<128>(mq, mk, mv, args, grid, st);
}

int tgpk_attn_paged_wait_test(unsigned long long limit_ns, int withhold_step) {
    if (cudaMemcpyToSymbol(g_wait_limit_ns, &limit_ns, sizeof(limit_ns)) != cudaSuccess) return TGP_E_CUDA;
    return cudaMemcpyToSymbol(g_withhold_step, &withhold_step, sizeof(withhold_step)) == cudaSuccess ? TGP_OK : TGP_E_CUDA;
}

int tgpk_attn_paged_status_clear() { const int z = 0; return cudaMemcpyToSymbol(g_attn_paged_error, &z, sizeof(z)) == cudaSuccess ? TGP_OK : TGP_E_CUDA; }
int tgpk_attn_paged_status(int *code) { return cudaMemcpyFromSymbol(code, g_attn_paged_error, sizeof(int)) == cudaSuccess ? TGP_OK : TGP_E_CUDA; }
