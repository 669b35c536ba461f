// Attention of a ragged batch over a KV cache in pages: single tokens and a few drafted ones, on mma.sync; the entry point.  (Prompts: tgp_attn_paged_sm100.cu.)
//
// A page is [Hkv, P, DH] in bf16, so the P keys of one head of a page are one piece of memory.  Rows of a sequence and KV head - new tokens x query heads of the group, up to 16 MT - are the
// rows of m16n8k16 tiles; a warp takes 16 keys at a time, which it stages itself with cp.async three chunks deep, and keeps for each row a running maximum, the sum of the rounded
// weights and an unnormalised output in fp32:  p = 2^(s - m),  l += p,  O += p V,  and both times 2^(m - m') where the maximum grows to m'.  Weights are rounded to bf16 for the second
// product, and those that are summed are the rounded ones, so what is divided by is what the values were multiplied by.
//
// Split: all chunks of all sequences and KV heads are one line, of which every CTA takes an equal stretch; lengths are known on the device only, so every CTA adds up the sequences' chunks for
// itself.  Where a stretch ends inside a (sequence, KV head), its CTA leaves (maximum, sum, output) in the scratch, and the last one to arrive at that pair's counter merges them
// all in the order of the stretches, so that results do not depend on who was last.
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include "tgp.h"
#include "tgp_kernels.h"
#include "tgp_launch.cuh"
#include "tgp_attn_paged.cuh"

namespace {

using namespace tgp_launch;
typedef __nv_bfloat16 bf16;
typedef unsigned long long u64;

constexpr uint32_t KEYS = 16, WARPS = 4, STAGES = 3, GROUP = 1024;          // GROUP: sequences of a launch, whose counts lie in shared memory
constexpr uint32_t MIN_STRETCH = 2 * WARPS;                                  // chunks
// A counter is a number of arrivals only with this in its upper half: a NaN that no arithmetic gives, so whatever else the memory held, partials of an earlier call among
// it, counts as 0.  The last arrival puts 0 back.
constexpr u64 COUNTS = 0xffa5c3d1ull << 32;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, uint32_t src_bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}
__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t &r0, uint32_t &r1, uint32_t &r2, uint32_t &r3) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(addr));
}
__device__ __forceinline__ void ldsm_x4_t(uint32_t addr, uint32_t &r0, uint32_t &r1, uint32_t &r2, uint32_t &r3) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(addr));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
// two weights as bf16, and what they are then
__device__ __forceinline__ uint32_t rounded2(float &a, float &b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    a = __low2float(h); b = __high2float(h);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ bool not_finite2(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }

template <int DH> __host__ __device__ constexpr uint32_t stage_bytes() { return 2 * KEYS * DH * 2; }
template <int DH, int MT> __host__ __device__ constexpr uint32_t q_bytes() { return MT > 1 ? MT * 16 * DH * 2 : 0; }
template <int DH, int MT> __host__ __device__ constexpr uint32_t fixed_smem() { return WARPS * STAGES * stage_bytes<DH>() + q_bytes<DH, MT>() + WARPS * 16 * 2 * 4 + 64; }
template <int DH, int MT> __host__ __device__ constexpr uint32_t slot_floats() { return MT * 16 * (DH + 2); }

struct FewArgs { TgpPagedAttn a; float *parts; u64 *counters; };

template <int DH, int MT>
__global__ void __launch_bounds__(WARPS * 32, DH == 128 ? 2 : MT == 1 ? 4 : 3) tgp_attn_paged_few_kernel(const FewArgs f) {
    pdl_enter();
    const TgpPagedAttn &a = f.a;
    extern __shared__ __align__(128) uint8_t few_sm[];
    constexpr uint32_t ROW = DH * 2, CPR = ROW / 16, KV_BYTES = KEYS * ROW, STAGE = stage_bytes<DH>();
    uint8_t *q_sm = few_sm + WARPS * STAGES * STAGE;
    float *ml = reinterpret_cast<float *>(q_sm + q_bytes<DH, MT>());       // [WARPS][16][2]: maxima and sums of the warps' partials
    uint32_t *shared_u = reinterpret_cast<uint32_t *>(ml + WARPS * 16 * 2);
    uint32_t *upto = shared_u + 16;                                         // [B] chunks of the sequences up to this one, all KV heads
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, c = lane & 3;

    // ---- the line of all chunks ----
    {
        uint32_t before = 0;
        for (uint32_t i0 = 0; i0 < a.B; i0 += WARPS * 32) {
            const uint32_t i = i0 + tid;
            uint32_t mine = 0;
            if (i < a.B) {
                const TgpPagedSeq s = tgp_paged_seq(a, a.b0 + i);
                if (s.n && !s.idle && s.n * a.G <= a.few) mine = tgp_paged_keys<KEYS>(a, s.end - s.n, s.end - 1).chunks * a.Hkv;
                else if (s.n && s.idle)                                     // rows of idle sequences are zero
                    for (u64 e = blockIdx.x; e < (u64)s.n * a.Hq * DH / 8; e += gridDim.x) reinterpret_cast<uint4 *>(a.o + (size_t)s.first * a.Hq * DH)[e] = make_uint4(0, 0, 0, 0);
            }
            uint32_t x = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const uint32_t y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
            if (lane == 31) shared_u[warp] = x;
            __syncthreads();
            uint32_t all = 0;
#pragma unroll
            for (uint32_t w = 0; w < WARPS; ++w) { if (w < warp) x += shared_u[w]; all += shared_u[w]; }
            if (i < a.B) upto[i] = before + x;
            before += all;
            __syncthreads();
        }
    }
    const uint32_t N = a.B ? upto[a.B - 1] : 0;
    const uint32_t ctas = min(gridDim.x, (N + MIN_STRETCH - 1) / MIN_STRETCH);
    if (blockIdx.x >= ctas) return;
    auto stretch = [&](uint32_t cta) { return (uint32_t)((u64)N * cta / ctas); };
    const uint32_t line_lo = stretch(blockIdx.x), line_hi = stretch(blockIdx.x + 1);

    // an item: a (sequence, KV head) and its place in the line
    struct Item { uint32_t b, hk, lo, hi; TgpPagedSeq s; TgpPagedKeys k; };
    auto enter = [&](Item &it, uint32_t g) {                                // the item of chunk g, whose sequence is it.b or a later one
        while (upto[it.b] <= g) ++it.b;
        it.s = tgp_paged_seq(a, a.b0 + it.b);
        it.k = tgp_paged_keys<KEYS>(a, it.s.end - it.s.n, it.s.end - 1);
        const uint32_t seq_lo = upto[it.b] - it.k.chunks * a.Hkv;
        it.hk = (g - seq_lo) / it.k.chunks;
        it.lo = seq_lo + it.hk * it.k.chunks;
        it.hi = it.lo + it.k.chunks;
    };
    Item ahead, now;
    {
        uint32_t lo = 0, hi = a.B - 1;                                      // the first sequence that ends behind line_lo
        while (lo < hi) { const uint32_t mid = (lo + hi) / 2; if (upto[mid] > line_lo) hi = mid; else lo = mid + 1; }
        ahead.b = lo;
    }
    enter(ahead, line_lo);
    now = ahead;

    // ---- staging: this warp's chunks are line_lo + warp, + WARPS, ... ----
    const uint32_t stages = (uint32_t)__cvta_generic_to_shared(few_sm) + warp * STAGES * STAGE;
    uint32_t issued = 0, next = line_lo + warp;                             // chunks asked for, and the next one to ask for
    auto page_of = [&](const Item &it, uint32_t g) {
        const uint32_t i = it.k.chunk(g - it.lo) * KEYS / a.P;
        return i < a.W ? a.table[(size_t)(a.b0 + it.b) * a.W + i] : -1;
    };
    int32_t page_next = -1;                                                 // of the next chunk to ask for: the table is read one chunk ahead
    if (next < line_hi) {
        if (next >= ahead.hi) enter(ahead, next);
        page_next = page_of(ahead, next);
    }
    uint32_t present = 0;                                                   // a bit per stage: its page is one of the cache's
    auto issue = [&]() {
        if (next < line_hi) {
            const uint32_t key0 = ahead.k.chunk(next - ahead.lo) * KEYS, stage = issued % STAGES;
            const bool there = (uint32_t)page_next < a.n_pages;
            present = there ? present | 1u << stage : present & ~(1u << stage);
            const size_t at = (((size_t)(there ? page_next : 0) * a.Hkv + ahead.hk) * a.P + key0 % a.P) * ROW;
            const uint8_t *kg = reinterpret_cast<const uint8_t *>(a.k) + at, *vg = reinterpret_cast<const uint8_t *>(a.v) + at;
            const uint32_t base = stages + stage * STAGE;
#pragma unroll
            for (uint32_t i = 0; i < KEYS * CPR / 32; ++i) {
                const uint32_t idx = i * 32 + lane, row = idx / CPR, j = idx % CPR, key = key0 + row;
                const uint32_t dst = row * ROW + ((j ^ (row & 7)) << 4);
                // keys that no row sees are zeros, not read
                const uint32_t bytes = there && key < ahead.s.end && (key >= ahead.k.low || key < a.sinks) ? 16u : 0u;
                cp_async16(base + dst, kg + (size_t)row * ROW + j * 16, bytes);
                cp_async16(base + KV_BYTES + dst, vg + (size_t)row * ROW + j * 16, bytes);
            }
            ++issued;
            next += WARPS;
            if (next < line_hi) {
                if (next >= ahead.hi) enter(ahead, next);
                page_next = page_of(ahead, next);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (uint32_t s = 0; s < STAGES - 1; ++s) issue();

    uint32_t done = 0;                                                      // chunks this warp has been through
    for (uint32_t seg_lo = line_lo; seg_lo < line_hi;) {                    // the CTA's part of an item
        if (seg_lo >= now.hi) enter(now, seg_lo);
        const uint32_t seg_hi = min(line_hi, now.hi), rows = now.s.n * a.G, first_pos = now.s.end - now.s.n;
        const bf16 *q_item = a.q + ((size_t)now.s.first * a.Hq + now.hk * a.G) * DH;
        auto q_row = [&](uint32_t row) { const uint32_t t = row / a.G; return q_item + ((size_t)t * a.Hq + (row - t * a.G)) * DH; };
        // ---- Q: in registers (one tile), or in shared memory, rows as wide as the keys' ----
        uint32_t qf[MT == 1 ? DH / 16 : 1][4];
        const uint32_t q_u = (uint32_t)__cvta_generic_to_shared(q_sm);
        if constexpr (MT == 1) {
            const bf16 *q0 = q_row(min(r, rows - 1)) + 2 * c, *q1 = q_row(min(r + 8, rows - 1)) + 2 * c;
#pragma unroll
            for (int ks = 0; ks < DH / 16; ++ks) {
                qf[ks][0] = *reinterpret_cast<const uint32_t *>(q0 + ks * 16);
                qf[ks][1] = *reinterpret_cast<const uint32_t *>(q1 + ks * 16);
                qf[ks][2] = *reinterpret_cast<const uint32_t *>(q0 + ks * 16 + 8);
                qf[ks][3] = *reinterpret_cast<const uint32_t *>(q1 + ks * 16 + 8);
            }
        } else {
            __syncthreads();                                                // (the item before has been multiplied)
            for (uint32_t i = tid; i < MT * 16 * CPR; i += WARPS * 32) {
                const uint32_t row = i / CPR, j = i % CPR;
                *reinterpret_cast<uint4 *>(q_sm + row * ROW + ((j ^ (row & 7)) << 4)) = *reinterpret_cast<const uint4 *>(q_row(min(row, rows - 1)) + j * 8);
            }
            __syncthreads();
        }
        float o[MT][DH / 8][4], m[MT][2], l[MT][2];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            // (from the least number, not from -inf: scores of -inf weigh nothing then, in whichever chunk they are met)
            m[t][0] = m[t][1] = -FLT_MAX;
            l[t][0] = l[t][1] = 0.f;
#pragma unroll
            for (int j = 0; j < DH / 8; ++j) o[t][j][0] = o[t][j][1] = o[t][j][2] = o[t][j][3] = 0.f;
        }
        uint32_t pos[MT][2];                                                // positions of this lane's rows (of the tile's last row where there is none)
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) pos[t][e] = first_pos + min(t * 16 + r + 8 * e, rows - 1) / a.G;

        for (uint32_t g = line_lo + warp + done * WARPS; g < seg_hi; g += WARPS, ++done) {
            issue();
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
            __syncwarp();
            const uint32_t stage = done % STAGES, key0 = now.k.chunk(g - now.lo) * KEYS;
            const uint32_t kb = stages + stage * STAGE, vb = kb + KV_BYTES;
            if (!(present >> stage & 1)) continue;                          // (the stage is refilled behind the next chunk's barrier)
            // whole: every row sees every key
            const bool whole = key0 + KEYS - 1 <= first_pos && (!a.window || now.s.end - 1 - key0 < a.window || key0 + KEYS <= a.sinks);
            // ---- S = Q K^T ----
            float s[MT][2][4];
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) s[t][nt][0] = s[t][nt][1] = s[t][nt][2] = s[t][nt][3] = 0.f;
#pragma unroll
            for (int kp = 0; kp < DH / 32; ++kp) {
                uint32_t b[2][4];
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) {
                    const uint32_t row = nt * 8 + (lane & 7), j = kp * 4 + (lane >> 3);
                    ldsm_x4(kb + row * ROW + ((j ^ (row & 7)) << 4), b[nt][0], b[nt][1], b[nt][2], b[nt][3]);
                }
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        uint32_t x0, x1, x2, x3;
                        if constexpr (MT == 1) { x0 = qf[2 * kp + e][0]; x1 = qf[2 * kp + e][1]; x2 = qf[2 * kp + e][2]; x3 = qf[2 * kp + e][3]; }
                        else {
                            const uint32_t row = t * 16 + (lane & 15), j = (2 * kp + e) * 2 + (lane >> 4);
                            ldsm_x4(q_u + row * ROW + ((j ^ (row & 7)) << 4), x0, x1, x2, x3);
                        }
#pragma unroll
                        for (int nt = 0; nt < 2; ++nt) mma_bf16(s[t][nt], x0, x1, x2, x3, b[nt][2 * e], b[nt][2 * e + 1]);
                    }
            }
            // ---- weights: this lane's keys are 2c, 2c + 1, 8 + 2c, 9 + 2c of rows r and r + 8 ----
            uint32_t pa[MT][4];
            float grow[MT][2];
            bool grows = false;
#pragma unroll
            for (int t = 0; t < MT; ++t) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float top = -INFINITY;
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            float &x = s[t][nt][2 * e + i];
                            x *= a.sl2;
                            if (!whole && !tgp_paged_sees(a, pos[t][e], key0 + nt * 8 + 2 * c + i)) x = -INFINITY;
                            top = fmaxf(top, x);
                        }
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    grow[t][e] = fmaxf(m[t][e], top);
                    grows |= grow[t][e] > m[t][e];
                }
            }
            if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float alpha = ex2(m[t][e] - grow[t][e]);       // (the first time: of zeros)
                        m[t][e] = grow[t][e];
                        l[t][e] *= alpha;
#pragma unroll
                        for (int j = 0; j < DH / 8; ++j) { o[t][j][2 * e] *= alpha; o[t][j][2 * e + 1] *= alpha; }
                    }
            }
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float &x = s[t][nt][2 * e], &y = s[t][nt][2 * e + 1];
                        x = ex2(x - m[t][e]);
                        y = ex2(y - m[t][e]);
                        pa[t][2 * nt + e] = rounded2(x, y);
                        l[t][e] += x + y;                                   // (of this lane's keys: the four lanes of a row meet at the end)
                    }
            // ---- O += P V ----
            // Where some rows see a key and others do not, a value that is no number must not reach the others as 0 x inf: then each row adds up what it sees.
            bool each = false;
            if (!whole && now.s.n > 1) {
                for (uint32_t i = lane; i < KEYS * CPR; i += 32) {
                    uint32_t w0, w1, w2, w3;
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w0), "=r"(w1), "=r"(w2), "=r"(w3) : "r"(vb + i * 16));
                    each |= not_finite2(w0) || not_finite2(w1) || not_finite2(w2) || not_finite2(w3);
                }
                each = __any_sync(0xffffffffu, each);
            }
            if (!each) {
#pragma unroll
                for (int jp = 0; jp < DH / 16; ++jp) {
                    const uint32_t row = ((lane >> 3) & 1) * 8 + (lane & 7), j = 2 * jp + (lane >> 4);
                    uint32_t v0, v1, v2, v3;
                    ldsm_x4_t(vb + row * ROW + ((j ^ (row & 7)) << 4), v0, v1, v2, v3);
#pragma unroll
                    for (int t = 0; t < MT; ++t) {
                        mma_bf16(o[t][2 * jp], pa[t][0], pa[t][1], pa[t][2], pa[t][3], v0, v1);
                        mma_bf16(o[t][2 * jp + 1], pa[t][0], pa[t][1], pa[t][2], pa[t][3], v2, v3);
                    }
                }
            } else {
#pragma unroll 1
                for (uint32_t key = 0; key < KEYS; ++key) {
                    const int from = (lane & ~3) | (key % 8 / 2);           // the lane of this row that has the key's weight
#pragma unroll
                    for (int t = 0; t < MT; ++t)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float w0 = __shfl_sync(0xffffffffu, key < 8 ? s[t][0][2 * e] : s[t][1][2 * e], from), w1 = __shfl_sync(0xffffffffu, key < 8 ? s[t][0][2 * e + 1] : s[t][1][2 * e + 1], from);
                            const float w = key & 1 ? w1 : w0;
                            if (!tgp_paged_sees(a, pos[t][e], key0 + key)) continue;
#pragma unroll
                            for (int j = 0; j < DH / 8; ++j) {
                                uint32_t v;
                                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(vb + key * ROW + ((j ^ (key & 7)) << 4) + 4 * c));
                                const __nv_bfloat162 h = *reinterpret_cast<const __nv_bfloat162 *>(&v);
                                o[t][j][2 * e] += w * __low2float(h);
                                o[t][j][2 * e + 1] += w * __high2float(h);
                            }
                        }
                }
            }
            __syncwarp();                                                   // the stage may be refilled
        }
        // ---- the four warps' partials: outputs go to the stage that each has free (the two behind it are under way), one tile at a time ----
        const bool complete = seg_lo == now.lo && seg_hi == now.hi;
        float *slot = f.parts + ((size_t)blockIdx.x * 2 + (seg_lo == line_lo ? 0 : 1)) * slot_floats<DH, MT>();
        float *mine = reinterpret_cast<float *>(few_sm + (size_t)(warp * STAGES + (done + STAGES - 1) % STAGES) * STAGE);
        auto finish = [&](uint32_t row, uint32_t d, float2 v, float sum) {  // (a row that sees nothing is zero; a NaN stays one)
            const uint32_t t = row / a.G;
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            const __nv_bfloat162 h = sum == 0.f ? __floats2bfloat162_rn(0.f, 0.f) : __floats2bfloat162_rn(v.x * inv, v.y * inv);
            *reinterpret_cast<__nv_bfloat162 *>(a.o + ((size_t)(now.s.first + t) * a.Hq + now.hk * a.G + (row - t * a.G)) * DH + d) = h;
        };
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            if (t && t * 16 >= rows) break;
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float sum = l[t][e];
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                const uint32_t row = r + 8 * e;
                if (t * 16 + row < rows) {
                    if (c == 0) { ml[(warp * 16 + row) * 2] = m[t][e]; ml[(warp * 16 + row) * 2 + 1] = sum; }
#pragma unroll
                    for (int j = 0; j < DH / 8; ++j) *reinterpret_cast<float2 *>(mine + row * DH + ((j * 8 + 2 * c) ^ (row & 7) * 8)) = make_float2(o[t][j][2 * e], o[t][j][2 * e + 1]);
                }
            }
            if (tid == 0) shared_u[8] = 0;
            if (lane == 0) shared_u[warp] = (uint32_t)(reinterpret_cast<uint8_t *>(mine) - few_sm);
            __syncthreads();
            const uint32_t tile_rows = min(16u, rows - t * 16);
            for (uint32_t i = tid; i < tile_rows * DH / 2; i += WARPS * 32) {
                const uint32_t row = i / (DH / 2), d = i % (DH / 2) * 2;
                float M = -FLT_MAX, sum = 0.f;
                float2 v = make_float2(0.f, 0.f);
#pragma unroll
                for (uint32_t w = 0; w < WARPS; ++w) M = fmaxf(M, ml[(w * 16 + row) * 2]);
#pragma unroll
                for (uint32_t w = 0; w < WARPS; ++w) {
                    const float2 x = *reinterpret_cast<const float2 *>(reinterpret_cast<const float *>(few_sm + shared_u[w]) + row * DH + (d ^ (row & 7) * 8));
                    const float wgt = ex2(ml[(w * 16 + row) * 2] - M);      // (a warp without a chunk: any weight of zeros)
                    sum += wgt * ml[(w * 16 + row) * 2 + 1];
                    v.x += wgt * x.x; v.y += wgt * x.y;
                }
                if (complete) finish(t * 16 + row, d, v, sum);
                else {
                    float *to = slot + (size_t)(t * 16 + row) * (DH + 2);
                    if (d == 0) { to[0] = M; to[1] = sum; }
                    *reinterpret_cast<float2 *>(to + 2 + d) = v;
                }
            }
            __syncthreads();
        }
        // ---- an item of several stretches: the last to arrive merges ----
        if (!complete) {
            const uint32_t item = (a.b0 + now.b) * a.Hkv + now.hk;
            // CTAs of the item's first and last chunk
            auto cta_of = [&](uint32_t g) {
                uint32_t x = (uint32_t)(((u64)g * ctas) / N);
                while (x + 1 < ctas && stretch(x + 1) <= g) ++x;
                while (stretch(x) > g) --x;
                return x;
            };
            const uint32_t c0 = cta_of(now.lo), c1 = cta_of(now.hi - 1), parts = c1 - c0 + 1;
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                u64 *counter = f.counters + item, old = *(volatile u64 *)counter, seen, to;
                do {
                    seen = old;
                    to = (seen & 0xffffffff00000000ull) == COUNTS ? seen + 1 : COUNTS + 1;
                    if ((uint32_t)to == parts) to = COUNTS;
                    old = atomicCAS(counter, seen, to);
                } while (old != seen);
                shared_u[8] = to == COUNTS;
                __threadfence();
            }
            __syncthreads();
            if (shared_u[8]) {
                for (uint32_t i = tid; i < rows * DH / 2; i += WARPS * 32) {
                    const uint32_t row = i / (DH / 2), d = i % (DH / 2) * 2;
                    float M = -FLT_MAX, sum = 0.f;
                    float2 v = make_float2(0.f, 0.f);
                    for (uint32_t p = 0; p < parts; ++p) {
                        const uint32_t cta = c0 + p;
                        const float *from = f.parts + ((size_t)cta * 2 + (stretch(cta) >= now.lo ? 0 : 1)) * slot_floats<DH, MT>() + (size_t)row * (DH + 2);
                        const float pm = __ldcg(from), pl = __ldcg(from + 1);
                        const float2 x = __ldcg(reinterpret_cast<const float2 *>(from + 2 + d));
                        const float M2 = fmaxf(M, pm), w_old = ex2(M - M2), w_new = ex2(pm - M2);
                        M = M2;
                        sum = sum * w_old + pl * w_new;
                        v.x = v.x * w_old + x.x * w_new; v.y = v.y * w_old + x.y * w_new;
                    }
                    finish(row, d, v, sum);
                }
            }
            __syncthreads();
        }
        seg_lo = seg_hi;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// CTAs that the GPU holds at a time
template <int DH, int MT> uint32_t few_ctas() { return (uint32_t)tgpk_sms() * (DH == 128 ? 2u : MT == 1 ? 4u : 3u); }

template <int DH, int MT>
int launch_few(FewArgs f, cudaStream_t st) {
    if (!tgpk_allow_smem<tgp_attn_paged_few_kernel<DH, MT>>(fixed_smem<DH, MT>() + GROUP * 4, true)) return TGP_E_CUDA;
    const uint32_t B = f.a.B;
    for (uint32_t b0 = 0; b0 < B; b0 += GROUP) {
        f.a.b0 = b0;
        f.a.B = std::min(GROUP, B - b0);
        if (int rc = launch(tgp_attn_paged_few_kernel<DH, MT>, dim3(few_ctas<DH, MT>()), dim3(WARPS * 32), fixed_smem<DH, MT>() + f.a.B * 4, st, 1, f)) return rc;
    }
    return TGP_OK;
}

bool shapes_ok(const tgp_model_cfg *c) { return c && (c->Dh == 64 || c->Dh == 128) && c->Hkv && c->Hq && c->Hq % c->Hkv == 0 && c->Hq / c->Hkv <= 128 && c->TK && c->TK % 16 == 0 && c->max_len; }

// bytes of the counters, and of the partials of a launch of few rows
uint64_t counter_bytes(const tgp_model_cfg *c, uint32_t B) { return ((uint64_t)B * c->Hkv * 8 + 255) / 256 * 256; }
uint64_t part_bytes(const tgp_model_cfg *c) {
    const uint32_t ctas = c->Dh == 128 ? few_ctas<128, 1>() : few_ctas<64, 1>();
    return (uint64_t)ctas * 2 * 32 * (c->Dh + 2) * 4;
}

}  // namespace

extern "C" int tgp_k_attn_paged_scratch_bytes(const tgp_model_cfg *cfg, uint32_t B, uint32_t T, uint32_t q_max, uint32_t kv_max, uint64_t *bytes) {
    if (!shapes_ok(cfg) || !bytes || B > cfg->B || kv_max > cfg->max_len) return TGP_E_INVAL;
    if (B > TGP_PAGED_MAX_B || cfg->max_len > 0x7fffffffu || T > 0x7fffffffu || cfg->Hq > (1u << 16)) return TGP_E_TOO_LARGE;
    *bytes = counter_bytes(cfg, B) + part_bytes(cfg);
    return TGP_OK;
}

extern "C" int tgp_k_attn_paged(const void *qb, const void *k_pages, const void *v_pages, void *ob, const int32_t *table_dev, const int32_t *start_dev, const int32_t *end_dev,
                                const tgp_model_cfg *cfg, uint32_t B, uint32_t T, uint32_t q_max, uint32_t kv_max, uint32_t n_pages, uint32_t window, uint32_t sinks, void *scratch_dev, void *stream) {
    if (!shapes_ok(cfg) || B > cfg->B || kv_max > cfg->max_len || !n_pages) return TGP_E_INVAL;
    if (!qb || !k_pages || !v_pages || !ob || !table_dev || !start_dev || !end_dev || !scratch_dev) return TGP_E_INVAL;
    const auto bits = [](auto... p) { return (reinterpret_cast<uintptr_t>(p) | ...); };
    if ((bits(qb, k_pages, v_pages, ob, scratch_dev) & 15u) || (bits(table_dev, start_dev, end_dev) & 3u)) return TGP_E_INVAL;
    if (B > TGP_PAGED_MAX_B || cfg->max_len > 0x7fffffffu || T > 0x7fffffffu || cfg->Hq > (1u << 16) || (uint64_t)n_pages * cfg->TK > 0x7fffffffu ||
        (uint64_t)n_pages * cfg->TK * cfg->Hkv > 0x7fffff00u || (uint64_t)std::min(B, GROUP) * ((kv_max + 15) / 16) * cfg->Hkv > 0x7fffffffu) return TGP_E_TOO_LARGE;
    if (!B || !T || !q_max || !kv_max) return TGP_OK;
    q_max = std::min(q_max, T);
    const uint32_t G = cfg->Hq / cfg->Hkv;
    FewArgs f{};
    f.a = TgpPagedAttn{(const bf16 *)qb, (const bf16 *)k_pages, (const bf16 *)v_pages, (bf16 *)ob, table_dev, start_dev, end_dev, cfg->Hq, cfg->Hkv, G, cfg->TK,
                       cfg->max_len / cfg->TK + (cfg->max_len % cfg->TK != 0), B, T, q_max, kv_max, n_pages, window, window ? sinks : 0, 0, 1.4426950408889634f / sqrtf((float)cfg->Dh), 0};
    f.counters = (u64 *)scratch_dev;
    f.parts = (float *)((uint8_t *)scratch_dev + counter_bytes(cfg, B));
    // one tile of 16 rows where all sequences fit it, else two; sequences of more rows are the other kernel's
    const bool one = (uint64_t)q_max * G <= 16;
    f.a.few = one ? 16 : 32;
    if (int rc = cfg->Dh == 64 ? (one ? launch_few<64, 1>(f, (cudaStream_t)stream) : launch_few<64, 2>(f, (cudaStream_t)stream))
                               : (one ? launch_few<128, 1>(f, (cudaStream_t)stream) : launch_few<128, 2>(f, (cudaStream_t)stream))) return rc;
    if ((uint64_t)q_max * G <= f.a.few) return TGP_OK;
    return tgpk_attn_paged_many(f.a, cfg->Dh, (cudaStream_t)stream);
}
