// A KV cache in pages: which pages a sequence has and where a step's new positions lie, from the lengths of the sequences, and the append that
// rotates a step's rows and puts their keys and values there.
//
// tgp_page_plan_kernel: with P positions per page a sequence that keeps len positions and adds add wants ceil((len + add) / P) pages.  What it holds
// beyond that goes to the top of the stack of free pages, what it lacks comes from there; the places of the new rows are prefix sums of the sequences' counts.
//   Every CTA of the one cluster adds up all sequences for itself (two scans of a few hundred cycles), so nothing but the stack passes between
//   them: pages given back are written, the cluster meets, pages are taken and the rows' places written.  A row finds its sequence by bisection in shared
//   memory.  Bound by latency: a launch, a load of the counts, the scans, a load of the stack or the table, a store: 5.4 us for
//   61 sequences, 7.7 us for 512 with 65536 rows (from cold caches 7 and 10).
// tgp_rope_kv_paged_kernel: bound by HBM: 9285 rows of 64 + 8 heads of 128 take 85 us, 6.7 TB/s; 204 rows of 32 + 8 take 2.8 us behind their like, 5.8 from cold caches.
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <algorithm>
#include <cstdint>
#include <initializer_list>
#include "tgp.h"
#include "tgp_kernels.h"
#include "tgp_launch.cuh"
#include "tgp_sm100.cuh"

namespace {

using namespace tgp_launch;
using tgp_sm100::cluster_sync_all;
typedef __nv_bfloat16 bf16;
typedef unsigned long long u64;

// ---- the plan of a step -----------------------------------------------------------------------------------------------------------

constexpr uint32_t PLAN_THREADS = 1024, PLAN_WARPS = PLAN_THREADS / 32;

struct PlanArgs {
    const int32_t *len, *add; int32_t *table, *held, *free, *n_free, *start, *end, *slot, *pos;
    uint32_t B, P, W, max_len, n_pages, T, parts;
};

// of one sequence: pages that it had, wants, and how many rows the step may give it (0 where its lengths make no sense: then it keeps what it has)
struct Wish { uint32_t had, want, add; };
__device__ __forceinline__ Wish wish_of(const PlanArgs &a, uint32_t b) {
    const int len = a.len[b], add = a.add[b], held = a.held[b];
    Wish w;
    w.had = min((uint32_t)max(held, 0), a.W);
    const bool valid = len >= 0 && add >= 0 && (u64)(uint32_t)len + (uint32_t)add <= a.max_len;
    w.want = valid ? ((uint32_t)len + (uint32_t)add) / a.P + (((uint32_t)len + (uint32_t)add) % a.P != 0) : w.had;
    w.add = valid ? (uint32_t)add : 0;
    return w;
}

// Sums over the threads up to this one, and of all, that stay at the largest number once they reach it.
__device__ __forceinline__ uint32_t plus(uint32_t x, uint32_t y) { const uint32_t s = x + y; return s < x ? 0xffffffffu : s; }
template <uint32_t N> __device__ __forceinline__ void scan(uint32_t (&x)[N], uint32_t (&all)[N], uint32_t (&sh)[N][PLAN_WARPS]) {
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto up = [&](uint32_t (&v)[N]) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1)
#pragma unroll
            for (uint32_t k = 0; k < N; ++k) { const uint32_t y = __shfl_up_sync(0xffffffffu, v[k], o); if (lane >= o) v[k] = plus(v[k], y); }
    };
    up(x);
    __syncthreads();                                             // (what an earlier scan left has been read)
    if (lane == 31)
#pragma unroll
        for (uint32_t k = 0; k < N; ++k) sh[k][warp] = x[k];
    __syncthreads();
    uint32_t w[N];                                               // a lane per warp
#pragma unroll
    for (uint32_t k = 0; k < N; ++k) w[k] = sh[k][lane];
    up(w);
#pragma unroll
    for (uint32_t k = 0; k < N; ++k) {
        const uint32_t before = __shfl_sync(0xffffffffu, w[k], warp ? warp - 1 : 0);
        all[k] = __shfl_sync(0xffffffffu, w[k], 31);
        if (warp) x[k] = plus(x[k], before);
    }
}

__global__ void __launch_bounds__(PLAN_THREADS) tgp_page_plan_kernel(const PlanArgs a) {
    pdl_enter();
    extern __shared__ uint32_t plan_sm[];
    // of each sequence: pages that those before it have given back, and taken; rows before it; pages that it had, and wants; positions that it keeps
    uint32_t *given = plan_sm, *taken = given + a.B, *start = taken + a.B, *had = start + a.B + 1, *want = had + a.B, *kept = want + a.B;
    __shared__ uint32_t sums[3][PLAN_WARPS], some[2][PLAN_WARPS];
    const uint32_t tid = threadIdx.x, lane = tid & 31, rank = blockIdx.x, all = a.parts * PLAN_THREADS;
    const uint32_t stack = min((uint32_t)max(*a.n_free, 0), a.n_pages);

    // What the sequences of a thread wish, added up: pages given back, pages needed, rows asked for.  How many pages there are to take is known behind all that go back, so beyond PLAN_THREADS
    // sequences the wishes are gone through once more.
    u64 n_given = 0, need_sum = 0, add_sum = 0, n_taken = 0, rows = 0;
    Wish w{0, 0, 0};
    uint32_t x[3], sum[3];
    auto wish = [&](uint32_t b) {
        w = b < a.B ? wish_of(a, b) : Wish{0, 0, 0};
        x[0] = w.had > w.want ? w.had - w.want : 0;
        x[1] = w.want > w.had ? w.want - w.had : 0;
        x[2] = w.add;
        scan(x, sum, sums);
    };
    for (uint32_t b0 = 0; b0 < a.B; b0 += PLAN_THREADS) {
        const uint32_t b = b0 + tid;
        wish(b);
        // (beyond the stack's size it only has to stay there: no more pages fit it)
        if (b < a.B) { given[b] = (uint32_t)min((u64)0x7fffffffu, n_given + x[0] - (w.had > w.want ? w.had - w.want : 0)); had[b] = w.had; want[b] = w.want; kept[b] = (uint32_t)a.len[b]; }
        n_given += sum[0];
    }
    // (a stack that holds every page cannot grow: the numbers on the device are not trusted beyond the arrays)
    const uint32_t top = (uint32_t)min((u64)a.n_pages, (u64)stack + n_given);
    for (uint32_t b0 = 0; b0 < a.B; b0 += PLAN_THREADS) {
        const uint32_t b = b0 + tid;
        if (a.B > PLAN_THREADS) wish(b);
        const uint32_t need = w.want > w.had ? w.want - w.had : 0;
        const bool served = (!need || need_sum + x[1] <= top) && (!w.add || add_sum + x[2] <= a.T);
        need_sum += sum[1]; add_sum += sum[2];
        const uint32_t take = served ? need : 0, n = served ? w.add : 0;
        uint32_t y[2] = {take, n}, both[2];
        scan(y, both, some);
        if (b < a.B) { taken[b] = (uint32_t)n_taken + y[0] - take; start[b] = (uint32_t)rows + y[1] - n; }
        n_taken += both[0]; rows += both[1];
    }
    if (tid == 0) start[a.B] = (uint32_t)rows;
    __syncthreads();

    // ---- pages go back: the first of them to the top, so that a step taken back leaves the stack as it was ----
    for (uint32_t b = (rank * PLAN_THREADS + tid) / 32; b < a.B; b += all / 32) {
        int32_t *row = a.table + (size_t)b * a.W;
        for (uint32_t i = want[b] + lane; i < had[b]; i += 32) {
            const uint32_t k = given[b] + (i - want[b]);
            if (k < top) a.free[top - 1 - k] = row[i];
            row[i] = -1;
        }
    }
    if (a.parts > 1) cluster_sync_all();
    else __syncthreads();

    // ---- pages are taken; every sequence's counts ----
    for (uint32_t b = (rank * PLAN_THREADS + tid) / 32; b < a.B; b += all / 32) {
        const uint32_t n = start[b + 1] - start[b], before = had[b], next = b + 1 < a.B ? taken[b + 1] : (uint32_t)n_taken;
        const uint32_t take = next - taken[b];
        int32_t *row = a.table + (size_t)b * a.W;
        for (uint32_t i = lane; i < take; i += 32) row[before + i] = a.free[top - 1 - (taken[b] + i)];
        if (lane == 0) {
            a.held[b] = (int32_t)(want[b] < before ? want[b] : before + take);
            a.start[b] = (int32_t)start[b];
            a.end[b] = (int32_t)(kept[b] + n);
        }
    }
    if (rank == 0 && tid == 0) { a.start[a.B] = (int32_t)rows; *a.n_free = (int32_t)(top - (uint32_t)n_taken); }

    // ---- the rows' places ----
    for (uint32_t t = rank * PLAN_THREADS + tid; t < a.T; t += all) {
        int32_t pos = -1, slot = -1;
        if (t < (uint32_t)rows) {
            uint32_t lo = 0, hi = a.B;                           // the last sequence that begins at t or before: those without rows end where they begin
            while (hi - lo > 1) { const uint32_t mid = (lo + hi) / 2; if (start[mid] <= t) lo = mid; else hi = mid; }
            const uint32_t at = kept[lo] + (t - start[lo]), i = at / a.P;
            const int32_t page = i < had[lo] ? a.table[(size_t)lo * a.W + i] : a.free[top - 1 - (taken[lo] + (i - had[lo]))];
            pos = (int32_t)at;
            slot = page >= 0 && (uint32_t)page < a.n_pages ? page * (int32_t)a.P + (int32_t)(at - i * a.P) : -1;
        }
        a.pos[t] = pos;
        a.slot[t] = slot;
    }
}

// ---- append ------------------------------------------------------------------------------------------------------------------------

struct AppendArgs {
    const float *q32, *k32, *v32; bf16 *qb, *kp, *vp; const float *cos_t, *sin_t; const int32_t *slot, *pos;
    uint32_t Hq, Hkv, P, max_len, slots;
};

// The roundings of the append to KV tiles, so a position has the same bits in a page and in a tile.
__device__ __forceinline__ float rope_lo(float x0, float x1, float c, float s) { return __fmaf_rn(x0, c, -__fmul_rn(x1, s)); }
__device__ __forceinline__ float rope_hi(float x0, float x1, float c, float s) { return __fmaf_rn(x1, c, __fmul_rn(x0, s)); }
__device__ __forceinline__ uint2 bf16x4(float a, float b, float c, float d) {
    const __nv_bfloat162 lo = __floats2bfloat162_rn(a, b), hi = __floats2bfloat162_rn(c, d);
    return make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
}

// A thread takes four neighbouring dimensions of a head and their partners half a head away: two 16-byte loads, two 8-byte stores; a row's heads are spread over
// gridDim.y CTAs while the rows alone do not fill the GPU.
template <int DH>
__global__ void __launch_bounds__(256) tgp_rope_kv_paged_kernel(const AppendArgs a) {
    pdl_enter();
    constexpr uint32_t HALF = DH / 2, V = HALF / 4;              // items per head
    const uint32_t t = blockIdx.x;
    const int slot = a.slot[t], at = a.pos[t];
    if (slot < 0 || (uint32_t)slot >= a.slots || at < 0 || (uint32_t)at >= a.max_len) return;              // a row without a place
    const uint32_t page = (uint32_t)slot / a.P, off = (uint32_t)slot - page * a.P, qd = a.Hq * DH, kd = a.Hkv * DH;
    for (uint32_t idx = blockIdx.y * blockDim.x + threadIdx.x; idx < (a.Hq + 2 * a.Hkv) * V; idx += gridDim.y * blockDim.x) {
        const uint32_t h = idx / V, i = idx % V * 4;
        const bool rot = h < a.Hq + a.Hkv;
        const uint32_t hk = h < a.Hq ? h : rot ? h - a.Hq : h - a.Hq - a.Hkv;
        const float *s = (h < a.Hq ? a.q32 + (size_t)t * qd : (rot ? a.k32 : a.v32) + (size_t)t * kd) + hk * DH + i;
        float4 x0 = *reinterpret_cast<const float4 *>(s), x1 = *reinterpret_cast<const float4 *>(s + HALF);
        if (rot) {
            const float4 c = *reinterpret_cast<const float4 *>(a.cos_t + (size_t)at * HALF + i), sv = *reinterpret_cast<const float4 *>(a.sin_t + (size_t)at * HALF + i);
            const float4 y0 = x0, y1 = x1;
            x0 = make_float4(rope_lo(y0.x, y1.x, c.x, sv.x), rope_lo(y0.y, y1.y, c.y, sv.y), rope_lo(y0.z, y1.z, c.z, sv.z), rope_lo(y0.w, y1.w, c.w, sv.w));
            x1 = make_float4(rope_hi(y0.x, y1.x, c.x, sv.x), rope_hi(y0.y, y1.y, c.y, sv.y), rope_hi(y0.z, y1.z, c.z, sv.z), rope_hi(y0.w, y1.w, c.w, sv.w));
        }
        bf16 *o = (h < a.Hq ? a.qb + (size_t)t * qd + h * DH : (rot ? a.kp : a.vp) + (((size_t)page * a.Hkv + hk) * a.P + off) * DH) + i;
        *reinterpret_cast<uint2 *>(o) = bf16x4(x0.x, x0.y, x0.z, x0.w);
        *reinterpret_cast<uint2 *>(o + HALF) = bf16x4(x1.x, x1.y, x1.z, x1.w);
    }
}

bool unaligned(std::initializer_list<const void *> ps, uintptr_t mask) {
    uintptr_t bits = 0;
    for (const void *p : ps) bits |= reinterpret_cast<uintptr_t>(p);
    return (bits & mask) != 0;
}

}  // namespace

extern "C" int tgp_k_page_plan(const int32_t *len_dev, const int32_t *add_dev, int32_t *table_dev, int32_t *held_dev, int32_t *free_dev, int32_t *n_free_dev, int32_t *start_dev, int32_t *end_dev,
                               int32_t *slot_dev, int32_t *pos_dev, const tgp_model_cfg *cfg, uint32_t B, uint32_t n_pages, uint32_t T, void *stream) {
    if (!cfg || !cfg->TK || !cfg->max_len || B > cfg->B || !n_pages) return TGP_E_INVAL;
    if (!len_dev || !add_dev || !table_dev || !held_dev || !free_dev || !n_free_dev || !start_dev || !end_dev || !slot_dev || !pos_dev) return TGP_E_INVAL;
    if (B > TGP_PAGED_MAX_B || cfg->max_len > 0x7fffffffu || T > 0x7fffffffu || (uint64_t)n_pages * cfg->TK > 0x7fffffffu) return TGP_E_TOO_LARGE;
    if (unaligned({len_dev, add_dev, table_dev, held_dev, free_dev, n_free_dev, start_dev, end_dev, slot_dev, pos_dev}, 3)) return TGP_E_INVAL;
    PlanArgs a{len_dev, add_dev, table_dev, held_dev, free_dev, n_free_dev, start_dev, end_dev, slot_dev, pos_dev, B, cfg->TK, cfg->max_len / cfg->TK + (cfg->max_len % cfg->TK != 0), cfg->max_len,
               n_pages, T, 1};
    while (a.parts < 8 && T > a.parts * 4 * PLAN_THREADS) a.parts *= 2;
    const size_t smem = (6 * (size_t)B + 1) * 4;
    if (!tgpk_allow_smem<tgp_page_plan_kernel>((6 * (size_t)TGP_PAGED_MAX_B + 1) * 4)) return TGP_E_CUDA;
    return launch(tgp_page_plan_kernel, dim3(a.parts), dim3(PLAN_THREADS), smem, (cudaStream_t)stream, a.parts, a);
}

extern "C" int tgp_k_rope_kv_paged(const float *q32, const float *k32, const float *v32, void *qb, void *k_pages, void *v_pages, const float *cos_dev, const float *sin_dev, const int32_t *slot_dev,
                                   const int32_t *pos_dev, const tgp_model_cfg *cfg, uint32_t T, uint32_t n_pages, void *stream) {
    if (!cfg || (cfg->Dh != 64 && cfg->Dh != 128) || !cfg->Hkv || !cfg->Hq || cfg->Hq % cfg->Hkv || !cfg->TK || !cfg->max_len || !n_pages) return TGP_E_INVAL;
    if (!q32 || !k32 || !v32 || !qb || !k_pages || !v_pages || !cos_dev || !sin_dev || !slot_dev || !pos_dev) return TGP_E_INVAL;
    if (unaligned({q32, k32, v32, qb, k_pages, v_pages, cos_dev, sin_dev}, 15) || unaligned({slot_dev, pos_dev}, 3)) return TGP_E_INVAL;
    if (T > 0x7fffffffu || cfg->max_len > 0x7fffffffu || (uint64_t)n_pages * cfg->TK > 0x7fffffffu || cfg->Hq > (1u << 16)) return TGP_E_TOO_LARGE;
    if (!T) return TGP_OK;
    const AppendArgs a{q32, k32, v32, (bf16 *)qb, (bf16 *)k_pages, (bf16 *)v_pages, cos_dev, sin_dev, slot_dev, pos_dev, cfg->Hq, cfg->Hkv, cfg->TK, cfg->max_len, n_pages * cfg->TK};
    const uint32_t items = (cfg->Hq + 2 * cfg->Hkv) * (cfg->Dh / 8);
    const uint32_t split = std::max(1u, std::min((items + 255) / 256, 4u * (uint32_t)tgpk_sms() / T));
    return launch(cfg->Dh == 64 ? tgp_rope_kv_paged_kernel<64> : tgp_rope_kv_paged_kernel<128>, dim3(T, split), dim3(256), 0, (cudaStream_t)stream, 1, a);
}
