// The next token of every sequence by temperature, top-k, top-p and min-p from a given random number.
//
// Tokens are ordered by logit, the lower index first of equals; each filter keeps a beginning of that order, so what is kept is everything above
// a logit t and the first so many of those equal to t.
// A token weighs exp((logit - max) / temperature) as a whole number of 2^-44: sums of whole numbers are exact in any order, so the result does not
// depend on which thread adds first.  A weight is off by 2^-45 of the largest at most (and by the last bits of its exponential), a sum of V of them by V 2^-45: what is drawn is
// what sums in 64-bit floating point would draw but for borders nearer than that, 4e-9 of the largest weight at 128256 tokens and 1.5e-8 at the largest V.  Tokens
// that round to 0 (more than 31.2 below the maximum, in units of the temperature) are never drawn.
// A row belongs to a cluster of CTAs, each with a contiguous part of it, which is read once per step from memory, then from L2; histograms, lists and sums
// meet through distributed shared memory.  Steps, after the maximum:
//   top-k of a few hundred: the k-th largest of the threads' own maxima is a lower bound of the k-th largest logit.  What is not below its bin is a list
//     of little more than k tokens, which the first CTA sorts; it finishes the row by itself, and only these tokens' weights are ever computed;
//   else top-p: a histogram of the weights over 2047 bins of 1 / 64 in (max - logit) / temperature tells the bin in which t lies; its tokens are such a list;
//   where a list would be too long (equal logits, a large top-k): further histograms, each 2048 times finer in the logits' bits, down to one value;
//   the draw: sums of the kept weights by warp, in the order of the tokens, and the one segment that the random number falls into once more.
// Bound by instructions, not by the 4 B V bytes (5.0 us at 64 x 128256): us at 1 x 32000 and 64 x 128256: the maximum alone 2.9 and 6.0 (5.5 TB/s), no filter 7.8 and 26 (one sum of weights
// more: nine operations in fp64 and a conversion for each token that can be drawn), top-k of 50 11.1 and 19 (two passes that compute no weights), top-p of 0.9 21 and 62 (a weight and two atomics per
// token, then the weights of those above the bin once more); a top-k of 900 sorts its list, 34 and 60.  Eight CTAs per row where that fits two to an SM (four at 64 rows; eight there are
// slower).  A weight with a table of 32 entries, without bank conflicts, and two more terms: 28 instead of 26.
#include <cuda_runtime.h>
#include <algorithm>
#include <cstdint>
#include "tgp.h"
#include "tgp_kernels.h"
#include "tgp_launch.cuh"
#include "tgp_sm100.cuh"

namespace {

using namespace tgp_launch;
using tgp_sm100::cluster_arrive; using tgp_sm100::cluster_sync_all; using tgp_sm100::cluster_wait;

constexpr int THREADS = 512, NW = THREADS / 32;
constexpr uint32_t BINS = 2048, CLUSTER_MAX = 8, LIST = 2048, OCTAVE = 512;
constexpr double ONE = 17592186044416.0;                        // 2^44, the weight of the maximum
typedef unsigned long long u64;

struct SampleArgs {
    const float *logits, *u, *temperature, *top_p, *min_p; const int32_t *top_k; int32_t *out;
    uint32_t V, per;                                             // logits of a row, and of a CTA's part
};

// what the cluster's CTAs share lies in the first one
struct Shared {
    uint32_t cnt[BINS], lo[BINS], hi[BINS];                      // histogram of the CTA's part: tokens, and their weight in two words
    u64 list[LIST]; u64 sums[LIST];                              // tokens as key << 32 | ~index, and sums of their weights (first CTA)
    double octave[OCTAVE];                                       // 2^(44 + i / OCTAVE)
    uint32_t listed, counts[CLUSTER_MAX];                        // tokens that this CTA found, and each CTA
    uint32_t all_cnt[BINS]; u64 all_w[BINS];                     // of the row (first CTA)
    float top[CLUSTER_MAX]; uint32_t top_i[CLUSTER_MAX];         // the parts' maxima (first CTA)
    u64 seg_w[CLUSTER_MAX * NW]; uint32_t seg_t[CLUSTER_MAX * NW];      // the warps' sums and ties (first CTA)
    u64 warp_w[NW]; uint32_t warp_t[NW];
    float warp_m[NW]; uint32_t warp_i[NW];
    // result of a search: bin, tokens and weight before it and in it
    uint32_t bin, before_n, in_n; u64 before_w, in_w;
    uint32_t seg, ties_before; u64 target;
    uint32_t key_lo, key_hi;
};

__device__ __forceinline__ uint32_t in_cta(const void *p, uint32_t rank) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return at;
}
__device__ __forceinline__ uint32_t get32(const uint32_t *p, uint32_t rank) { uint32_t v; asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(in_cta(p, rank)) : "memory"); return v; }
__device__ __forceinline__ void put32(uint32_t *p, uint32_t rank, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(in_cta(p, rank)), "r"(v) : "memory"); }
__device__ __forceinline__ void put64(u64 *p, uint32_t rank, u64 v) { asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(in_cta(p, rank)), "l"(v) : "memory"); }


// additions to shared memory under a predicate, without a branch
__device__ __forceinline__ uint32_t atom_if(bool p, uint32_t at, uint32_t v) {
    uint32_t old = 0;
    asm volatile("{.reg .pred p; setp.ne.u32 p, %1, 0; @p atom.shared.add.u32 %0, [%2], %3;}" : "+r"(old) : "r"((uint32_t)p), "r"(at), "r"(v) : "memory");
    return old;
}
__device__ __forceinline__ void red_if_nonzero(uint32_t at, uint32_t v) { asm volatile("{.reg .pred p; setp.ne.u32 p, %1, 0; @p red.shared.add.u32 [%0], %1;}" ::"r"(at), "r"(v) : "memory"); }

template <typename T> __device__ __forceinline__ T warp_total(T v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <typename T> __device__ __forceinline__ T warp_upto(T v) {                      // inclusive
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const T w = __shfl_up_sync(0xffffffffu, v, o); if ((threadIdx.x & 31) >= o) v += w; }
    return v;
}

// numbers as unsigned integers of the same order; zeros of either sign are one
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

struct Row {
    float top, half, step, low;                                  // the maximum, and half of it; 128 / temperature; what is below weighs nothing (and is no NaN, nor -inf)
    double top64, rate;                                          // the maximum (0 where it is infinite); OCTAVE * log2(e) / temperature
    const double *octave;
    // bin of a logit that is no NaN and above -inf; those of BINS - 1 weigh nothing.  (Half of the difference: the whole may be more than fp32 holds.  Rounded by what 2^23 leaves of the
    // fraction, without a conversion.)
    __device__ __forceinline__ uint32_t bin(float x) const {
        const float z = x == top ? 0.f : fminf(fmaf(x, -0.5f, half) * step, (float)(BINS - 1));            // (fminf: a NaN, infinity times 0, is BINS - 1)
        return __float_as_uint(z + 8388608.f) & (BINS - 1);
    }
    // The weight of a logit not below `low` (of others: any number): with t = OCTAVE log2(e) (x - top) / temperature = n + f, |f| <= 1/2, it is 2^(n / OCTAVE)
    // exp(f ln2 / OCTAVE), the latter by its series, whose fourth power is below 2^-46, the former from a table (Tang's way of computing exponentials).  The last sum with 2^52 puts the point behind its last bit.
    __device__ __forceinline__ u64 weight(float x) const {
        constexpr double MAGIC = 6755399441055744.0;             // 1.5 * 2^52: a number plus this has its nearest integer in its low bits
        constexpr double C = 0.69314718055994530942 / OCTAVE;
        const double t = ((double)(top == INFINITY ? 0.f : x) - top64) * rate, m = t + MAGIC, f = t - (m - MAGIC);
        const int n = __double2loint(m);
        const double p = fma(f, fma(f, fma(f, C * C * C / 6, C * C / 2), C), 1.0), o = octave[n & (OCTAVE - 1)];
        const double scale = __hiloint2double((int)((uint32_t)__double2hiint(o) + (((uint32_t)n & ~(OCTAVE - 1)) << 11)), __double2loint(o));
        return (u64)__double_as_longlong(fma(p, scale, 4503599627370496.0)) & 0xfffffffffffffull;
    }
};
static_assert(OCTAVE << 11 == 1 << 20, "weight() adds n / OCTAVE to an exponent");

// Sorts the first n of a list of different numbers, the largest first; all threads of the CTA.  Up to 256 by counting, for each, those that are larger - a
// warp per number - else in a bitonic network over a power of two.
__device__ __forceinline__ void sort_list(u64 *list, uint32_t n) {
    __syncthreads();
    if (n <= 256) {
        const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        u64 x[8], mine = 0;
        uint32_t at = 0;
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) x[j] = j * 32 + lane < n ? list[j * 32 + lane] : 0;
        for (uint32_t i = warp, turn = 0; i < n; i += NW, ++turn) {
            const u64 y = list[i];
            uint32_t larger = 0;
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) if (j * 32 < n) larger += x[j] > y;
            larger = __reduce_add_sync(0xffffffffu, larger);
            if (turn == lane) { mine = y; at = larger; }
        }
        __syncthreads();
        if (warp + NW * lane < n) list[at] = mine;
        __syncthreads();
        return;
    }
    uint32_t size = 512;
    while (size < n) size *= 2;
    for (uint32_t i = n + threadIdx.x; i < size; i += THREADS) list[i] = 0;
    n = size;
    // (a warp's 32 pairs of a step with j <= 32 are 64 neighbours, which it alone touches in all such steps)
    __syncthreads();
    for (uint32_t k = 2; k <= n; k <<= 1)
        for (uint32_t j = k >> 1; j; j >>= 1) {
            if (j >= 64 || (j == 32 && k > 64)) __syncthreads();
            else __syncwarp();
            for (uint32_t i = threadIdx.x; i < n / 2; i += THREADS) {
                const uint32_t x = 2 * i - (i & (j - 1)), y = x + j;
                const u64 p = list[x], q = list[y];
                if ((p < q) == ((x & k) == 0)) { list[x] = q; list[y] = p; }
            }
        }
    __syncthreads();
}

__global__ void __launch_bounds__(THREADS, 2) tgp_sample_kernel(const SampleArgs a) {
    pdl_enter();
    extern __shared__ __align__(16) uint8_t sample_sm[];
    Shared &sh = *reinterpret_cast<Shared *>(sample_sm);
    uint32_t rank, parts;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, b = blockIdx.x / parts;
    const float *row = a.logits + (size_t)b * a.V;
    const uint32_t first = min(a.V, rank * a.per), end = min(a.V, first + a.per);

    cluster_arrive();                                            // (the first access to another CTA's memory waits for it to run)
    for (uint32_t i = tid; i < OCTAVE; i += THREADS) sh.octave[i] = ONE * exp2((double)i / OCTAVE);
    if (tid == 0) sh.listed = 0;
    for (uint32_t i = tid; i < BINS; i += THREADS) sh.cnt[i] = 0;

    // every logit of this CTA's part once, each thread every THREADS-th, eight loads under way; -inf behind the end; f has a thread's eight and the first one's index.
    // (Only the last eight are loaded with a look at the end, and they together: one by one behind the full ones, or all with a look, 1 x 32000 with no filter takes 9.1 instead of 7.8 us,
    // 64 x 128256 with top-p 71 instead of 61.)
    auto each_eight = [&](auto &&f) {
        for (uint32_t i = first; i < end; i += 8 * THREADS) {
            float x[8];
            const float *from = row + i + tid;
            if (end - i >= 8 * THREADS) {
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) x[j] = from[j * THREADS];
            } else {
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) x[j] = end - i > j * THREADS + tid ? from[j * THREADS] : -INFINITY;
            }
            f(x, i + tid);
        }
    };
    auto each = [&](auto &&f) {
        each_eight([&](const float (&x)[8], uint32_t i) {
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) f(x[j], i + j * THREADS);
        });
    };
    // a warp's logits of [lo, hi), 256 at a time, -inf behind the end: f has a lane's eight, every 32nd, and the first one's index
    auto by_eight = [&](uint32_t lo, uint32_t hi, auto &&f) {
        for (uint32_t i = lo; i < hi; i += 8 * 32) {
            float x[8];
            const float *from = row + i + lane;
            if (hi - i >= 8 * 32) {
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) x[j] = from[j * 32];
            } else {
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) x[j] = hi - i > j * 32 + lane ? from[j * 32] : -INFINITY;
            }
            f(x, i + lane);
        }
    };
    auto top_of = [](const float (&x)[8]) { return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7]))); };

    // ---- the maximum ----
    Row r;
    uint32_t best;
    float mine = -INFINITY;                                      // this thread's own
    {
        uint32_t at = 0;                                         // a row of nothing but -inf and NaN gives token 0, as the argmax does
        each([&](float x, uint32_t i) { if (x > mine) { mine = x; at = i; } });
        float m = mine;
        auto merge = [&](float om, uint32_t oi) { if (om > m || (om == m && oi < at)) { m = om; at = oi; } };
#pragma unroll
        for (int o = 16; o; o >>= 1) { const float om = __shfl_xor_sync(0xffffffffu, m, o); const uint32_t oi = __shfl_xor_sync(0xffffffffu, at, o); merge(om, oi); }
        if (lane == 0) { sh.warp_m[warp] = m; sh.warp_i[warp] = at; }
        cluster_wait();
        __syncthreads();
        if (warp == 0) {
            m = lane < NW ? sh.warp_m[lane] : -INFINITY;
            at = lane < NW ? sh.warp_i[lane] : 0xffffffffu;
#pragma unroll
            for (int o = NW / 2; o; o >>= 1) { const float om = __shfl_xor_sync(0xffffffffu, m, o); const uint32_t oi = __shfl_xor_sync(0xffffffffu, at, o); merge(om, oi); }
            if (lane < parts) { put32(reinterpret_cast<uint32_t *>(&sh.top[rank]), lane, __float_as_uint(m)); put32(&sh.top_i[rank], lane, at); }          // to every CTA
        }
        cluster_sync_all();
        m = -INFINITY; at = 0;
        for (uint32_t p = 0; p < parts; ++p) merge(sh.top[p], sh.top_i[p]);
        r.top = m; best = at;
    }
    const float temperature = a.temperature ? a.temperature[b] : 1.f, min_p = a.min_p ? a.min_p[b] : 0.f, top_p = a.top_p ? a.top_p[b] : 1.f;
    const int32_t top_k = a.top_k ? a.top_k[b] : 0;
    if (!(temperature > 0.f) || r.top == -INFINITY || min_p > 1.f || top_k == 1 || top_p <= 0.f) {               // the cluster's CTAs agree
        if (rank == 0 && tid == 0) a.out[b] = (int32_t)best;
        return;
    }
    const double inv = 1.0 / (double)fmaxf(temperature, 7.52316384526264e-37f);        // 2^-120: bins are told in fp32
    r.rate = inv * (OCTAVE * 1.4426950408889634074);
    r.step = (float)(128.0 * inv);
    r.half = 0.5f * r.top;
    r.top64 = (double)r.top;
    r.low = r.top == INFINITY ? INFINITY : fmaxf((float)(r.top64 - 33.0 / inv), -3.402823466e38f);
    r.octave = sh.octave;
    if (r.top == INFINITY) r.top64 = 0.0;
    const u64 least = min_p > 0.f ? (u64)ceil((double)min_p * ONE) : 0;
    const uint32_t per_warp = (a.per + NW - 1) / NW, lo = min(end, first + warp * per_warp), hi = min(end, lo + per_warp);      // this warp's segment of the row, for the draw

    // ---- the keys of a bin, as key_lo and key_hi of every CTA's Shared: bins ascend where keys descend.  Warp 0: the lowest key with bin <= z; warp 1: the lowest
    // with bin < z; 32 candidates at a time ----
    auto keys_of = [&](uint32_t z) {
        if (warp < 2) {
            u64 lo = 0, hi = (u64)key_of(r.top) + 1;             // the answer lies in [lo, hi]; hi: of warp 1 where the bin holds the maximum
            while (lo < hi) {
                const u64 step = (hi - lo + 31) / 32, k = lo + lane * step;
                const float x = of_key((uint32_t)k);
                const bool in = k < hi && !isnan(x) && x > -INFINITY && (warp == 0 ? r.bin(x) <= z : r.bin(x) < z);
                const uint32_t mask = __ballot_sync(0xffffffffu, in || k >= hi);                 // a beginning of zeros, then ones
                const uint32_t at = mask ? __ffs(mask) - 1 : 32;
                const u64 new_hi = at == 32 ? hi : min(hi, lo + at * step);
                lo = at == 0 ? new_hi : min(hi, lo + (at - 1) * step + 1);
                hi = new_hi;
            }
            if (lane == 0) { if (warp == 0) sh.key_lo = (uint32_t)hi; else sh.key_hi = (uint32_t)(hi - 1); }
        }
        __syncthreads();
    };
    // the lists that the CTAs have made, behind one another in the first one's; how many tokens they hold (more than LIST: there is no list)
    auto send_lists = [&]() {
        __syncthreads();
        const uint32_t n = sh.listed;
        if (tid < parts) put32(&sh.counts[rank], tid, n);
        cluster_sync_all();
        uint32_t before = 0, all = 0;
        for (uint32_t p = 0; p < parts; ++p) { if (p < rank) before += sh.counts[p]; all += sh.counts[p]; }
        if (rank && all <= LIST) for (uint32_t i = tid; i < n; i += THREADS) put64(&sh.list[before + i], 0, sh.list[i]);
        if (tid == 0) sh.listed = 0;
        cluster_sync_all();
        return all;
    };
    // ---- tokens whose key is in [key_lo, key_hi], which are those of numbers, as a list in the first CTA ----
    auto gather = [&](uint32_t key_lo, uint32_t key_hi) {
        const float x_lo = of_key(key_lo), x_hi = of_key(key_hi);
        each_eight([&](const float (&x)[8], uint32_t i) {
            if (!(top_of(x) >= x_lo)) return;
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j)
                if (x[j] >= x_lo && x[j] <= x_hi) {
                    const uint32_t at = atomicAdd(&sh.listed, 1u);
                    if (at < LIST) sh.list[at] = (u64)key_of(x[j]) << 32 | (uint32_t)~(i + j * THREADS);
                }
        });
        return send_lists();
    };
    // (first CTA) sorts n listed tokens, and gives the running sums of their weights: of their logits, or of the numbers in the low `bits`
    auto sorted_sums = [&](uint32_t n, uint32_t bits) {
        sort_list(sh.list, n);
        u64 before = 0;
        for (uint32_t i0 = 0; i0 < n; i0 += THREADS) {
            const uint32_t i = i0 + tid;
            u64 w = i >= n ? 0 : bits ? sh.list[i] & ((1ull << bits) - 1) : r.weight(of_key((uint32_t)(sh.list[i] >> 32)));
            w = warp_upto(w);
            if (lane == 31) sh.warp_w[warp] = w;
            __syncthreads();
            u64 all = 0;
            for (uint32_t v = 0; v < NW; ++v) { if (v < warp) w += sh.warp_w[v]; all += sh.warp_w[v]; }
            if (i < n) sh.sums[i] = before + w;
            before += all;
            __syncthreads();
        }
    };
    const double u = fmin(fmax((double)a.u[b], 0.0), 1.0);          // (a NaN is 0); of a row's 2^19 weights of 2^44 at most it is 2^63 at most
    auto draw = [&](u64 sum) { return min((u64)(u * (double)sum), sum - 1); };
    auto share = [&](u64 sum) { return max(1ull, min(sum, (u64)ceil((double)top_p * (double)sum))); };            // top_p of it

    // ---- top-k by the list of what is not below the k-th largest of the threads' maxima ----
    if (top_k > 0 && (uint32_t)top_k <= min(LIST / 2, parts * THREADS) && (uint32_t)top_k < a.V) {
        // (bins of eight: a histogram of 256, which every CTA adds up for itself)
        constexpr uint32_t EIGHT = BINS / 8;
        if (mine >= r.low) atomicAdd(&sh.cnt[r.bin(mine) / 8], 1u);
        cluster_sync_all();
        uint32_t n = 0, c[CLUSTER_MAX];
        if (tid < EIGHT) {
#pragma unroll
            for (uint32_t p = 0; p < CLUSTER_MAX; ++p) if (p < parts) c[p] = get32(&sh.cnt[tid], p);
#pragma unroll
            for (uint32_t p = 0; p < CLUSTER_MAX; ++p) if (p < parts) n += c[p];
        }
        uint32_t upto = warp_upto(n);
        if (lane == 31) sh.warp_t[warp] = upto;
        if (tid == 0) sh.bin = BINS - 2;                         // fewer maxima than k that weigh anything: whatever does
        __syncthreads();
        for (uint32_t v = 0; v < warp; ++v) upto += sh.warp_t[v];
        if (upto - n < (uint32_t)top_k && upto >= (uint32_t)top_k) sh.bin = min(tid * 8 + 7, BINS - 2);
        __syncthreads();
        keys_of(sh.bin);
        const uint32_t listed = gather(sh.key_lo, key_of(r.top));
        if (listed <= LIST) {
            if (rank) return;                                    // (nobody touches another CTA's memory any more)
            sorted_sums(listed, 0);
            uint32_t m = min(listed, (uint32_t)top_k);
            // how many of the first m have a running sum below the need, or a weight of `least` at least: weights fall, so either is a beginning
            auto count = [&](u64 need, bool weights) {
                uint32_t n = 0;
                for (uint32_t i = tid; i < m; i += THREADS) n += weights ? sh.sums[i] - (i ? sh.sums[i - 1] : 0) >= need : sh.sums[i] < need;
                n = __reduce_add_sync(0xffffffffu, n);
                if (lane == 0) sh.warp_t[warp] = n;
                __syncthreads();
                n = 0;
                for (uint32_t v = 0; v < NW; ++v) n += sh.warp_t[v];
                __syncthreads();
                return n;
            };
            if (top_p < 1.f) m = count(share(sh.sums[m - 1]), false) + 1;
            if (least) m = count(least, true);
            const u64 target = draw(sh.sums[m - 1]);
            // once more by index: the weight has 45 bits, the index below them is the order
            u64 packed[LIST / 2 / THREADS];
#pragma unroll
            for (uint32_t j = 0; j < LIST / 2 / THREADS; ++j) {
                const uint32_t i = j * THREADS + tid;
                packed[j] = i < m ? (u64)(TGP_SAMPLE_MAX_V - 1 - ~(uint32_t)sh.list[i]) << 45 | (sh.sums[i] - (i ? sh.sums[i - 1] : 0)) : 0;
            }
            __syncthreads();
#pragma unroll
            for (uint32_t j = 0; j < LIST / 2 / THREADS; ++j) if (j * THREADS + tid < m) sh.list[j * THREADS + tid] = packed[j];
            __syncthreads();
            sorted_sums(m, 45);
            for (uint32_t i = tid; i < m; i += THREADS)
                if ((i ? sh.sums[i - 1] : 0) <= target && sh.sums[i] > target) a.out[b] = (int32_t)(TGP_SAMPLE_MAX_V - 1 - (uint32_t)(sh.list[i] >> 45));
            return;
        }
    }

    // ---- histogram of the tokens at or above key_lo, by bin (level 0) or by (key_hi - key) >> shift; the bin in which the need-th token (or
    // unit of weight) lies goes to the Shared of every CTA, bin BINS if there is none, and what all weigh as `target`.  By weight, level 0 counts no tokens and
    // the need is top_p of all (of kept_w), which goes to `target` ----
    u64 kept_w = 0;                                              // what the tokens kept so far weigh, once a search has told
    uint32_t cut = 0, ties = 0xffffffffu;                        // kept: keys above cut, and the first `ties` tokens of that key
    bool summed = false;                                         // the first CTA has the segments' sums, and what is kept is in key_lo (the cut) and key_hi (ties)
    auto search = [&](bool level0, uint32_t key_lo, uint32_t key_hi, uint32_t shift, bool by_weight, u64 need) {
        for (uint32_t i = tid; i < BINS; i += THREADS) { sh.cnt[i] = 0; sh.lo[i] = 0; sh.hi[i] = 0; }
        auto add = [&](uint32_t bin, u64 w) {
            const uint32_t lo = (uint32_t)w, old = atomicAdd(&sh.lo[bin], lo), hi = (uint32_t)(w >> 32) + (old + lo < old);
            if (hi) atomicAdd(&sh.hi[bin], hi);
        };
        auto cta_total = [&](u64 w) {                            // of all threads
            w = warp_total(w);
            if (lane == 0) sh.warp_w[warp] = w;
            __syncthreads();
            w = 0;
            for (uint32_t v = 0; v < NW; ++v) w += sh.warp_w[v];
            __syncthreads();
            return w;
        };
        if (level0 && by_weight) {
            // What weighs less than w1 = (1 - top_p) * sum / V adds up to less than (1 - top_p) * sum, so t weighs w1 at least, and bins beyond are left out; the sum is at
            // least that of the threads' maxima (of this CTA: its bins go further than they need to)
            const float floor_x = cut ? fmaxf(r.low, of_key(cut)) : r.low;
            const u64 sum = max(kept_w ? kept_w : cta_total(mine >= r.low ? r.weight(mine) : 0), (u64)ONE);
            const float z1 = 64.f * logf((float)((double)a.V * ONE / ((1.0 - (double)top_p) * (double)sum))) + 2.f;
            const uint32_t last = z1 < (float)(BINS - 2) ? (uint32_t)fmaxf(z1, 0.f) : BINS - 2;
            __syncthreads();
            u64 all = 0;
            const uint32_t lo_at = (uint32_t)__cvta_generic_to_shared(sh.lo), hi_at = (uint32_t)__cvta_generic_to_shared(sh.hi);
            // four at a time: their weights, then their additions to the low words, then what those carry
            auto four = [&](const float (&x)[4]) {
                u64 w[4];
                uint32_t z[4], old[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    w[j] = r.weight(x[j]);
                    z[j] = x[j] >= floor_x ? r.bin(x[j]) : BINS;
                    all += z[j] < BINS ? w[j] : 0;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) old[j] = atom_if(z[j] <= last, lo_at + z[j] * 4, (uint32_t)w[j]);
#pragma unroll
                for (int j = 0; j < 4; ++j) red_if_nonzero(hi_at + z[j] * 4, z[j] <= last ? (uint32_t)(w[j] >> 32) + (old[j] + (uint32_t)w[j] < old[j]) : 0);
            };
            each_eight([&](const float (&x)[8], uint32_t) {
                four({x[0], x[1], x[2], x[3]});
                four({x[4], x[5], x[6], x[7]});
            });
            all = cta_total(all);
            if (tid == 0) put64(&sh.seg_w[rank], 0, all);
        } else {
        __syncthreads();
        each([&](float x, uint32_t) {
            if (!(x >= r.low)) return;
            const uint32_t key = key_of(x);
            if (key < key_lo || key > key_hi) return;
            const uint32_t z = r.bin(x);
            if (z >= BINS - 1) return;
            // (the highest keys first, as the bins of level 0)
            const uint32_t bin = level0 ? z : (key_hi - key) >> shift;
            atomicAdd(&sh.cnt[bin], 1u);
            add(bin, r.weight(x));
        });
        }
        cluster_sync_all();
        for (uint32_t i = rank * THREADS + tid; i < BINS; i += parts * THREADS) {
            uint32_t n = 0;
            u64 w = 0;
            uint32_t c[CLUSTER_MAX], l[CLUSTER_MAX], h[CLUSTER_MAX];
#pragma unroll
            for (uint32_t p = 0; p < CLUSTER_MAX; ++p) if (p < parts) { c[p] = get32(&sh.cnt[i], p); l[p] = get32(&sh.lo[i], p); h[p] = get32(&sh.hi[i], p); }
#pragma unroll
            for (uint32_t p = 0; p < CLUSTER_MAX; ++p) if (p < parts) { n += c[p]; w += (u64)l[p] + ((u64)h[p] << 32); }
            put32(&sh.all_cnt[i], 0, n);
            put64(&sh.all_w[i], 0, w);
        }
        cluster_sync_all();
        if (rank == 0) {                                         // four bins a thread: sums of the threads before, then the bin where the need is met
            constexpr uint32_t PER = BINS / THREADS;
            uint32_t n = 0;
            u64 w = 0;
            for (uint32_t i = 0; i < PER; ++i) { n += sh.all_cnt[tid * PER + i]; w += sh.all_w[tid * PER + i]; }
            uint32_t n_to = warp_upto(n);
            u64 w_to = warp_upto(w);
            if (lane == 31) { sh.warp_t[warp] = n_to; sh.warp_w[warp] = w_to; }
            if (tid == 0) { sh.in_n = 0; sh.in_w = 0; sh.bin = BINS; }
            __syncthreads();
            u64 total = 0;
            for (uint32_t v = 0; v < NW; ++v) { if (v < warp) { n_to += sh.warp_t[v]; w_to += sh.warp_w[v]; } total += sh.warp_w[v]; }
            n_to -= n; w_to -= w;
            if (level0 && by_weight) {
                total = 0;
                for (uint32_t p = 0; p < parts; ++p) total += sh.seg_w[p];
                need = share(kept_w ? kept_w : total);
            }
            for (uint32_t i = 0; i < PER; ++i) {
                const uint32_t bn = sh.all_cnt[tid * PER + i];
                const u64 bw = sh.all_w[tid * PER + i], have = by_weight ? w_to : n_to, more = by_weight ? bw : bn;
                if (have < need && have + more >= need) { sh.bin = tid * PER + i; sh.before_n = n_to; sh.before_w = w_to; sh.in_n = bn; sh.in_w = bw; }
                n_to += bn; w_to += bw;
            }
            __syncthreads();
            if (tid == 0) {
                sh.target = level0 && by_weight ? need : total;
                for (uint32_t p = 1; p < parts; ++p) {
                    put32(&sh.bin, p, sh.bin); put32(&sh.before_n, p, sh.before_n); put32(&sh.in_n, p, sh.in_n);
                    put64(&sh.before_w, p, sh.before_w); put64(&sh.in_w, p, sh.in_w); put64(&sh.target, p, sh.target);
                }
            }
        }
        cluster_sync_all();
    };

    auto narrow = [&](bool by_weight, u64 need) {
        search(true, cut, 0xffffffffu, 0, by_weight, need);
        if (sh.bin == BINS) { kept_w = sh.target; return; }      // fewer tokens than asked for: all
        if (by_weight) need = sh.target;
        u64 before_w = sh.before_w;
        u64 before = by_weight ? sh.before_w : sh.before_n;
        keys_of(sh.bin);
        uint32_t key_lo = max(sh.key_lo, cut), key_hi = sh.key_hi, in_n = sh.in_n;
        u64 in_w = sh.in_w;
        __syncthreads();
        if (by_weight) {
            // One pass lists the tokens of the bin and adds up the weights above it, by segment.  The first CTA sorts the list: the first token that reaches the need is the last
            // one kept, and those before it are added to their segments' sums.
            const float x_lo = of_key(key_lo), x_hi = of_key(key_hi);
            u64 w = 0;
            auto weigh = [&](float x) { const u64 e = r.weight(x); w += x > x_hi && e >= least ? e : 0; };
            auto list = [&](float x, uint32_t i) {
                if (x >= x_lo && x <= x_hi) { const uint32_t at = atomicAdd(&sh.listed, 1u); if (at < LIST) sh.list[at] = (u64)key_of(x) << 32 | (uint32_t)~i; }
            };
            by_eight(lo, hi, [&](const float (&x)[8], uint32_t i) {
                if (!__any_sync(0xffffffffu, top_of(x) >= x_lo)) return;
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) weigh(x[j]);
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) list(x[j], i + j * 32);
            });
            w = warp_total(w);
            if (lane == 0) { put64(&sh.seg_w[rank * NW + warp], 0, w); put32(&sh.seg_t[rank * NW + warp], 0, 0); }
            const uint32_t n = send_lists();
            if (n <= LIST) {
                summed = true;
                if (rank) return;
                sorted_sums(n, 0);
                for (uint32_t j = tid; j < n; j += THREADS)
                    if ((j ? sh.sums[j - 1] : 0) < need - before && sh.sums[j] >= need - before) {
                        const uint32_t key = (uint32_t)(sh.list[j] >> 32);
                        uint32_t same = 1;
                        for (uint32_t k = j; k && (uint32_t)(sh.list[k - 1] >> 32) == key; --k) ++same;
                        sh.bin = j;
                        for (uint32_t p = 0; p < parts; ++p) { put32(&sh.key_lo, p, key); put32(&sh.key_hi, p, same); }
                    }
                __syncthreads();
                for (uint32_t j = tid; j <= sh.bin; j += THREADS) {
                    const uint32_t i = ~(uint32_t)sh.list[j], part = i / a.per, seg = part * NW + (i - part * a.per) / per_warp;
                    const u64 e = sh.sums[j] - (j ? sh.sums[j - 1] : 0);
                    if (e < least) continue;
                    if ((uint32_t)(sh.list[j] >> 32) == sh.key_lo) atomicAdd(&sh.seg_t[seg], 1u); else atomicAdd(&sh.seg_w[seg], e);
                }
                __syncthreads();
                return;
            }
        }
        for (int level = 0; level < 4; ++level) {                // (32 bits at most, each search takes 11)
            // one token, or all that the bin holds: the cut is its lowest key (a lower cut found before keeps its ties)
            if (in_n == 1 || (!by_weight && need - before == in_n)) {            // (by weight, in_n is known from the second search on)
                if (key_lo > cut) { cut = key_lo; ties = 0xffffffffu; }
                kept_w = before_w + in_w;
                return;
            }
            if (key_lo == key_hi) {                              // equals: the first so many
                const u64 one = r.weight(of_key(key_lo)), n = by_weight ? (need - before + one - 1) / one : need - before;
                ties = (uint32_t)min((u64)(key_lo == cut ? ties : 0xffffffffu), n);
                cut = key_lo;
                kept_w = before_w + ties * one;
                return;
            }
            uint32_t shift = 0;
            while ((key_hi - key_lo) >> shift >= BINS) ++shift;
            search(false, key_lo, key_hi, shift, by_weight, need - before);
            before += by_weight ? sh.before_w : sh.before_n;
            before_w += sh.before_w;
            in_n = sh.in_n; in_w = sh.in_w;
            const uint32_t top_key = key_hi - (sh.bin << shift);
            key_lo = max(key_lo, top_key >= (1u << shift) - 1 ? top_key - ((1u << shift) - 1) : 0u);
            key_hi = top_key;
            __syncthreads();
        }
    };
    if (top_k > 0 && (uint32_t)top_k < a.V) narrow(false, (u64)top_k);
    if (top_p < 1.f) narrow(true, 0);

    // ---- the draw: sums of the warps' segments, in the order of the tokens ----
    float lowest, tie_x;                                         // no token below is kept; of the tokens of logit tie_x only the first so many are
    u64 tie_w;
    auto bounds = [&]() {
        if (summed) { ties = sh.key_lo == cut ? min(ties, sh.key_hi) : sh.key_hi; cut = sh.key_lo; }
        lowest = cut ? fmaxf(r.low, of_key(cut)) : r.low;
        tie_x = ties == 0xffffffffu ? NAN : lowest;
        tie_w = cut && ties != 0xffffffffu ? r.weight(of_key(cut)) : 0;
        // too far from the maximum for min_p (by more than what rounding the bound to fp32 takes)
        if (ties == 0xffffffffu && least) lowest = fmaxf(lowest, (float)(r.top64 + (log((double)min_p) - 1e-3) / inv) - fabsf(r.top) * 1e-6f);
    };
    // weight above the cut, and ties, of [lo, hi)
    auto counts = [&](float x, u64 &w, uint32_t &t) {
        const u64 e = r.weight(x);
        const bool kept = x >= lowest && e >= least, tie = kept && x == tie_x;
        w += kept && !tie ? e : 0;
        t += tie;
    };
    auto segment = [&](uint32_t lo, uint32_t hi, u64 &w, uint32_t &t) {
        w = 0; t = 0;
        by_eight(lo, hi, [&](const float (&x)[8], uint32_t) {
            // (few tokens are kept as a rule: none of 256 saves their weights, one of them costs eight a lane that do not wait for one another)
            if (!__any_sync(0xffffffffu, top_of(x) >= lowest)) return;
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) counts(x[j], w, t);
        });
        w = warp_total(w); t = warp_total(t);
    };
    if (!summed || rank == 0) bounds();
    if (!summed) {
        u64 w; uint32_t t;
        segment(lo, hi, w, t);
        if (lane == 0) { put64(&sh.seg_w[rank * NW + warp], 0, w); put32(&sh.seg_t[rank * NW + warp], 0, t); }
        cluster_sync_all();
    }
    if (rank == 0 && warp == 0) {                                // four segments a lane: ties before them, then weight before them
        constexpr uint32_t PER = CLUSTER_MAX * NW / 32;
        uint32_t t[PER], all = 0;
        u64 w[PER], sum = 0;
#pragma unroll
        for (uint32_t i = 0; i < PER; ++i) { t[i] = lane * PER + i < parts * NW ? sh.seg_t[lane * PER + i] : 0; all += t[i]; }
        uint32_t seen = warp_upto(all) - all;
#pragma unroll
        for (uint32_t i = 0; i < PER; ++i) {
            w[i] = (lane * PER + i < parts * NW ? sh.seg_w[lane * PER + i] : 0) + min(ties - min(ties, seen), t[i]) * tie_w;
            seen += t[i];
            sum += w[i];
        }
        u64 upto = warp_upto(sum);
        const u64 target = draw(__shfl_sync(0xffffffffu, upto, 31));
        seen -= all;
        upto -= sum;
#pragma unroll
        for (uint32_t i = 0; i < PER; ++i) {
            if (upto <= target && upto + w[i] > target)
                for (uint32_t p = 0; p < parts; ++p) { put32(&sh.seg, p, lane * PER + i); put64(&sh.target, p, target - upto); put32(&sh.ties_before, p, seen); }
            upto += w[i];
            seen += t[i];
        }
    }
    cluster_sync_all();
    if (summed && rank) bounds();
    // ---- the CTA of the segment: its warps take a sixteenth of it each, then the one into which the rest of the target falls goes through its part ----
    if (sh.seg / NW != rank) return;
    const uint32_t s_lo = min(end, first + sh.seg % NW * per_warp), s_hi = min(end, s_lo + per_warp), per_part = (s_hi - s_lo + NW - 1) / NW;
    const uint32_t m_lo = min(s_hi, s_lo + warp * per_part), m_hi = min(s_hi, m_lo + per_part);
    {
        u64 w; uint32_t t;
        segment(m_lo, m_hi, w, t);
        if (lane == 0) { sh.warp_w[warp] = w; sh.warp_t[warp] = t; }
    }
    __syncthreads();
    u64 target = sh.target;
    uint32_t seen = sh.ties_before;
    for (uint32_t v = 0; v < NW; ++v) {
        const u64 w = sh.warp_w[v] + min(ties - min(ties, seen), sh.warp_t[v]) * tie_w;
        if (target < w) { if (v != warp) return; break; }
        target -= w;
        seen += sh.warp_t[v];
    }
    for (uint32_t i0 = m_lo; i0 < m_hi; i0 += 32) {
        const uint32_t i = i0 + lane;
        u64 w = 0;
        uint32_t t = 0;
        if (i < m_hi) counts(row[i], w, t);
        const uint32_t tie_mask = __ballot_sync(0xffffffffu, t != 0);
        if (t && seen + __popc(tie_mask & ((1u << lane) - 1)) < ties) w = tie_w;
        const u64 upto = warp_upto(w);
        const uint32_t found = __ballot_sync(0xffffffffu, upto > target);
        if (found) {
            if (lane == __ffs(found) - 1) a.out[b] = (int32_t)i;
            break;
        }
        target -= __shfl_sync(0xffffffffu, upto, 31);
        seen += __popc(tie_mask);
    }
}

}  // namespace

extern "C" int tgp_k_sample(const float *logits, const float *u_dev, int32_t *out, uint32_t B, uint32_t V, const float *temperature_dev, const int32_t *top_k_dev, const float *top_p_dev,
                            const float *min_p_dev, void *stream) {
    if (!logits || !u_dev || !out || !V) return TGP_E_INVAL;
    if (V > TGP_SAMPLE_MAX_V) return TGP_E_TOO_LARGE;
    if (!B) return TGP_OK;
    uint32_t parts = V > 4096 ? 8 : 1;
    while (parts > 1 && (uint64_t)B * parts > 2u * (uint32_t)tgpk_sms()) parts /= 2;
    if ((uint64_t)B * parts > 0x7fffffffu) return TGP_E_TOO_LARGE;
    if (!tgpk_allow_smem<tgp_sample_kernel>(sizeof(Shared))) return TGP_E_CUDA;
    const SampleArgs a{logits, u_dev, temperature_dev, top_p_dev, min_p_dev, top_k_dev, out, V, (V + parts - 1) / parts};
    return launch(tgp_sample_kernel, dim3(B * parts), dim3(THREADS), sizeof(Shared), (cudaStream_t)stream, parts, a);
}
