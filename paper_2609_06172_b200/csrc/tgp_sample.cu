// The next token of every sequence by temperature, top-k, top-p and min-p from a given random number.
//
// Tokens are ordered by logit, the lower index first of equals; each filter keeps a beginning of that order, so what is kept is everything above
// a logit t and the first so many of those equal to t.  Nothing is sorted: t is found by histograms that narrow the bin in which it lies -
// first 2047 bins of 1 / 64 in (max - logit) / temperature, then equal ranges of the logits' bits, each 2048 times finer.
// A token weighs exp((logit - max) / temperature) as a whole number of 2^-44: sums of whole numbers are exact in any order, so the result does not
// depend on which thread adds first, and what is drawn is what sums in 64-bit floating point would draw but for borders nearer than
// about 1e-10 of the sum.  Tokens that round to 0 (31 below the maximum, in units of the temperature) are never drawn.
// A row belongs to a cluster of CTAs, each with a contiguous part of it; histograms and sums meet through distributed shared memory.
#include <cuda_runtime.h>
#include <algorithm>
#include <cstdint>
#include "tgp.h"
#include "tgp_kernels.h"
#include "tgp_launch.cuh"

namespace {

using namespace tgp_launch;

constexpr int THREADS = 512, NW = THREADS / 32;
constexpr uint32_t BINS = 2048, CLUSTER_MAX = 8;
constexpr double ONE = 17592186044416.0;                        // 2^44, the weight of the maximum
typedef unsigned long long u64;

struct SampleArgs {
    const float *logits, *u, *temperature, *top_p, *min_p; const int32_t *top_k; int32_t *out;
    uint32_t V, per;                                             // logits of a row, and of a CTA's part
};

// what the cluster's CTAs share lies in the first one
struct Shared {
    uint32_t cnt[BINS], lo[BINS], hi[BINS];                      // histogram of the CTA's part: tokens, and their weight in two words
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

__device__ __forceinline__ void cluster_sync() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_cta(const void *p, uint32_t rank) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return at;
}
__device__ __forceinline__ uint32_t get32(const uint32_t *p, uint32_t rank) { uint32_t v; asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(in_cta(p, rank)) : "memory"); return v; }
__device__ __forceinline__ void put32(uint32_t *p, uint32_t rank, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(in_cta(p, rank)), "r"(v) : "memory"); }
__device__ __forceinline__ void put64(u64 *p, uint32_t rank, u64 v) { asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(in_cta(p, rank)), "l"(v) : "memory"); }

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
    float top, step;                                             // the maximum; 64 / temperature
    double inv;                                                  // 1 / temperature
    // bin of a logit that is no NaN and above -inf; BINS - 1 and more weigh nothing
    __device__ __forceinline__ uint32_t bin(float x) const {
        if (x == top) return 0;
        const float z = (top - x) * step;
        return z < (float)(BINS - 1) ? (uint32_t)z : BINS - 1;   // (a NaN: infinity times 0)
    }
    __device__ __forceinline__ double weight(float x) const { return x == top ? 1.0 : exp(((double)x - (double)top) * inv); }
};
__device__ __forceinline__ u64 whole(double w) { return (u64)__double_as_longlong(fma(w, ONE, 4503599627370496.0)) & 0xfffffffffffffull; }      // 2^52 puts the point behind the last bit

__global__ void __launch_bounds__(THREADS) tgp_sample_kernel(const SampleArgs a) {
    pdl_enter();
    extern __shared__ __align__(16) uint8_t sample_sm[];
    Shared &sh = *reinterpret_cast<Shared *>(sample_sm);
    uint32_t rank, parts;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, b = blockIdx.x / parts;
    const float *row = a.logits + (size_t)b * a.V;
    const uint32_t first = min(a.V, rank * a.per), end = min(a.V, first + a.per);

    // ---- the maximum ----
    Row r;
    uint32_t best;
    {
        float m = -INFINITY;
        uint32_t at = 0;                                         // a row of nothing but -inf and NaN gives token 0, as the argmax does
        for (uint32_t i = first + tid; i < end; i += THREADS) { const float x = row[i]; if (x > m) { m = x; at = i; } }
        auto merge = [&](float om, uint32_t oi) { if (om > m || (om == m && oi < at)) { m = om; at = oi; } };
#pragma unroll
        for (int o = 16; o; o >>= 1) { const float om = __shfl_xor_sync(0xffffffffu, m, o); const uint32_t oi = __shfl_xor_sync(0xffffffffu, at, o); merge(om, oi); }
        if (lane == 0) { sh.warp_m[warp] = m; sh.warp_i[warp] = at; }
        cluster_sync();                                          // (and all CTAs run)
        if (tid == 0) {
            for (int w = 0; w < NW; ++w) merge(sh.warp_m[w], sh.warp_i[w]);
            put32(reinterpret_cast<uint32_t *>(&sh.top[rank]), 0, __float_as_uint(m));
            put32(&sh.top_i[rank], 0, at);
        }
        cluster_sync();
        m = -INFINITY; at = 0;
        for (uint32_t p = 0; p < parts; ++p) merge(__uint_as_float(get32(reinterpret_cast<const uint32_t *>(&sh.top[p]), 0)), get32(&sh.top_i[p], 0));
        r.top = m; best = at;
    }
    const float temperature = a.temperature ? a.temperature[b] : 1.f, min_p = a.min_p ? a.min_p[b] : 0.f, top_p = a.top_p ? a.top_p[b] : 1.f;
    const int32_t top_k = a.top_k ? a.top_k[b] : 0;
    if (!(temperature > 0.f) || r.top == -INFINITY || min_p > 1.f || top_k == 1) {               // the cluster's CTAs agree
        if (rank == 0 && tid == 0) a.out[b] = (int32_t)best;
        cluster_sync();
        return;
    }
    r.inv = 1.0 / (double)temperature;
    r.step = (float)fmin(64.0 * r.inv, 3.0e38);
    auto live = [&](float x) { return x > -INFINITY; };

    // ---- histogram of the tokens at or above key_lo, by bin (level 0) or by (key_hi - key) >> shift; the bin in which the need-th token (or
    // unit of weight) lies goes to the Shared of every CTA, in_n = 0 if there is none ----
    auto search = [&](bool level0, uint32_t key_lo, uint32_t key_hi, uint32_t shift, bool by_weight, u64 need) {
        for (uint32_t i = tid; i < BINS; i += THREADS) { sh.cnt[i] = 0; sh.lo[i] = 0; sh.hi[i] = 0; }
        __syncthreads();
        for (uint32_t i = first + tid; i < end; i += THREADS) {
            const float x = row[i];
            if (!live(x)) continue;
            const uint32_t key = key_of(x);
            if (key < key_lo || key > key_hi) continue;
            const uint32_t z = r.bin(x);
            if (z >= BINS - 1) continue;
            // (the highest keys first, as the bins of level 0)
            const uint32_t bin = level0 ? z : (key_hi - key) >> shift;
            atomicAdd(&sh.cnt[bin], 1u);
            const u64 w = whole(r.weight(x));
            const uint32_t lo = (uint32_t)w, old = atomicAdd(&sh.lo[bin], lo), hi = (uint32_t)(w >> 32) + (old + lo < old);
            if (hi) atomicAdd(&sh.hi[bin], hi);
        }
        cluster_sync();
        for (uint32_t i = rank * THREADS + tid; i < BINS; i += parts * THREADS) {
            uint32_t n = 0;
            u64 w = 0;
            for (uint32_t p = 0; p < parts; ++p) { n += get32(&sh.cnt[i], p); w += (u64)get32(&sh.lo[i], p) + ((u64)get32(&sh.hi[i], p) << 32); }
            put32(&sh.all_cnt[i], 0, n);
            put64(&sh.all_w[i], 0, w);
        }
        cluster_sync();
        if (rank == 0) {                                         // four bins a thread: sums of the threads before, then the bin where the need is met
            constexpr uint32_t PER = BINS / THREADS;
            uint32_t n = 0;
            u64 w = 0;
            for (uint32_t i = 0; i < PER; ++i) { n += sh.all_cnt[tid * PER + i]; w += sh.all_w[tid * PER + i]; }
            uint32_t n_to = warp_upto(n);
            u64 w_to = warp_upto(w);
            if (lane == 31) { sh.warp_t[warp] = n_to; sh.warp_w[warp] = w_to; }
            if (tid == 0) { sh.in_n = 0; sh.in_w = 0; }
            __syncthreads();
            for (uint32_t v = 0; v < warp; ++v) { n_to += sh.warp_t[v]; w_to += sh.warp_w[v]; }
            n_to -= n; w_to -= w;
            for (uint32_t i = 0; i < PER; ++i) {
                const uint32_t bn = sh.all_cnt[tid * PER + i];
                const u64 bw = sh.all_w[tid * PER + i], have = by_weight ? w_to : n_to, more = by_weight ? bw : bn;
                if (have < need && have + more >= need) { sh.bin = tid * PER + i; sh.before_n = n_to; sh.before_w = w_to; sh.in_n = bn; sh.in_w = bw; }
                n_to += bn; w_to += bw;
            }
            __syncthreads();
            if (tid == THREADS - 1) {                            // what all weigh
                sh.target = w_to;
                for (uint32_t p = 1; p < parts; ++p) {
                    put32(&sh.bin, p, sh.bin); put32(&sh.before_n, p, sh.before_n); put32(&sh.in_n, p, sh.in_n);
                    put64(&sh.before_w, p, sh.before_w); put64(&sh.in_w, p, sh.in_w); put64(&sh.target, p, sh.target);
                }
            }
        }
        cluster_sync();
    };

    uint32_t cut = 0, ties = 0xffffffffu;                        // kept: keys above cut, and the first `ties` tokens of that key
    u64 kept_w = 0;                                              // their weight, once a search has told
    auto narrow = [&](bool by_weight, u64 need) {
        search(true, cut, 0xffffffffu, 0, by_weight, need);
        if (sh.in_n == 0) { kept_w = sh.target; return; }        // fewer tokens than asked for: all
        u64 before_w = sh.before_w;
        u64 before = by_weight ? sh.before_w : sh.before_n;
        // the keys of the bin: the bins ascend where keys descend
        if (warp < 2) {                                          // warp 0: the lowest key with bin <= z; warp 1: the lowest with bin < z; 32 candidates at a time
            const uint32_t z = sh.bin;
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
        uint32_t key_lo = max(sh.key_lo, cut), key_hi = sh.key_hi, in_n = sh.in_n;
        u64 in_w = sh.in_w;
        __syncthreads();
        for (int level = 0; level < 4; ++level) {                // (32 bits at most, each search takes 11)
            // one token, or all that the bin holds: the cut is its lowest key (a lower cut found before keeps its ties)
            if (in_n == 1 || (!by_weight && need - before == in_n)) {
                if (key_lo > cut) { cut = key_lo; ties = 0xffffffffu; }
                kept_w = before_w + in_w;
                return;
            }
            if (key_lo == key_hi) {                              // equals: the first so many
                const u64 one = in_w / in_n, n = by_weight ? (need - before + one - 1) / one : need - before;
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
    if (top_p < 1.f) {
        if (kept_w == 0) { search(true, cut, 0xffffffffu, 0, true, ~0ull); kept_w = sh.target; __syncthreads(); }
        const double want = ceil(fmax((double)top_p, 0.0) * (double)kept_w);
        narrow(true, max(1ull, min(kept_w, (u64)want)));
    }

    // ---- the draw: sums of the warps' segments, in the order of the tokens ----
    const double least = min_p > 0.f ? (double)min_p : 0.0;
    auto segment = [&](uint32_t lo, uint32_t hi, u64 &w, uint32_t &t) {       // weight above the cut, and ties, of [lo, hi)
        w = 0; t = 0;
        for (uint32_t i = lo + lane; i < hi; i += 32) {
            const float x = row[i];
            if (!live(x)) continue;
            const uint32_t key = key_of(x);
            if (key < cut || r.bin(x) >= BINS - 1) continue;
            const double e = r.weight(x);
            if (!(e >= least)) continue;
            if (key == cut) ++t; else w += whole(e);
        }
        w = warp_total(w); t = warp_total(t);
    };
    const u64 tie_w = cut ? whole(r.weight(of_key(cut))) : 0;
    const uint32_t per_warp = (a.per + NW - 1) / NW, lo = min(end, first + warp * per_warp), hi = min(end, lo + per_warp);
    {
        u64 w; uint32_t t;
        segment(lo, hi, w, t);
        if (lane == 0) { put64(&sh.seg_w[rank * NW + warp], 0, w); put32(&sh.seg_t[rank * NW + warp], 0, t); }
    }
    cluster_sync();
    if (rank == 0 && tid == 0) {
        u64 sum = 0;
        uint32_t left = ties;
        for (uint32_t s = 0; s < parts * NW; ++s) { const uint32_t t = min(left, sh.seg_t[s]); left -= t; sum += sh.seg_w[s] + t * tie_w; }
        const double u = (double)a.u[b];
        u64 target = u > 0.0 ? (u64)fmin(u * (double)sum, 9.0e18) : 0;
        target = min(target, sum - 1);
        u64 before = 0;
        uint32_t seen = 0, s = 0;
        for (; s < parts * NW; ++s) {
            const uint32_t t = min(ties - min(ties, seen), sh.seg_t[s]);
            const u64 w = sh.seg_w[s] + t * tie_w;
            if (before + w > target) break;
            before += w;
            seen += sh.seg_t[s];
        }
        for (uint32_t p = 0; p < parts; ++p) { put32(&sh.seg, p, s); put64(&sh.target, p, target - before); put32(&sh.ties_before, p, seen); }
    }
    cluster_sync();
    if (sh.seg / NW == rank && sh.seg % NW == warp) {
        u64 target = sh.target;
        uint32_t seen = sh.ties_before;
        for (uint32_t i0 = lo; i0 < hi; i0 += 32) {
            const uint32_t i = i0 + lane;
            const float x = i < hi ? row[i] : -INFINITY;
            u64 w = 0;
            bool tie = false;
            if (live(x) && key_of(x) >= cut && r.bin(x) < BINS - 1) {
                const double e = r.weight(x);
                if (e >= least) { tie = key_of(x) == cut; w = whole(e); }
            }
            const uint32_t tie_mask = __ballot_sync(0xffffffffu, tie);
            if (tie && seen + __popc(tie_mask & ((1u << lane) - 1)) >= ties) w = 0;
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
}

}  // namespace

extern "C" int tgp_k_sample(const float *logits, const float *u_dev, int32_t *out, uint32_t B, uint32_t V, const float *temperature_dev, const int32_t *top_k_dev, const float *top_p_dev,
                            const float *min_p_dev, void *stream) {
    if (!logits || !u_dev || !out || !V) return TGP_E_INVAL;
    if (V > TGP_SAMPLE_MAX_V) return TGP_E_TOO_LARGE;
    if (!B) return TGP_OK;
    uint32_t parts = V > 4096 ? 8 : 1;
    while (parts > 1 && (uint64_t)B * parts > (uint32_t)tgpk_sms()) parts /= 2;
    if ((uint64_t)B * parts > 0x7fffffffu) return TGP_E_TOO_LARGE;
    if (!tgpk_allow_smem<tgp_sample_kernel>(sizeof(Shared))) return TGP_E_CUDA;
    const SampleArgs a{logits, u_dev, temperature_dev, top_p_dev, min_p_dev, top_k_dev, out, V, (V + parts - 1) / parts};
    return launch(tgp_sample_kernel, dim3(B * parts), dim3(THREADS), sizeof(Shared), (cudaStream_t)stream, parts, a);
}
