// Drafted tokens verified against the target's distribution: accepted, or replaced by a token of what the target has more of than the draft.
//
// Row r of a sequence holds the target's logits x behind its r-th token, and the draft's logits y from which the next token d was drawn.  With p = softmax(x / t) and
// q = softmax(y / t), d is accepted where u q(d) < p(d); the first row whose token is not gives a token of max(p - q, 0), the last row (nothing is drafted behind it) one of p.  So the tokens are distributed as
// the target's own.
// Two kernels.  The first adds up exp((x - max) / t) of every row in parts, once through the logits; the second, a cluster of CTAs per sequence, joins the parts, finds the
// first row that refuses, adds up what may be drawn there by segments of the vocabulary and goes through the one segment that the random number falls into.
// Weights and sums are in 64 bits: a draw is decided by sums over the vocabulary, and with 2^-24 in each weight one draw in some hundred thousand of flat rows would be another token than
// exact sums give.  All sums are in an order that depends on sizes alone.
#include <cuda_runtime.h>
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include "tgp.h"
#include "tgp_kernels.h"
#include "tgp_launch.cuh"
#include "tgp_sm100.cuh"

namespace {

using namespace tgp_launch;
using tgp_sm100::cluster_arrive; using tgp_sm100::cluster_sync_all; using tgp_sm100::cluster_wait;

constexpr uint32_t STAT_THREADS = 256, PER_THREAD = 32, PART = STAT_THREADS * PER_THREAD;       // logits of a CTA of the first kernel
constexpr uint32_t DRAW_THREADS = 512, NW = DRAW_THREADS / 32, CLUSTER_MAX = 8;
constexpr double LOG2E = 1.4426950408889634074;

struct Stat { double sum; float top; uint32_t at; };             // of a part of a row: weights relative to its maximum, the maximum, its lowest index

struct VerifyArgs {
    const float *x, *y; const int32_t *tokens, *start; const float *u, *u_draw, *temperature; int32_t *out, *n_out;
    uint32_t B, T, V, parts, per;                                // parts of a row in the first kernel; logits of a CTA in the second
    Stat *stats;                                                 // [2][T][parts]: target, draft
};

// 2^y for y <= 0: 2^n times the series of 2^f, |f| <= 1/2, whose eleventh term is below 2^-41 of it; 0 below 2^-1000
__device__ __forceinline__ double exp2_64(double y) {
    constexpr double MAGIC = 6755399441055744.0;                 // 1.5 * 2^52: a number plus this has its nearest integer in its low bits
    constexpr double L = 0.69314718055994530942, C2 = L * L / 2, C3 = C2 * L / 3, C4 = C3 * L / 4, C5 = C4 * L / 5, C6 = C5 * L / 6, C7 = C6 * L / 7, C8 = C7 * L / 8, C9 = C8 * L / 9, C10 = C9 * L / 10;
    const double m = y + MAGIC, f = y - (m - MAGIC);
    const double f2 = f * f, a = fma(f, C3, C2), b = fma(f, C5, C4), c = fma(f, C7, C6), d = fma(f, C9, C8), f4 = f2 * f2;
    const double p = fma(f, L, 1.0) + f2 * fma(f4, fma(f2, fma(f2, C10, d), c), fma(f2, b, a));
    return y < -1000.0 ? 0.0 : __hiloint2double(__double2hiint(p) + (__double2loint(m) << 20), __double2loint(p));
}
// weight of a logit in a row whose maximum is `top`; -inf and NaN weigh nothing, and the maximum 1, infinite or not
__device__ __forceinline__ double weight(float x, float top, double rate) {
    return !(x > -INFINITY) ? 0.0 : x == top ? 1.0 : exp2_64(((double)x - (double)top) * rate);
}

// a sequence's first row and number of rows (none where they do not lie in the arrays), and log2(e) / temperature, 0: the likeliest token
struct Seq { uint32_t first, n; double rate; };
__device__ __forceinline__ Seq seq_of(const VerifyArgs &a, uint32_t b) {
    const int s0 = a.start[b], s1 = a.start[b + 1];
    const float t = a.temperature ? a.temperature[b] : 1.f;
    return {(uint32_t)s0, s0 < 0 || s1 <= s0 || (uint32_t)s1 > a.T ? 0u : (uint32_t)(s1 - s0), t > 0.f ? LOG2E / (double)t : 0.0};
}

__global__ void __launch_bounds__(STAT_THREADS) tgp_verify_stat_kernel(const VerifyArgs a) {
    pdl_enter();
    __shared__ uint32_t sh_b;
    __shared__ float sh_m[STAT_THREADS / 32];
    __shared__ uint32_t sh_i[STAT_THREADS / 32];
    __shared__ double sh_s[STAT_THREADS / 32];
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, draft = blockIdx.y >= a.T, row = draft ? blockIdx.y - a.T : blockIdx.y, part = blockIdx.x;
    if (tid == 0) sh_b = 0xffffffffu;
    __syncthreads();
    for (uint32_t b = tid; b < a.B; b += STAT_THREADS) {         // the row's sequence
        const int s0 = a.start[b], s1 = a.start[b + 1];
        if (s0 >= 0 && (int)row >= s0 && (int)row < s1 && (uint32_t)s1 <= a.T) sh_b = b;
    }
    __syncthreads();
    if (sh_b == 0xffffffffu) return;
    const Seq s = seq_of(a, sh_b);
    if (draft && (row + 1 == s.first + s.n || s.rate == 0.0)) return;                    // nothing is drafted behind the last row, and the likeliest token needs no draft
    const float *from = (draft ? a.y : a.x) + (size_t)row * a.V;
    const uint32_t lo = part * PART;
    float x[PER_THREAD];
#pragma unroll
    for (uint32_t j = 0; j < PER_THREAD; ++j) { const uint32_t i = lo + j * STAT_THREADS + tid; x[j] = i < a.V ? from[i] : -INFINITY; }
    float m = -INFINITY;
    uint32_t at = 0;
#pragma unroll
    for (uint32_t j = 0; j < PER_THREAD; ++j) if (x[j] > m) { m = x[j]; at = lo + j * STAT_THREADS + tid; }
    auto merge = [](float &m, uint32_t &at, float om, uint32_t oi) { if (om > m || (om == m && oi < at)) { m = om; at = oi; } };
#pragma unroll
    for (int o = 16; o; o >>= 1) { const float om = __shfl_xor_sync(0xffffffffu, m, o); const uint32_t oi = __shfl_xor_sync(0xffffffffu, at, o); merge(m, at, om, oi); }
    if (lane == 0) { sh_m[warp] = m; sh_i[warp] = at; }
    __syncthreads();
    m = -INFINITY; at = 0xffffffffu;
#pragma unroll
    for (uint32_t w = 0; w < STAT_THREADS / 32; ++w) merge(m, at, sh_m[w], sh_i[w]);
    double sum = 0.0;
    if (s.rate != 0.0 && m > -INFINITY) {
#pragma unroll
        for (uint32_t j = 0; j < PER_THREAD; ++j) sum += weight(x[j], m, s.rate);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) sh_s[warp] = sum;
    __syncthreads();
    if (tid == 0) {
        sum = 0.0;
        for (uint32_t w = 0; w < STAT_THREADS / 32; ++w) sum += sh_s[w];
        a.stats[(size_t)blockIdx.y * a.parts + part] = {sum, m, m > -INFINITY ? at : 0};
    }
}

// a row's parts joined, by a warp
__device__ __forceinline__ Stat join(const Stat *s, uint32_t parts, double rate) {
    const uint32_t lane = threadIdx.x & 31;
    Stat all{0.0, -INFINITY, 0xffffffffu};
    for (uint32_t i = lane; i < parts; i += 32) if (s[i].top > all.top || (s[i].top == all.top && s[i].at < all.at)) { all.top = s[i].top; all.at = s[i].at; }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const float om = __shfl_xor_sync(0xffffffffu, all.top, o);
        const uint32_t oi = __shfl_xor_sync(0xffffffffu, all.at, o);
        if (om > all.top || (om == all.top && oi < all.at)) { all.top = om; all.at = oi; }
    }
    for (uint32_t i = lane; i < parts; i += 32) all.sum += s[i].sum * weight(s[i].top, all.top, rate);
#pragma unroll
    for (int o = 16; o; o >>= 1) all.sum += __shfl_xor_sync(0xffffffffu, all.sum, o);
    if (all.top == -INFINITY) all.at = 0;
    return all;
}

__device__ __forceinline__ uint32_t in_cta(const void *p, uint32_t rank) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return at;
}
__device__ __forceinline__ void put_f64(double *p, uint32_t rank, double v) { asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(in_cta(p, rank)), "d"(v) : "memory"); }

__global__ void __launch_bounds__(DRAW_THREADS) tgp_verify_draw_kernel(const VerifyArgs a) {
    pdl_enter();
    __shared__ uint32_t sh_refused;                              // first row, counted from the sequence's first, whose token is not taken
    __shared__ Stat sh_x, sh_y;                                  // of that row
    __shared__ double seg[CLUSTER_MAX * NW], sub[NW];            // sums of the segments of the vocabulary, one per warp of the cluster, in every CTA; of the parts of one
    uint32_t rank, ctas;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, b = blockIdx.x / ctas;
    cluster_arrive();                                            // (the first access to another CTA's memory waits for it to run)
    const Seq s = seq_of(a, b);
    if (tid == 0) sh_refused = s.n ? s.n - 1 : 0;
    __syncthreads();
    // ---- which rows take their token; every CTA for itself ----
    for (uint32_t i = warp; i + 1 < s.n; i += NW) {
        const uint32_t r = s.first + i, d = (uint32_t)a.tokens[r + 1];
        const Stat x = join(a.stats + (size_t)r * a.parts, a.parts, s.rate);
        bool taken;
        if (s.rate == 0.0) taken = d == x.at;
        else if (d >= a.V) taken = false;
        else {
            const double px = weight(a.x[(size_t)r * a.V + d], x.top, s.rate);
            double q = 1.0, sum_q = 1.0;
            if (a.y) {
                const Stat y = join(a.stats + (size_t)(a.T + r) * a.parts, a.parts, s.rate);
                q = weight(a.y[(size_t)r * a.V + d], y.top, s.rate);
                sum_q = y.sum > 0.0 ? y.sum : 1.0;               // (a row of nothing: q is 0)
            }
            const double u = fmin(fmax((double)a.u[r], 0.0), 1.0);
            taken = u * q * x.sum < px * sum_q;
        }
        if (!taken && lane == 0) atomicMin(&sh_refused, i);
    }
    __syncthreads();
    const uint32_t refused = sh_refused, r = s.first + refused;
    const bool last = refused + 1 == s.n;
    uint32_t d = 0xffffffffu;                                    // the token that was refused, where the draft's distribution is it alone
    if (s.n) {
        if (warp == 0) { const Stat v = join(a.stats + (size_t)r * a.parts, a.parts, s.rate); if (lane == 0) sh_x = v; }
        if (warp == 1 && !last && a.y && s.rate != 0.0) { const Stat v = join(a.stats + (size_t)(a.T + r) * a.parts, a.parts, s.rate); if (lane == 0) sh_y = v; }
        if (!last && !a.y) d = (uint32_t)a.tokens[r + 1];
    }
    __syncthreads();
    const Stat sx = s.n ? sh_x : Stat{0.0, -INFINITY, 0};
    const bool draw = s.n && s.rate != 0.0 && sx.top > -INFINITY;
    const bool minus = draw && !last && a.y && sh_y.sum > 0.0;
    const double inv_x = draw ? 1.0 / sx.sum : 0.0, inv_y = minus ? 1.0 / sh_y.sum : 0.0;
    const float top_y = minus ? sh_y.top : 0.f;
    const float *px = a.x + (size_t)(draw ? r : 0) * a.V, *py = a.y + (size_t)(minus ? r : 0) * a.V;
    const uint32_t first = min(a.V, rank * a.per), end = min(a.V, first + a.per), per_warp = (a.per + NW - 1) / NW;
    bool whole = last;                                           // the target's distribution as it is
    auto rest = [&](uint32_t i) {
        // (products that are rounded, both: equal ones leave nothing, where a fused multiply and subtract would leave a rounding)
        double w = __dmul_rn(weight(px[i], sx.top, s.rate), inv_x);
        if (!whole) w = minus ? fmax(__dsub_rn(w, __dmul_rn(weight(py[i], top_y, s.rate), inv_y)), 0.0) : i == d ? 0.0 : w;
        return w;
    };
    auto total_of = [&](uint32_t lo, uint32_t hi) {              // by a warp
        double w = 0.0;
        for (uint32_t i = lo + lane; i < hi; i += 32) w += rest(i);
#pragma unroll
        for (int o = 16; o; o >>= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
        return w;
    };
    cluster_wait();
    int32_t token = (int32_t)sx.at;                              // the likeliest, or token 0 of a row of nothing but -inf and NaN
    bool mine = rank == 0;                                       // this CTA writes the answer
    double sum = 0.0;
    for (int turn = 0; turn < 2; ++turn) {                       // (a second one where nothing is left of p - q)
        if (draw) {
            const uint32_t lo = min(end, first + warp * per_warp), hi = min(end, lo + per_warp);
            const double w = total_of(lo, hi);
            if (lane < ctas) put_f64(&seg[rank * NW + warp], lane, w);
        }
        cluster_sync_all();                                      // (also before a CTA leaves)
        sum = 0.0;
        if (draw) for (uint32_t i = 0; i < ctas * NW; ++i) sum += seg[i];
        const bool again = draw && turn == 0 && !(sum > 0.0) && !whole;                  // the same in every CTA
        if (!again) break;
        cluster_sync_all();                                      // (everyone has read the sums)
        whole = true;
    }
    if (draw) {
        double target = fmin(fmax((double)a.u_draw[b], 0.0), 1.0 - 0x1p-24) * sum;
        uint32_t found = 0;                                      // the segment into which it falls (rounding: the last that weighs anything)
        for (uint32_t i = 0; i < ctas * NW; ++i) if (seg[i] > 0.0) { found = i; if (seg[i] > target) break; target -= seg[i]; }
        mine = found / NW == rank;
        if (!mine) return;
        // ---- the segment, a sixteenth a warp, then the part that the rest of the target falls into ----
        const uint32_t lo = min(end, first + found % NW * per_warp), hi = min(end, lo + per_warp), per_part = (hi - lo + NW - 1) / NW;
        const uint32_t m_lo = min(hi, lo + warp * per_part), m_hi = min(hi, m_lo + per_part);
        const double w = total_of(m_lo, m_hi);
        if (lane == 0) sub[warp] = w;
        __syncthreads();
        uint32_t part = 0;
        for (uint32_t i = 0; i < NW; ++i) if (sub[i] > 0.0) { part = i; if (sub[i] > target) break; target -= sub[i]; }
        if (part != warp) return;
        if (!(sub[part] > target)) target = DBL_MAX;             // (rounding: the last token of the part that weighs anything)
        token = 0;
        double upto = 0.0;
        for (uint32_t i0 = m_lo; i0 < m_hi; i0 += 32) {
            double w = i0 + lane < m_hi ? rest(i0 + lane) : 0.0;
            const uint32_t some = __ballot_sync(0xffffffffu, w > 0.0);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const double v = __shfl_up_sync(0xffffffffu, w, o); if (lane >= o) w += v; }
            const uint32_t over = __ballot_sync(0xffffffffu, upto + w > target) & some;
            if (some) token = (int32_t)(i0 + (over ? __ffs(over) - 1 : 31 - __clz(some)));
            if (over) break;
            upto += __shfl_sync(0xffffffffu, w, 31);
        }
    } else if (!mine || warp) return;
    // ---- one warp writes the sequence's tokens ----
    for (uint32_t i = lane; i < s.n; i += 32) a.out[s.first + i] = i < refused ? a.tokens[s.first + i + 1] : i == refused ? token : -1;
    if (lane == 0) a.n_out[b] = s.n ? (int32_t)(refused + 1) : 0;
}

uint32_t parts_of(uint32_t V) { return (V + PART - 1) / PART; }

}  // namespace

extern "C" int tgp_k_verify_scratch_bytes(uint32_t T, uint32_t V, uint64_t *bytes) {
    if (!bytes || !V) return TGP_E_INVAL;
    if (V > TGP_SAMPLE_MAX_V || T > 32767) return TGP_E_TOO_LARGE;
    *bytes = std::max<uint64_t>(16, (uint64_t)2 * T * parts_of(V) * sizeof(Stat));
    return TGP_OK;
}

extern "C" int tgp_k_verify(const float *logits, const float *draft_logits, const int32_t *tokens_dev, const int32_t *start_dev, const float *u_dev, const float *u_draw_dev, int32_t *out_dev,
                            int32_t *n_out_dev, uint32_t B, uint32_t T, uint32_t V, const float *temperature_dev, void *scratch_dev, void *stream) {
    if (!logits || !tokens_dev || !start_dev || !u_dev || !u_draw_dev || !out_dev || !n_out_dev || !scratch_dev || !V) return TGP_E_INVAL;
    if (((reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(draft_logits) | reinterpret_cast<uintptr_t>(tokens_dev) | reinterpret_cast<uintptr_t>(start_dev) |
          reinterpret_cast<uintptr_t>(u_dev) | reinterpret_cast<uintptr_t>(u_draw_dev) | reinterpret_cast<uintptr_t>(out_dev) | reinterpret_cast<uintptr_t>(n_out_dev) |
          reinterpret_cast<uintptr_t>(temperature_dev)) & 3u) || (reinterpret_cast<uintptr_t>(scratch_dev) & 15u)) return TGP_E_INVAL;
    if (V > TGP_SAMPLE_MAX_V || T > 32767 || B > TGP_PAGED_MAX_B) return TGP_E_TOO_LARGE;
    if (!B) return TGP_OK;
    uint32_t ctas = V > 4096 ? CLUSTER_MAX : 1;
    while (ctas > 1 && B * ctas > 2u * (uint32_t)tgpk_sms()) ctas /= 2;
    const VerifyArgs a{logits, draft_logits, tokens_dev, start_dev, u_dev, u_draw_dev, temperature_dev, out_dev, n_out_dev, B, T, V, parts_of(V), (V + ctas - 1) / ctas, (Stat *)scratch_dev};
    if (T) if (int rc = launch(tgp_verify_stat_kernel, dim3(a.parts, draft_logits ? 2 * T : T), dim3(STAT_THREADS), 0, (cudaStream_t)stream, 1, a)) return rc;
    return launch(tgp_verify_draw_kernel, dim3(B * ctas), dim3(DRAW_THREADS), 0, (cudaStream_t)stream, ctas, a);
}
