// Drafted tokens verified against the target's distribution: accepted, or replaced by a token of what the target has more of than the draft.
//
// Row r of a sequence holds the target's logits x behind its r-th token, and the draft's logits y from which the next token d was drawn.  With p = softmax(x / t) and
// q = softmax(y / t), d is accepted where u q(d) < p(d); the first row whose token is not gives a token of max(p - q, 0), the last row (nothing is drafted behind it) one of p.  So the tokens are distributed as
// the target's own.
// Two kernels.  The first adds up exp((x - max) / t) of every row in parts, once through the logits; the second, a cluster of CTAs per sequence, joins the parts, finds the
// first row that refuses, adds up what may be drawn there by segments of the vocabulary and their units, and goes through the one unit that the random number falls into.
// The first kernel takes instructions and HBM in about equal parts: 32 sequences of up to five rows of 128256 logits with a draft's, 134 MB, some 38 us (HBM: 20; more than half of the issue slots).  Three operations
// in 64 bits and ten in 32 per weight instead of seven in 64 took as long, two CTAs of 384 threads an SM too; four of 256 took 2 % longer.  The second one takes 20 us of it, a chain: rows judged, one row of each sequence weighed from L2 or
// HBM, sums over the cluster, the token found.  Both 63.5 us (42.8 where the draft has no distribution, 16.6 where the likeliest tokens are asked for); one sequence, 32000 logits, 14.6 us.
// Of more than some 340 sequences the first kernel's 32 bytes each in shared memory leave two CTAs an SM instead of three, on the same grid: 336 -> 352 of up to two rows of 16000 logits with a draft's 47.6 -> 60.4 us.
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

constexpr uint32_t STAT_THREADS = 256, STAT_WARPS = STAT_THREADS / 32, PER_THREAD = 16, PART = STAT_THREADS * PER_THREAD, RING = 3;       // PART: logits of a part of a row
constexpr uint32_t DRAW_THREADS = 256, NW = DRAW_THREADS / 32, CLUSTER_MAX = 8, BATCH = 8, UNITS = 128;        // UNITS: of a warp's segment, at most
constexpr double LOG2E = 1.4426950408889634074;
constexpr int OCTAVE = 128, COPIES = 16, TABLE = OCTAVE * COPIES; // entries of the table of powers of two, and copies of it: a lane reads its own, without bank conflicts (with one, these took half of the time)

struct Stat { double sum; float top; uint32_t at; };             // of a part of a row: its weights, relative to the reference of its maximum; the maximum and its lowest index

struct VerifyArgs {
    const float *x, *y; const int32_t *tokens, *start; const float *u, *u_draw, *temperature; int32_t *out, *n_out;
    uint32_t B, T, V, parts, per, unit;                          // parts of a row in the first kernel; logits of a CTA in the second, and of a unit, 32 * BATCH at a time
    Stat *stats;                                                 // [2][T][parts]: target, draft
    double c[4];                                                 // of Weights
};

// Weights of logits, exp(x / t) relative to a reference near a maximum: with rate = OCTAVE log2(e) / t and the integer R nearest to top rate, x rate - R = n + f, |f| <= 1/2, and the weight is 2^(n / OCTAVE) 2^(f / OCTAVE),
// the former from a table (Tang's way of computing exponentials), the latter by its series to the third power, the fourth laid upon the others by its Chebyshev polynomial: off by 2^-41 of itself.  Seven
// operations in 64 bits, the addition to a sum among them; references differ by whole steps of the table, so sums are brought to another exactly.  Weights of less than some 2^-1000, of -inf and of NaN are 0.
struct Weights {
    double rate, shift;                                          // shift: MAGIC - R
    float top, low;                                              // the maximum, and what weighs something at least
    bool sharp;                                                  // no number but the maximum weighs anything: it is infinite, or the next one is hundreds of octaves away (so in others R is below 2^41)
    static constexpr double MAGIC = 6755399441055744.0;          // 1.5 * 2^52: a number plus this has its nearest integer in its low bits
    static constexpr double L = 0.69314718055994530942 / OCTAVE, Q = L * L * L * L / 24, C0 = 1.0 - Q / 128, C1 = L, C2 = L * L / 2 + Q / 4, C3 = L * L * L / 6;
    // span: 1000 OCTAVE / rate
    __device__ __forceinline__ Weights(float top, double rate, double span) : rate(rate), shift(MAGIC - rint((double)top * rate)), top(top) {
        low = (float)((double)top - span);
        sharp = !((double)top - (double)low >= 0.5 * span);
        low = fmaxf(low, -FLT_MAX);
    }
    // (entry k of the table is 2^(k / OCTAVE) with k << 13 taken from its upper half, so that n << 13 makes it 2^(n / OCTAVE); `table`: this lane's copy)
    static __device__ __forceinline__ double power(int n, const double *table) {
        const double o = table[(n & (OCTAVE - 1)) * COPIES];
        return __hiloint2double(__double2hiint(o) + (n << 13), __double2loint(o));
    }
    __device__ __forceinline__ void factors(float x, const double *table, double &p, double &series) const {
        const double d = (double)x, m = fma(d, rate, shift), f = fma(d, rate, shift - m);
        p = power(__double2loint(m), table);
        series = fma(f, fma(f, fma(f, C3, C2), C1), C0);
    }
    // the sum with a weight more (of a number below `low`: that of `low`), where the row is not sharp
    // (c: C0 ... C3 as arguments of the kernel, which an instruction takes as they are; literals were moved to registers for every weight)
    __device__ __forceinline__ double plus(double sum, float x, const double *table, const double (&c)[4]) const {
        const double d = (double)fmaxf(x, low), m = fma(d, rate, shift), f = fma(d, rate, shift - m);
        return fma(power(__double2loint(m), table), fma(f, fma(f, fma(f, c[3], c[2]), c[1]), c[0]), sum);
    }
    __device__ __forceinline__ double operator()(float x, const double *table) const {
        if (sharp) return x == top ? 1.0 : 0.0;
        double p, series;
        factors(fmaxf(x, low), table, p, series);
        return x >= low ? p * series : 0.0;
    }
    // a sum relative to the reference of another maximum, of this one's at most
    __device__ __forceinline__ double rescaled(double sum, float other, const double *table) const {
        if (sharp) return other == top ? sum : 0.0;
        return other >= low ? sum * power(__double2loint(rint((double)other * rate) + shift), table) : 0.0;
    }
};
// the same times a factor; equal logits, references and factors give equal numbers
struct Scaled {
    double rate, shift, c0, c1, c2, c3;
    float top, low;
    bool sharp;
    __device__ __forceinline__ void set(const Weights &w, double by) {
        rate = w.rate; shift = w.shift; top = w.top; low = w.low; sharp = w.sharp;
        c0 = w.sharp ? by : Weights::C0 * by; c1 = Weights::C1 * by; c2 = Weights::C2 * by; c3 = Weights::C3 * by;
    }
    template <uint32_t N> __device__ __forceinline__ void operator()(const float (&x)[N], double (&w)[N], const double *table) const {
        if (sharp) {
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) w[j] = x[j] == top ? c0 : 0.0;
            return;
        }
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) {
            const double d = (double)fmaxf(x[j], low), m = fma(d, rate, shift), f = fma(d, rate, shift - m);
            const double p = __dmul_rn(Weights::power(__double2loint(m), table), fma(f, fma(f, fma(f, c3, c2), c1), c0));
            w[j] = x[j] >= low ? p : 0.0;
        }
    }
};
static_assert(OCTAVE << 13 == 1 << 20, "n / OCTAVE is added to an exponent");
// the table, by the first threads of a CTA (a barrier follows); this lane's copy
__device__ __forceinline__ const double *fill_table(double *table) {
    if (threadIdx.x < OCTAVE) {
        const double o = exp2((double)threadIdx.x / OCTAVE), entry = __hiloint2double(__double2hiint(o) - ((int)threadIdx.x << 13), __double2loint(o));
#pragma unroll
        for (uint32_t i = 0; i < COPIES; ++i) table[threadIdx.x * COPIES + (i + threadIdx.x) % COPIES] = entry;
    }
    return table + threadIdx.x % COPIES;
}

// a sequence's first row and number of rows (none where they do not lie in the arrays), OCTAVE log2(e) / temperature, 0: the likeliest token, and 1000 octaves
struct Seq { uint32_t first, n; double rate, span; };
__device__ __forceinline__ Seq seq_of(const VerifyArgs &a, uint32_t b) {
    const int s0 = a.start[b], s1 = a.start[b + 1];
    const float t = a.temperature ? a.temperature[b] : 1.f;
    return {(uint32_t)s0, s0 < 0 || s1 <= s0 || (uint32_t)s1 > a.T ? 0u : (uint32_t)(s1 - s0), t > 0.f ? fmax(OCTAVE * LOG2E / (double)t, 1e-300) : 0.0, (double)t * (1000.0 / LOG2E)};
}
// A sequence has rows only from the highest start before its own on (of those in [0, T]).  So a row belongs to one sequence at most, whatever the device holds, and the line of all rows below has 2 T at most: its
// numbers of parts and costs, products in 32 bits, are bounded by the sizes that the call was checked with.
__device__ __forceinline__ uint32_t start_in(const VerifyArgs &a, uint32_t start) { return start > a.T ? 0u : start; }
constexpr uint32_t T_MAX = 32767, PARTS_MAX = (TGP_SAMPLE_MAX_V + PART - 1) / PART;
static_assert(2ull * 2 * T_MAX * PARTS_MAX < 1u << 31, "all parts' costs");

// The rows that the first kernel adds up, one line of them: of each sequence the target's, then the draft's that something was drawn from - none behind the last row, none where the likeliest token is taken.
// A part costs 1 where the likeliest token is asked for, else 2 (a part of weights took twice as long: with as many parts each, stretches of a mixed batch ended after 17 to 38 us).
struct LineSeq { Seq s; uint32_t upto, cost; };                  // of the sequences up to this one: rows, and rows times the cost of their parts
__device__ __forceinline__ uint32_t cost_of(const Seq &s) { return s.rate != 0.0 ? 2 : 1; }

// the first sequence whose value exceeds v
template <class F> __device__ __forceinline__ uint32_t first_above(uint32_t B, uint32_t v, F &&value) {
    uint32_t lo = 0, hi = B - 1;
    while (lo < hi) { const uint32_t mid = (lo + hi) / 2; if (value(mid) > v) hi = mid; else lo = mid + 1; }
    return lo;
}
// the first part, in the line of all, that begins at cost c or behind it
__device__ __forceinline__ uint32_t part_at(const LineSeq *line, uint32_t B, uint32_t parts, uint32_t c) {
    const uint32_t b = first_above(B, c / parts, [&](uint32_t i) { return line[i].cost; }), w = cost_of(line[b].s), rows = b ? line[b - 1].upto : 0, cost = b ? line[b - 1].cost : 0;
    return min(line[b].upto * parts, rows * parts + (c - cost * parts + w - 1) / w);
}

// A place in the line of all parts of these rows: part `part` of row k of sequence b, `left` of them up to a stretch's end.
struct Place {
    uint32_t b, k, part, left;
    __device__ __forceinline__ Place(const LineSeq *line, uint32_t B, uint32_t parts, uint32_t step, uint32_t left) : left(left) {
        const uint32_t row = step / parts;
        part = step - row * parts;
        b = first_above(B, row, [&](uint32_t i) { return line[i].upto; });
        k = row - (b ? line[b - 1].upto : 0);
    }
    __device__ __forceinline__ bool drafts(const LineSeq *line) const { return k >= line[b].s.n; }
    __device__ __forceinline__ uint32_t row(const LineSeq *line) const { const Seq &s = line[b].s; return s.first + (k < s.n ? k : k - s.n); }
    // true where another row begins
    __device__ __forceinline__ bool next(const LineSeq *line, uint32_t parts) {
        --left;
        if (++part < parts) return false;
        part = 0;
        ++k;
        if (left) while (line[b].upto - (b ? line[b - 1].upto : 0) <= k) { ++b; k = 0; }
        return true;
    }
};

__device__ __forceinline__ void cp_async(uint32_t dst, const float *src, bool wide) {
    if (wide) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// All parts of all rows are one line, of which a CTA takes a stretch.  A thread copies its logits of the next three parts to shared memory, in places that it alone reads, and no thread waits for another
// before a row's or the stretch's end, as each has a reference of its own: the maximum of its first logits, and another only where one lies hundreds of octaves above it.  The sum goes to the place of the
// row's first part in the stretch, the others are empty.  WIDE: rows that begin on 16 bytes, copied 16 at a time, else 4.
template <bool WIDE>
__global__ void __launch_bounds__(STAT_THREADS, 3) tgp_verify_stat_kernel(const VerifyArgs a) {
    __shared__ double table_of_all[TABLE], sh_s[2][STAT_WARPS];
    __shared__ float sh_m[2][STAT_WARPS];
    __shared__ uint32_t sh_i[2][STAT_WARPS], sh_start[STAT_WARPS];
    extern __shared__ __align__(16) float ring[];                // [RING][PART], then [B] sequences
    LineSeq *line = reinterpret_cast<LineSeq *>(ring + RING * PART);
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const double *table = fill_table(table_of_all);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");          // not before the wait: the draw's kernel reads the call's arguments without one of its own
    uint32_t rows = 0, cost = 0, highest = 0;
    for (uint32_t b0 = 0; b0 < a.B; b0 += STAT_THREADS) {
        Seq s{0, 0, 0.0, 0.0};
        uint32_t from = 0;
        if (b0 + tid < a.B) { s = seq_of(a, b0 + tid); from = start_in(a, s.first); }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const uint32_t v = __shfl_up_sync(0xffffffffu, from, o); if (lane >= o) from = max(from, v); }
        if (lane == 31) sh_start[warp] = from;
        __syncthreads();
        from = max(from, highest);
#pragma unroll
        for (uint32_t w = 0; w < STAT_WARPS; ++w) { if (w < warp) from = max(from, sh_start[w]); highest = max(highest, sh_start[w]); }
        if (s.first < from) s.n = 0;
        uint32_t upto = s.n + (s.n && a.y && s.rate != 0.0 ? s.n - 1 : 0);
        uint32_t costs = upto * cost_of(s);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o), c = __shfl_up_sync(0xffffffffu, costs, o); if (lane >= o) { upto += v; costs += c; } }
        if (lane == 31) { sh_i[0][warp] = upto; sh_i[1][warp] = costs; }
        __syncthreads();
        uint32_t all = 0, all_cost = 0;
#pragma unroll
        for (uint32_t w = 0; w < STAT_WARPS; ++w) { if (w < warp) { upto += sh_i[0][w]; costs += sh_i[1][w]; } all += sh_i[0][w]; all_cost += sh_i[1][w]; }
        if (b0 + tid < a.B) line[b0 + tid] = {s, rows + upto, cost + costs};
        rows += all;
        cost += all_cost;
        __syncthreads();
    }
    const uint32_t costs = cost * a.parts, ctas = min(gridDim.x, (costs + 1) / 2);
    if (blockIdx.x >= ctas) return;
    const uint32_t each = costs / ctas, longer = costs - each * ctas;
    auto begin_of = [&](uint32_t cta) { return cta == ctas ? rows * a.parts : part_at(line, a.B, a.parts, cta * each + min(cta, longer)); };
    const uint32_t lo = begin_of(blockIdx.x), steps = begin_of(blockIdx.x + 1) - lo;
    if (!steps) return;

    // element j of this thread: of four neighbours at a time, or of every 256th
    constexpr uint32_t W = WIDE ? 4 : 1;
    const uint32_t mine = tid * W;
    auto offset = [&](uint32_t j) { return j / W * (STAT_THREADS * W) + j % W; };
    const uint32_t ring_u = (uint32_t)__cvta_generic_to_shared(ring) + mine * 4;
    Place now(line, a.B, a.parts, lo, steps), ahead = now;
    auto logits_of = [&](const Place &p) { return (p.drafts(line) ? a.y : a.x) + (size_t)p.row(line) * a.V + mine; };
    const float *source = logits_of(ahead);
    uint32_t slot = 0;
    auto ask = [&](uint32_t to) {
        if (ahead.left) {
            const uint32_t at = ahead.part * PART, dst = ring_u + to * (PART * 4);
            const float *from = source + at;
            if (at + PART <= a.V) {
#pragma unroll
                for (uint32_t j = 0; j < PER_THREAD; j += W) cp_async(dst + offset(j) * 4, from + offset(j), WIDE);
            } else {
#pragma unroll
                for (uint32_t j = 0; j < PER_THREAD; j += W) if (at + mine + offset(j) < a.V) cp_async(dst + offset(j) * 4, from + offset(j), WIDE);
            }
            if (ahead.next(line, a.parts) && ahead.left) source = logits_of(ahead);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (uint32_t i = 0; i < RING - 1; ++i) ask(i);
    auto merge = [](float &m, uint32_t &at, float om, uint32_t oi) { if (om > m || (om == m && oi < at)) { m = om; at = oi; } };

    // of the row so far: this thread's reference, what a logit has to be above for another one, weights relative to it, and, where the likeliest token is asked for, the lowest index of the maximum
    float top = -INFINITY, limit = -INFINITY;
    uint32_t best = 0xffffffffu, set = 0;
    double sums[2] = {0.0, 0.0};
    Weights weight(0.f, 1.0, 1.0);
    bool plain = true;                                           // the row is not sharp, and what weighs nothing is told by the clamp
    uint32_t begin = now.part;                                   // the row's first part in the stretch
    double rate = line[now.b].s.rate, of_rate = line[now.b].s.span;
    while (now.left) {
        const uint32_t part = now.part, at = part * PART + mine;
        ask(slot == 0 ? RING - 1 : slot - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(RING - 1) : "memory");
        float x[PER_THREAD], m;
        const float *from = ring + slot * PART + mine;
        slot = slot + 1 == RING ? 0 : slot + 1;
#pragma unroll
        for (uint32_t j = 0; j < PER_THREAD; j += W) {
            if constexpr (WIDE) { const float4 v = *reinterpret_cast<const float4 *>(from + offset(j)); x[j] = v.x; x[j + 1] = v.y; x[j + 2] = v.z; x[j + 3] = v.w; }
            else x[j] = from[offset(j)];
        }
        if (at - mine + PART > a.V) {
#pragma unroll
            for (uint32_t j = 0; j < PER_THREAD; ++j) if (at + offset(j) >= a.V) x[j] = -INFINITY;
        }
        m = x[0];
#pragma unroll
        for (uint32_t j = 1; j < PER_THREAD; ++j) m = fmaxf(m, x[j]);
        if (m > limit) {
            if (rate == 0.0) {
#pragma unroll
                for (int j = PER_THREAD - 1; j >= 0; --j) if (x[j] == m) best = at + offset(j);
                limit = m;
            } else {
                const Weights higher(m, rate, of_rate);
                sums[0] = top > -INFINITY ? higher.rescaled(sums[0] + sums[1], top, table) : 0.0;
                sums[1] = 0.0;
                weight = higher;
                plain = !higher.sharp && higher.low > -FLT_MAX;
                limit = higher.sharp ? m : fminf((float)((double)m + 0.4 * of_rate), FLT_MAX);      // (an infinite one is above any)
            }
            top = m;
        }
        if (rate != 0.0 && top > -INFINITY) {
            if (plain) {
#pragma unroll
                for (uint32_t j = 0; j < PER_THREAD; ++j) sums[j % 2] = weight.plus(sums[j % 2], x[j], table, a.c);
            } else {                                             // (temperatures so high that the least number weighs something, or so low that the next one does not)
#pragma unroll
                for (uint32_t j = 0; j < PER_THREAD; ++j) sums[j % 2] += weight(x[j], table);
            }
        }
        Stat *place = a.stats + ((size_t)(now.drafts(line) ? a.T : 0) + now.row(line)) * a.parts + begin;
        const double r = rate, of_r = of_rate;
        if (!now.next(line, a.parts) && now.left) continue;
        if (now.left) { rate = line[now.b].s.rate; of_rate = line[now.b].s.span; }
        // ---- the row's or the stretch's end: of a warp, then of the CTA, the highest reference, and the sums relative to it ----
        const float own = top;
        double sum = sums[0] + sums[1];
#pragma unroll
        for (int o = 16; o; o >>= 1) { const float om = __shfl_xor_sync(0xffffffffu, top, o); const uint32_t oi = __shfl_xor_sync(0xffffffffu, best, o); merge(top, best, om, oi); }
        if (r != 0.0) sum = own > -INFINITY ? Weights(top, r, of_r).rescaled(sum, own, table) : 0.0;
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) { sh_m[set][warp] = top; sh_i[set][warp] = best; sh_s[set][warp] = sum; }
        __syncthreads();                                         // (two sets in turn: the next row's barrier is behind what is read here)
        if (tid == 0) {
            top = -INFINITY; best = 0xffffffffu; sum = 0.0;
            for (uint32_t w = 0; w < STAT_WARPS; ++w) merge(top, best, sh_m[set][w], sh_i[set][w]);
            if (r != 0.0 && top > -INFINITY) {
                const Weights highest(top, r, of_r);
                for (uint32_t w = 0; w < STAT_WARPS; ++w) if (sh_m[set][w] > -INFINITY) sum += highest.rescaled(sh_s[set][w], sh_m[set][w], table);
            }
            *place = {sum, top, top > -INFINITY ? best : 0};
        } else if (begin + tid <= part) place[tid] = {0.0, -INFINITY, 0xffffffffu};               // (a row has 128 parts at most)
        set ^= 1;
        top = limit = -INFINITY; best = 0xffffffffu;
        sums[0] = sums[1] = 0.0;
        begin = now.part;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}
// a row's parts (128 at most) joined, by a warp; the loads of two rows may be on their way together
struct Parts { Stat s[4]; };
__device__ __forceinline__ Parts load_parts(const Stat *s, uint32_t parts) {
    const uint32_t lane = threadIdx.x & 31;
    Parts p;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) { p.s[j] = {0.0, -INFINITY, 0xffffffffu}; if (lane + 32 * j < parts) p.s[j] = s[lane + 32 * j]; }
    return p;
}
__device__ __forceinline__ Stat join(const Parts &p, double rate, double span, const double *table) {
    auto merge = [](Stat &x, float top, uint32_t at) { if (top > x.top || (top == x.top && at < x.at)) { x.top = top; x.at = at; } };
    Stat all = p.s[0];
#pragma unroll
    for (uint32_t j = 1; j < 4; ++j) merge(all, p.s[j].top, p.s[j].at);
#pragma unroll
    for (int o = 16; o; o >>= 1) { const float om = __shfl_xor_sync(0xffffffffu, all.top, o); const uint32_t oi = __shfl_xor_sync(0xffffffffu, all.at, o); merge(all, om, oi); }
    all.sum = 0.0;
    if (__all_sync(0xffffffffu, all.top == -INFINITY)) { all.at = 0; return all; }                // (by all lanes: the shuffles below are of all, whatever a scratch that is not this call's alone may hold)
    if (rate != 0.0) {
        const Weights weight(all.top, rate, span);
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) all.sum += p.s[j].top > -INFINITY ? weight.rescaled(p.s[j].sum, p.s[j].top, table) : 0.0;
#pragma unroll
        for (int o = 16; o; o >>= 1) all.sum += __shfl_xor_sync(0xffffffffu, all.sum, o);
    }
    return all;
}

__device__ __forceinline__ uint32_t in_cta(const void *p, uint32_t rank) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return at;
}
__device__ __forceinline__ void put_f64(double *p, uint32_t rank, double v) { asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(in_cta(p, rank)), "d"(v) : "memory"); }

// Of n <= 128 sums: all, and the first at which the sum up to it exceeds the target - the last that is not 0, if rounding has it that none does -, with the sum before it; by a warp, in an order of its own.
struct Found { double sum, before; uint32_t at; };
__device__ __forceinline__ Found scan_of(const double *v, uint32_t n, double target) {
    const uint32_t lane = threadIdx.x & 31;
    double x[4], upto = 0.0;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) { x[j] = lane * 4 + j < n ? v[lane * 4 + j] : 0.0; upto += x[j]; }
    const double mine = upto;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const double y = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += y; }
    Found f{__shfl_sync(0xffffffffu, upto, 31), 0.0, 0};
    const uint32_t some = __ballot_sync(0xffffffffu, mine > 0.0), over = __ballot_sync(0xffffffffu, upto > target) & some;
    const int from = over ? __ffs(over) - 1 : some ? 31 - __clz(some) : 0;
    double before = upto - mine;
    uint32_t at = lane * 4;
    double at_before = before;
    bool hit = false;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
        if (x[j] > 0.0 && !hit) { at = lane * 4 + j; at_before = before; hit = before + x[j] > target; }
        before += x[j];
    }
    f.before = __shfl_sync(0xffffffffu, at_before, from);
    f.at = __shfl_sync(0xffffffffu, at, from);
    return f;
}

constexpr uint32_t KEPT = 32;                                    // rows that are judged at a time

__global__ void __launch_bounds__(DRAW_THREADS, 2) tgp_verify_draw_kernel(const VerifyArgs a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ bool sh_none[NW];                                 // (a warp each) a sequence before this one starts behind its first row
    __shared__ uint32_t sh_first, sh_n;                          // first row and rows, for the end
    __shared__ uint32_t sh_refused;                              // first row, counted from the sequence's first, whose token is not taken
    __shared__ Stat kept[2][KEPT];                               // target, draft
    __shared__ Scaled sh_w[2];
    __shared__ double table_of_all[TABLE];
    __shared__ double seg[CLUSTER_MAX * NW], sub[NW][UNITS];     // sums of the segments of the vocabulary, one per warp of the cluster, in every CTA; of this CTA's ones' units
    uint32_t rank, ctas;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, b = blockIdx.x / ctas;
    if (tid < CLUSTER_MAX * NW) seg[tid] = 0.0;
    cluster_arrive();                                            // (the first access to another CTA's memory waits for it to run)
    const double *table = fill_table(table_of_all);
    // what the sums are not needed for is read while the first kernel, which has waited for it, still runs (no rows: there is none)
    if (!a.T) asm volatile("griddepcontrol.wait;" ::: "memory");
    const Seq s = seq_of(a, b);
    if (tid == 0) { sh_refused = s.n ? s.n - 1 : 0; sh_first = s.first; sh_n = s.n; }
    // Does it begin before the start of one before it?  Then the first kernel has left its rows out, and nothing of their parts may be read.
    bool none = false;
    for (uint32_t i = tid; i < b; i += DRAW_THREADS) none |= start_in(a, (uint32_t)a.start[i]) > s.first;
    none = __any_sync(0xffffffffu, none);
    if (lane == 0) sh_none[warp] = none;
    __syncthreads();
    if (__any_sync(0xffffffffu, lane < NW && sh_none[lane])) {                  // (the same in every CTA of the cluster)
        asm volatile("griddepcontrol.wait;" ::: "memory");
        cluster_wait();
        if (rank == 0 && tid == 0) a.n_out[b] = 0;
        return;
    }
    // ---- which rows take their token, every CTA for itself: a warp joins a row of the target or of the draft, then a thread judges a row ----
    uint32_t group = 0;
    bool waited = false;
    for (; group < s.n; group += KEPT) {
        const uint32_t i = group + tid, r = s.first + i;         // (of the threads that judge)
        const bool judge = tid < KEPT && i + 1 < s.n, drawn = judge && a.y && s.rate != 0.0;
        const uint32_t d = judge ? (uint32_t)a.tokens[r + 1] : 0xffffffffu;
        const bool real = d < a.V && s.rate != 0.0;
        const float x_d = real ? a.x[(size_t)r * a.V + d] : 0.f, y_d = real && drawn ? a.y[(size_t)r * a.V + d] : 0.f;
        const double u = judge ? fmin(fmax((double)a.u[r], 0.0), 1.0) : 0.0;
        if (!waited) { asm volatile("griddepcontrol.wait;" ::: "memory"); waited = true; }
        for (uint32_t k = warp; k < 2 * KEPT; k += NW) {
            const uint32_t row = group + k / 2, draft = k % 2;
            if (row < s.n && !(draft && (row + 1 == s.n || !a.y || s.rate == 0.0))) {
                const Stat v = join(load_parts(a.stats + (size_t)(draft * a.T + s.first + row) * a.parts, a.parts), s.rate, s.span, table);
                if (lane == 0) kept[draft][k / 2] = v;
            }
        }
        __syncthreads();
        if (judge) {
            const Stat x = kept[0][tid], y = drawn ? kept[1][tid] : Stat{1.0, 0.f, 0};
            bool taken = d == x.at && x.top > -INFINITY;         // (the likeliest; a row of nothing takes none)
            if (s.rate != 0.0) {
                const double p = real && x.top > -INFINITY ? Weights(x.top, s.rate, s.span)(x_d, table) : 0.0;
                const double q = !drawn ? 1.0 : real && y.top > -INFINITY ? Weights(y.top, s.rate, s.span)(y_d, table) : 0.0;
                taken = u * q * x.sum < p * (y.sum > 0.0 ? y.sum : 1.0);     // (a draft's row of nothing: q is 0)
            }
            if (!taken) atomicMin(&sh_refused, i);
        }
        __syncthreads();
        if (sh_refused < group + KEPT) break;
    }
    if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t refused = sh_refused, r = s.first + refused;
    const bool last = refused + 1 == s.n, two = s.n && !last && a.y && s.rate != 0.0;
    const float top_x = s.n ? kept[0][refused - group].top : -INFINITY;
    const bool draw = s.n && s.rate != 0.0 && top_x > -INFINITY, minus = draw && two && kept[1][refused - group].sum > 0.0;
    if (lane == 0 && warp < 2 && (warp ? minus : draw)) {
        const Stat v = kept[warp][refused - group];
        sh_w[warp].set(Weights(v.top, s.rate, s.span), 1.0 / v.sum);
    }
    const uint32_t likeliest = s.n ? kept[0][refused - group].at : 0;
    const uint32_t d = s.n && !last && !a.y ? (uint32_t)a.tokens[r + 1] : 0xffffffffu;             // the token that was refused, where the draft's distribution is it alone
    __syncthreads();
    const Scaled wx = sh_w[0], wy = sh_w[1];
    const float *px = a.x + (size_t)(draw ? r : 0) * a.V, *py = a.y + (size_t)(minus ? r : 0) * a.V;
    const uint32_t first = min(a.V, rank * a.per), end = min(a.V, first + a.per), per_warp = (a.per + NW - 1) / NW;
    bool whole = last;                                           // the target's distribution as it is
    // what may be drawn of tokens i, i + 32, ... below hi: their logits, and their weights
    auto fetch = [&](auto &x, auto &y, uint32_t i, uint32_t hi) {
        constexpr uint32_t N = sizeof(x) / sizeof(float);
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) x[j] = i + j * 32 < hi ? px[i + j * 32] : -INFINITY;
        if (minus && !whole)
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) y[j] = i + j * 32 < hi ? py[i + j * 32] : -INFINITY;
    };
    auto rest = [&](const auto &x, const auto &y, auto &w, uint32_t i) {
        constexpr uint32_t N = sizeof(w) / sizeof(double);
        wx(x, w, table);
        if (minus && !whole) {
            double q[N];
            wy(y, q, table);
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) w[j] = fmax(__dsub_rn(w[j], q[j]), 0.0);
        } else if (!whole) {
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) if (i + j * 32 == d) w[j] = 0.0;
        }
    };
    // by a warp, unit by unit, of which each one's sum is kept, the next logits on their way while these are weighed
    auto total_of = [&](uint32_t lo, uint32_t hi) {
        double all = 0.0, sum = 0.0, w[BATCH];
        float x[BATCH], y[BATCH], next_x[BATCH], next_y[BATCH];
        fetch(next_x, next_y, lo + lane, hi);
        uint32_t n = 0, unit = 0;
        for (uint32_t i = lo + lane; i - lane < hi; i += 32 * BATCH) {
#pragma unroll
            for (uint32_t j = 0; j < BATCH; ++j) { x[j] = next_x[j]; y[j] = next_y[j]; }
            if (i - lane + 32 * BATCH < hi) fetch(next_x, next_y, i + 32 * BATCH, hi);
            rest(x, y, w, i);
            sum += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
            if (++n < a.unit && i - lane + 32 * BATCH < hi) continue;
#pragma unroll
            for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (lane == 0) sub[warp][unit] = sum;
            all += sum;
            sum = 0.0;
            n = 0;
            ++unit;
        }
        return all;
    };
    cluster_wait();
    int32_t token = (int32_t)likeliest;                           // the likeliest, or token 0 of a row of nothing but -inf and NaN
    if (s.rate != 0.0) token = 0;
    bool mine = rank == 0;                                       // this CTA writes the answer
    double sum = 0.0;
    for (int turn = 0; turn < 2; ++turn) {                       // (a second one where nothing is left of p - q)
        if (draw) {
            const uint32_t lo = min(end, first + warp * per_warp), hi = min(end, lo + per_warp);
            const double w = total_of(lo, hi);
            if (lane < ctas) put_f64(&seg[rank * NW + warp], lane, w);
        }
        cluster_sync_all();                                      // (also before a CTA leaves)
        if (draw) sum = scan_of(seg, CLUSTER_MAX * NW, 0.0).sum;  // (segments of CTAs that are not there are 0)
        const bool again = draw && turn == 0 && !(sum > 0.0) && !whole;                  // the same in every CTA
        if (!again) break;
        cluster_sync_all();                                      // (everyone has read the sums)
        whole = true;
    }
    if (draw) {
        double target = fmin(fmax((double)a.u_draw[b], 0.0), 1.0 - 0x1p-24) * sum;
        const Found in_row = scan_of(seg, CLUSTER_MAX * NW, target);
        const uint32_t found = in_row.at;
        target -= in_row.before;
        mine = found / NW == rank;
        if (!mine) return;
        // ---- the segment's warp: the unit, then the token that the rest of the target falls into ----
        if (found % NW != warp) return;
        const uint32_t lo = min(end, first + warp * per_warp), hi = min(end, lo + per_warp), tokens = a.unit * 32 * BATCH;
        const Found in_segment = scan_of(sub[warp], (hi - lo + tokens - 1) / tokens, target);
        target -= in_segment.before;
        const uint32_t m_lo = lo + in_segment.at * tokens, m_hi = min(hi, m_lo + tokens);
        if (!(sub[warp][in_segment.at] > target)) target = DBL_MAX;          // (rounding: the last token of the unit that weighs anything)
        double upto = 0.0;
        bool over = false;
        for (uint32_t i0 = m_lo; i0 < m_hi && !over; i0 += 32 * BATCH) {
            float x[BATCH], y[BATCH];
            double w[BATCH];
            fetch(x, y, i0 + lane, m_hi);
            rest(x, y, w, i0 + lane);
#pragma unroll 1
            for (uint32_t j = 0; j < BATCH && !over; ++j) {
                double v = w[0];
#pragma unroll
                for (uint32_t k = 0; k + 1 < BATCH; ++k) w[k] = w[k + 1];
                const uint32_t some = __ballot_sync(0xffffffffu, v > 0.0);
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) { const double before = __shfl_up_sync(0xffffffffu, v, o); if (lane >= o) v += before; }
                const uint32_t above = __ballot_sync(0xffffffffu, upto + v > target) & some;
                if (some) token = (int32_t)(i0 + j * 32 + (above ? __ffs(above) - 1 : 31 - __clz(some)));
                over = above != 0;
                upto += __shfl_sync(0xffffffffu, v, 31);
            }
        }
    } else if (!mine || warp) return;
    // ---- one warp writes the sequence's tokens ----
    const uint32_t out = sh_first, n = sh_n, taken = sh_refused;
    for (uint32_t i = lane; i < n; i += 32) a.out[out + i] = i < taken ? a.tokens[out + i + 1] : i == taken ? token : -1;
    if (lane == 0) a.n_out[b] = n ? (int32_t)(taken + 1) : 0;
}

uint32_t parts_of(uint32_t V) { return (V + PART - 1) / PART; }
static_assert(PARTS_MAX <= 128, "a warp joins a row's parts");

}  // namespace

extern "C" int tgp_k_verify_scratch_bytes(uint32_t T, uint32_t V, uint64_t *bytes) {
    if (!bytes || !V) return TGP_E_INVAL;
    if (V > TGP_SAMPLE_MAX_V || T > T_MAX) return TGP_E_TOO_LARGE;
    *bytes = std::max<uint64_t>(16, (uint64_t)2 * T * parts_of(V) * sizeof(Stat));
    return TGP_OK;
}

extern "C" int tgp_k_verify(const float *logits, const float *draft_logits, const int32_t *tokens_dev, const int32_t *start_dev, const float *u_dev, const float *u_draw_dev, int32_t *out_dev,
                            int32_t *n_out_dev, uint32_t B, uint32_t T, uint32_t V, const float *temperature_dev, void *scratch_dev, void *stream) {
    if (!logits || !tokens_dev || !start_dev || !u_dev || !u_draw_dev || !out_dev || !n_out_dev || !scratch_dev || !V) return TGP_E_INVAL;
    if (((reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(draft_logits) | reinterpret_cast<uintptr_t>(tokens_dev) | reinterpret_cast<uintptr_t>(start_dev) |
          reinterpret_cast<uintptr_t>(u_dev) | reinterpret_cast<uintptr_t>(u_draw_dev) | reinterpret_cast<uintptr_t>(out_dev) | reinterpret_cast<uintptr_t>(n_out_dev) |
          reinterpret_cast<uintptr_t>(temperature_dev)) & 3u) || (reinterpret_cast<uintptr_t>(scratch_dev) & 15u)) return TGP_E_INVAL;
    if (V > TGP_SAMPLE_MAX_V || T > T_MAX || B > TGP_PAGED_MAX_B) return TGP_E_TOO_LARGE;
    if (!B) return TGP_OK;
    uint32_t ctas = V > 4096 ? CLUSTER_MAX : 1;
    while (ctas > 1 && B * ctas > 2u * (uint32_t)tgpk_sms()) ctas /= 2;
    VerifyArgs a{logits, draft_logits, tokens_dev, start_dev, u_dev, u_draw_dev, temperature_dev, out_dev, n_out_dev, B, T, V, parts_of(V), (V + ctas - 1) / ctas, 0, (Stat *)scratch_dev, {Weights::C0, Weights::C1, Weights::C2, Weights::C3}};
    const uint32_t per_warp = (a.per + NW - 1) / NW;
    a.unit = (per_warp + UNITS * 32 * BATCH - 1) / (UNITS * 32 * BATCH);
    const uint64_t steps = (uint64_t)(draft_logits ? 2 * T : T) * a.parts;
    if (T) {
        const uintptr_t bits = reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(draft_logits) | (uintptr_t)V * 4;
        const size_t smem = RING * PART * 4 + B * sizeof(LineSeq), most = RING * PART * 4 + TGP_PAGED_MAX_B * sizeof(LineSeq);
        if (!tgpk_allow_smem<tgp_verify_stat_kernel<true>>(most) || !tgpk_allow_smem<tgp_verify_stat_kernel<false>>(most)) return TGP_E_CUDA;
        if (int rc = launch(bits & 15 ? tgp_verify_stat_kernel<false> : tgp_verify_stat_kernel<true>, dim3((uint32_t)std::min<uint64_t>(steps, 3 * tgpk_sms())), dim3(STAT_THREADS), smem,
                            (cudaStream_t)stream, 1, a)) return rc;
    }
    return launch(tgp_verify_draw_kernel, dim3(B * ctas), dim3(DRAW_THREADS), 0, (cudaStream_t)stream, ctas, a);
}
