// Attention of a ragged batch over a KV cache in pages: single tokens and a few drafted ones, on mma.sync; the entry point.  (Prompts: tgp_attn_paged_sm100.cu.)
//
// A page is [Hkv, P, DH] in bf16, so the P keys of one head of a page are one piece of memory.  Rows of a sequence and KV head - new tokens x query heads of the group, up to 16 MT - are the
// rows of m16n8k16 tiles; a warp takes 16 keys at a time, which it stages itself with cp.async three chunks deep, and keeps for each row a running maximum, the sum of the rounded
// weights and an unnormalised output in fp32:  p = 2^(s - m),  l += p,  O += p V,  and both times 2^(m - m') where the maximum grows to m'.  Weights are rounded to bf16 for the second
// product, and those that are summed are the rounded ones, so what is divided by is what the values were multiplied by.
//
// Split: all chunks of all sequences and KV heads are one line, of which every CTA takes a stretch: an equal one, or where there are CTAs enough one within a (sequence, KV head); lengths are known on the
// device only, so every CTA adds up the sequences' chunks for itself.  Where a stretch ends inside a (sequence, KV head), its CTA leaves (maximum, sum, output) in the scratch, and the last one to arrive at that pair's counter merges them
// all in the order of the stretches, so that results do not depend on who was last.
//
// What bounds it: HBM where contexts are long (24 of up to 12000 keys, 64 heads of 128 over 8: 106 us, 6.1 TB/s; 61 of up to 2500, 32 over 8: 63 us, 5.3 TB/s), else a fixed 3.5 us - a launch, the sequences'
// counts, table, keys, the merge in the CTA - and where CTAs share a context another 3 of their merge, each a chain of memory latencies, and with 17 to 32 rows the instructions (32 sequences of five tokens that see 1028 keys: 35 us, 0.56 of HBM's rate; 2500 keys without a window 51.6, 0.54).  A chunk's
// second tile of rows is multiplied even for sequences that have only one: leaving it out by a test was no faster.
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

constexpr uint32_t KEYS = 16, WARPS = 4, STAGES = 3, GROUP = 512;          // GROUP: sequences of a launch, which lie in shared memory
constexpr uint32_t MIN_STRETCH = 2 * WARPS;                                  // chunks
constexpr float LIFT = 16.f;
constexpr uint32_t ONES = 0x3f803f80u;                                       // two bf16
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void cp_async16_or_zeros(uint32_t dst, const void *src, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
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
__device__ __forceinline__ uint32_t bf16x2(float a, float b) { const __nv_bfloat162 h = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const uint32_t *>(&h); }
__device__ __forceinline__ bool not_finite2(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }

template <int DH> __host__ __device__ constexpr uint32_t stage_bytes() { return 2 * KEYS * DH * 2; }
template <int DH, int MT> __host__ __device__ constexpr uint32_t q_bytes() { return MT > 1 ? MT * 16 * DH * 2 : 0; }
template <int DH, int MT> __host__ __device__ constexpr uint32_t fixed_smem() { return WARPS * STAGES * stage_bytes<DH>() + q_bytes<DH, MT>() + WARPS * 16 * 2 * 4 + 64 + 256; }
template <int DH, int MT> __host__ __device__ constexpr uint32_t slot_floats() { return MT * 16 * (DH + 2); }

struct FewArgs {
    TgpPagedAttn a; float *parts; u64 *counters;
    bool beside;                                                            // launched behind the prompts' kernel of the same call
    uint32_t magic, shift;                                                  // a chunk's page: chunk * magic >> shift (chunks are below 2^27)
    uint32_t per_token;                                                     // a row's token: row * per_token >> 16 (rows are below 32)
    __device__ __forceinline__ uint32_t page_of_chunk(uint32_t chunk) const { return (uint32_t)((u64)chunk * magic >> shift); }
};

template <int DH, int MT>
__global__ void __launch_bounds__(WARPS * 32, DH == 128 ? 2 : MT == 1 ? 4 : 3) tgp_attn_paged_few_kernel(const FewArgs f) {
    // Beside the prompts' kernel: it is launched once that one has waited for what both read, and their rows are different ones.  Then it waits only before it ends, so that its successor waits for both.
    // (Between other kernels, one after the other -> beside: eight sequences, two of them chunks of 100 tokens, 38 -> 27 us; twelve, two of 509, 70 -> 71; 96, sixteen of 40, 125 -> 128; prompts alone
    // 188 -> 189.  From cold caches 46 -> 31, 78 -> 72, 127 -> 120 and 207 -> 201.)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (!f.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
    const TgpPagedAttn &a = f.a;
    extern __shared__ __align__(16) uint8_t few_raw[];
    uint8_t *few_sm = few_raw + (-(uint32_t)__cvta_generic_to_shared(few_raw) & 255u);       // stages begin on 256 bytes
    constexpr uint32_t ROW = DH * 2, CPR = ROW / 16, KV_BYTES = KEYS * ROW, STAGE = stage_bytes<DH>();
    uint8_t *q_sm = few_sm + WARPS * STAGES * STAGE;
    float *ml = reinterpret_cast<float *>(q_sm + q_bytes<DH, MT>());       // [WARPS][16][2]: maxima and sums of the warps' partials
    uint32_t *shared_u = reinterpret_cast<uint32_t *>(ml + WARPS * 16 * 2);
    uint4 *seqs = reinterpret_cast<uint4 *>(shared_u + 16);                 // [B] first row, rows, length, and chunks of the sequences up to this one, all KV heads
    uint32_t *upto = reinterpret_cast<uint32_t *>(seqs + a.B);              // [B] stretches of up to `unit` chunks of the sequences up to this one, none of which crosses from one KV head to another
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, c = lane & 3;

    // ---- the line of all chunks ----
    uint32_t own = 0;                                                       // chunks of an item of the thread's (last) sequence
    {
        uint32_t before = 0, before_u = 0;
        for (uint32_t i0 = 0; i0 < a.B; i0 += WARPS * 32) {
            const uint32_t i = i0 + tid;
            uint32_t mine = 0, mine_u = 0;
            TgpPagedSeq s{0, 0, 0, false};
            if (i < a.B) {
                s = tgp_paged_seq(a, a.b0 + i);
                if (s.n && !s.idle && s.n * a.G <= a.few) { own = mine = tgp_paged_keys<KEYS>(a, s.end - s.n, s.end - 1).chunks; mine_u = (mine + MIN_STRETCH - 1) / MIN_STRETCH * a.Hkv; mine *= a.Hkv; }
                else if (s.n && s.idle)                                     // rows of idle sequences are zero
                    for (u64 e = blockIdx.x; e < (u64)s.n * a.Hq * DH / 8; e += gridDim.x) reinterpret_cast<uint4 *>(a.o + (size_t)s.first * a.Hq * DH)[e] = make_uint4(0, 0, 0, 0);
            }
            uint32_t x = mine, x_u = mine_u;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const uint32_t y = __shfl_up_sync(0xffffffffu, x, o), y_u = __shfl_up_sync(0xffffffffu, x_u, o); if (lane >= o) { x += y; x_u += y_u; } }
            if (lane == 31) { shared_u[warp] = x; shared_u[WARPS + warp] = x_u; }
            __syncthreads();
            uint32_t all = 0, all_u = 0;
#pragma unroll
            for (uint32_t w = 0; w < WARPS; ++w) { if (w < warp) { x += shared_u[w]; x_u += shared_u[WARPS + w]; } all += shared_u[w]; all_u += shared_u[WARPS + w]; }
            if (i < a.B) { seqs[i] = make_uint4(s.first, s.n, s.end, before + x); upto[i] = before_u + x_u; }
            before += all;
            before_u += all_u;
            __syncthreads();
        }
    }
    // Where the CTAs suffice for stretches that each lie within an item, they do: one that crosses is two chains of merges one after the other (one sequence of 700 keys, 8 KV heads of 64, 9.4 -> 6.8 us; of 20 keys 7.5 -> 3.5).
    // Longer contexts, as long as no stretch is more than eight chunks longer than an equal share (one sequence of 16000 keys 19.7 -> 17.4 us, five drafted tokens over 8000
    // 29.6 -> 25.4, eight sequences of up to 2000 keys 13.5 -> 10.8; 24 of up to 12000 have too many items and stay as they were).
    const uint32_t N = seqs[a.B - 1].w;
    uint32_t units = upto[a.B - 1], unit = MIN_STRETCH;
    if (units > gridDim.x && a.B <= WARPS * 32 && a.B * a.Hkv <= gridDim.x) {
        const uint32_t share = max(MIN_STRETCH, (N + gridDim.x - 1) / gridDim.x);
        auto with = [&](uint32_t u) { return (own + u - 1) / u * a.Hkv; };
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) {
            const uint32_t all = __reduce_add_sync(0xffffffffu, with(share + (1u << k)));
            if (lane == 0) shared_u[k * WARPS + warp] = all;
        }
        __syncthreads();
#pragma unroll
        for (int k = 3; k >= 0; --k) {
            uint32_t all = 0;
#pragma unroll
            for (uint32_t w = 0; w < WARPS; ++w) all += shared_u[k * WARPS + w];
            if (all <= gridDim.x) { units = all; unit = share + (1u << k); }
        }
        __syncthreads();
        if (unit != MIN_STRETCH) {
            uint32_t x = with(unit);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const uint32_t y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
            if (lane == 31) shared_u[warp] = x;
            __syncthreads();
#pragma unroll
            for (uint32_t w = 0; w < WARPS; ++w) if (w < warp) x += shared_u[w];
            if (tid < a.B) upto[tid] = x;
            __syncthreads();
        }
    }
    const bool within = units <= gridDim.x;
    const uint32_t ctas = within ? units : min(gridDim.x, (N + MIN_STRETCH - 1) / MIN_STRETCH);
    if (blockIdx.x >= ctas) {
        if (f.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
        return;
    }
    const uint32_t each_cta = N / ctas, longer = N - each_cta * ctas;       // the first `longer` stretches have a chunk more
    auto stretch = [&](uint32_t cta) { return cta * each_cta + min(cta, longer); };
    uint32_t line_lo = stretch(blockIdx.x), line_hi = stretch(blockIdx.x + 1), item_parts = 0, item_part = 0;             // (of stretches within items: how many the item has, and which this is)

    // an item: a (sequence, KV head) and its place in the line
    struct Item { uint32_t b, hk, lo, hi; TgpPagedSeq s; TgpPagedKeys k; };
    auto enter = [&](Item &it, uint32_t g) {                                // the item of chunk g, whose sequence is it.b or a later one
        uint4 q = seqs[it.b];
        while (q.w <= g) q = seqs[++it.b];
        it.s = TgpPagedSeq{q.x, q.y, q.z, false};
        it.k = tgp_paged_keys<KEYS>(a, it.s.end - it.s.n, it.s.end - 1);
        const uint32_t seq_lo = q.w - it.k.chunks * a.Hkv;
        it.hk = (g - seq_lo) / it.k.chunks;
        it.lo = seq_lo + it.hk * it.k.chunks;
        it.hi = it.lo + it.k.chunks;
    };
    Item ahead, now;
    {
        uint32_t lo = 0, hi = a.B - 1;                                      // the first sequence that ends behind line_lo, or this CTA
        while (lo < hi) { const uint32_t mid = (lo + hi) / 2; if (within ? upto[mid] > blockIdx.x : seqs[mid].w > line_lo) hi = mid; else lo = mid + 1; }
        ahead.b = lo;
        if (within) {
            const uint32_t seq_lo = lo ? seqs[lo - 1].w : 0, chunks = (seqs[lo].w - seq_lo) / a.Hkv, rel = blockIdx.x - (lo ? upto[lo - 1] : 0);
            item_parts = (chunks + unit - 1) / unit;
            const uint32_t hk = rel / item_parts;
            item_part = rel - hk * item_parts;
            const uint32_t each = chunks / item_parts, more = chunks - each * item_parts;
            line_lo = seq_lo + hk * chunks + item_part * each + min(item_part, more);
            line_hi = line_lo + each + (item_part < more);
        }
    }
    enter(ahead, line_lo);
    now = ahead;

    // ---- staging: this warp's chunks are line_lo + warp, + WARPS, ...; lane l copies the 16-byte pieces i * 32 + l of a chunk's keys and of its values, piece j of a row to place
    // j ^ (row & 7).  (What differs between the pieces of a lane is a constant, added or exclusive-ored: every stage begins on 256 bytes.) ----
    const uint32_t stages = (uint32_t)__cvta_generic_to_shared(few_sm) + warp * STAGES * STAGE;
    constexpr uint32_t RPI = 32 / CPR;                                      // rows that a warp's pieces cover
    const uint32_t put = (lane / CPR) * ROW + ((lane % CPR ^ lane / CPR) << 4);
    uint32_t next = line_lo + warp;                                         // the next chunk to ask for
    // The table's entries of the warp's next 32 chunks of an item are read together, a lane each, a chunk ahead of the first one's copy.
    int32_t pages = -1;
    uint32_t pages_at = 0;                                                  // chunk of lane 0's
    auto read_pages = [&]() {
        if (next >= line_hi) return;
        if (next >= ahead.hi) enter(ahead, next);
        else if (next - pages_at < 32 * WARPS) return;
        pages_at = next;
        const uint32_t g = next + lane * WARPS, i = f.page_of_chunk(ahead.k.chunk(g - ahead.lo));
        pages = g < ahead.hi && i < a.W ? a.table[(size_t)(a.b0 + ahead.b) * a.W + i] : -1;
    };
    pages_at = next - 32 * WARPS;
    read_pages();
    uint32_t present = 0;                                                   // a bit per stage: its page is one of the cache's
    auto issue = [&](uint32_t stage) {
        if (next < line_hi) {
            const uint32_t chunk = ahead.k.chunk(next - ahead.lo), key0 = chunk * KEYS;
            const int32_t page = __shfl_sync(0xffffffffu, pages, (next - pages_at) / WARPS);
            const bool there = (uint32_t)page < a.n_pages;
            present = there ? present | 1u << stage : present & ~(1u << stage);
            if (there) {
                const size_t at = (((size_t)page * a.Hkv + ahead.hk) * a.P + (key0 - f.page_of_chunk(chunk) * a.P)) * ROW + lane * 16;
                const uint8_t *kg = reinterpret_cast<const uint8_t *>(a.k) + at, *vg = reinterpret_cast<const uint8_t *>(a.v) + at;
                const uint32_t base = stages + stage * STAGE + put;
                if (key0 + KEYS <= ahead.s.end && (key0 >= ahead.k.low || key0 + KEYS <= a.sinks)) {
#pragma unroll
                    for (uint32_t i = 0; i < KEYS * CPR / 32; ++i) {
                        const uint32_t dst = (base ^ (i * RPI % 8) << 4) + i * 512;
                        cp_async16(dst, kg + i * 512);
                        cp_async16(dst + KV_BYTES, vg + i * 512);
                    }
                } else {                                                    // keys that no row sees are zeros, not read
#pragma unroll
                    for (uint32_t i = 0; i < KEYS * CPR / 32; ++i) {
                        const uint32_t key = key0 + i * RPI + lane / CPR, dst = (base ^ (i * RPI % 8) << 4) + i * 512;
                        const uint32_t bytes = key < ahead.s.end && (key >= ahead.k.low || key < a.sinks) ? 16u : 0u;
                        cp_async16_or_zeros(dst, kg + i * 512, bytes);
                        cp_async16_or_zeros(dst + KV_BYTES, vg + i * 512, bytes);
                    }
                }
            }
            next += WARPS;
            read_pages();
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (uint32_t s = 0; s < STAGES - 1; ++s) issue(s);

    // what a lane reads of a stage with ldmatrix, up to constants: of the keys as they lie, of the values transposed
    const uint32_t k_get = (lane & 7) * ROW + ((lane >> 3 ^ (lane & 7)) << 4), v_get = KV_BYTES + ((lane >> 3 & 1) * 8 + (lane & 7)) * ROW + ((lane >> 4 ^ (lane & 7)) << 4);
    const uint32_t q_get = (uint32_t)__cvta_generic_to_shared(q_sm) + (lane & 15) * ROW + ((lane >> 4 ^ (lane & 7)) << 4);
    uint32_t done = 0, stage = 0;                                           // chunks this warp has been through; the stage of the next one
    for (uint32_t seg_lo = line_lo; seg_lo < line_hi;) {                    // the CTA's part of an item
        if (seg_lo >= now.hi) enter(now, seg_lo);
        const uint32_t seg_hi = min(line_hi, now.hi), rows = now.s.n * a.G, first_pos = now.s.end - now.s.n;
        const bf16 *q_item = a.q + ((size_t)now.s.first * a.Hq + now.hk * a.G) * DH;
        auto token_of = [&](uint32_t row) { return row * f.per_token >> 16; };
        auto q_row = [&](uint32_t row) { const uint32_t t = token_of(row); return q_item + ((size_t)t * a.Hq + (row - t * a.G)) * DH; };
        // ---- Q: in registers (one tile), or in shared memory, rows as wide as the keys' ----
        uint32_t qf[MT == 1 ? DH / 16 : 1][4];
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
        // The reference m of a row's exponents follows its maximum where that is more than 2^LIFT above it: weights and sums are floating point, and are as exact anywhere.  So a chunk
        // asks one question of all rows, those for which it is true move, and O is hardly ever multiplied.  (It starts from the least number, not from -inf: scores of -inf weigh nothing then, in whichever chunk they are met.)
        float o[MT][DH / 8][4], m[MT][2], l[MT][4];                         // l: the sums of the rounded weights, of rows r (0) and r + 8 (2), by a product with ones
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            m[t][0] = m[t][1] = -FLT_MAX;
            l[t][0] = l[t][1] = l[t][2] = l[t][3] = 0.f;
#pragma unroll
            for (int j = 0; j < DH / 8; ++j) o[t][j][0] = o[t][j][1] = o[t][j][2] = o[t][j][3] = 0.f;
        }
        auto pos_of = [&](int t, int e) { return first_pos + token_of(min(t * 16 + r + 8 * e, rows - 1)); };      // of this lane's rows (of the last row where there is none)

        for (uint32_t g = line_lo + warp + done * WARPS; g < seg_hi; g += WARPS, ++done, stage = stage + 1 == STAGES ? 0 : stage + 1) {
            issue(stage == 0 ? STAGES - 1 : stage - 1);
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
            __syncwarp();
            if (!(present >> stage & 1)) continue;                          // (the stage is refilled behind the next chunk's barrier)
            const uint32_t key0 = now.k.chunk(g - now.lo) * KEYS, at = stages + stage * STAGE;
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
                for (int nt = 0; nt < 2; ++nt) ldsm_x4((at + k_get ^ kp << 6) + nt * 8 * ROW, b[nt][0], b[nt][1], b[nt][2], b[nt][3]);
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        uint32_t x0, x1, x2, x3;
                        if constexpr (MT == 1) { x0 = qf[2 * kp + e][0]; x1 = qf[2 * kp + e][1]; x2 = qf[2 * kp + e][2]; x3 = qf[2 * kp + e][3]; }
                        else ldsm_x4((q_get ^ (2 * kp + e) << 5) + t * 16 * ROW, x0, x1, x2, x3);
#pragma unroll
                        for (int nt = 0; nt < 2; ++nt) mma_bf16(s[t][nt], x0, x1, x2, x3, b[nt][2 * e], b[nt][2 * e + 1]);
                    }
            }
            // ---- weights: this lane's keys are 2c, 2c + 1, 8 + 2c, 9 + 2c of rows r and r + 8 ----
            if (!whole) {
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t pos = pos_of(t, e);
#pragma unroll
                        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                            for (int i = 0; i < 2; ++i) if (!tgp_paged_sees(a, pos, key0 + nt * 8 + 2 * c + i)) s[t][nt][2 * e + i] = -INFINITY;
                    }
            }
            float x[MT][2][4], top = -INFINITY;
            auto exponents = [&]() {
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[t][nt][i] = fmaf(s[t][nt][i], a.sl2, -m[t][i >> 1]);
            };
            exponents();
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) top = fmaxf(top, fmaxf(fmaxf(x[t][nt][0], x[t][nt][1]), fmaxf(x[t][nt][2], x[t][nt][3])));
            if (__any_sync(0xffffffffu, top > LIFT)) {
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float best = fmaxf(fmaxf(s[t][0][2 * e], s[t][0][2 * e + 1]), fmaxf(s[t][1][2 * e], s[t][1][2 * e + 1]));
                        best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, 1));
                        best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, 2));
                        // only a row that asked itself (its largest exponent, by the same operation): its bits do not depend on the others
                        best = fmaf(best, a.sl2, -m[t][e]) > LIFT ? best * a.sl2 : m[t][e];
                        const float alpha = ex2(m[t][e] - best);             // (the first time: of zeros)
                        m[t][e] = best;
                        l[t][2 * e] *= alpha;
#pragma unroll
                        for (int j = 0; j < DH / 8; ++j) { o[t][j][2 * e] *= alpha; o[t][j][2 * e + 1] *= alpha; }
                    }
                exponents();
            }
            uint32_t pa[MT][4];
#pragma unroll
            for (int t = 0; t < MT; ++t) {
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) pa[t][2 * nt + e] = bf16x2(ex2(x[t][nt][2 * e]), ex2(x[t][nt][2 * e + 1]));
                mma_bf16(l[t], pa[t][0], pa[t][1], pa[t][2], pa[t][3], ONES, ONES);
            }
            // ---- O += P V ----
            // Where some rows see a key and others do not, a value that is no number must not reach the others as 0 x inf: it is added to the rows that see it, and zero in the product, which is the same
            // operations for the others as with any number there.
            bool each = false;
            if (!whole && now.s.n > 1) {
                for (uint32_t i = lane; i < KEYS * CPR; i += 32) {
                    uint32_t w0, w1, w2, w3;
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w0), "=r"(w1), "=r"(w2), "=r"(w3) : "r"(at + KV_BYTES + i * 16));
                    each |= not_finite2(w0) || not_finite2(w1) || not_finite2(w2) || not_finite2(w3);
                }
                each = __any_sync(0xffffffffu, each);
            }
            if (each) {
#pragma unroll 1
                for (uint32_t key = 0; key < KEYS; ++key) {
                    const int from = (lane & ~3) | (key % 8 / 2);           // the lane of this row that has the key's weight
#pragma unroll
                    for (int t = 0; t < MT; ++t)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint32_t two = __shfl_sync(0xffffffffu, key < 8 ? pa[t][e] : pa[t][2 + e], from);
                            const float w = __uint_as_float(key & 1 ? two & 0xffff0000u : two << 16);
                            const bool sees = tgp_paged_sees(a, pos_of(t, e), key0 + key);
#pragma unroll
                            for (int j = 0; j < DH / 8; ++j) {
                                uint32_t v;
                                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(at + KV_BYTES + key * ROW + ((j ^ (key & 7)) << 4) + 4 * c));
                                const float v0 = __uint_as_float(v << 16), v1 = __uint_as_float(v & 0xffff0000u);
                                if (sees && !(fabsf(v0) < INFINITY)) o[t][j][2 * e] += w * v0;
                                if (sees && !(fabsf(v1) < INFINITY)) o[t][j][2 * e + 1] += w * v1;
                            }
                        }
                }
                __syncwarp();
                for (uint32_t i = lane; i < KEYS * CPR * 4; i += 32) {
                    uint32_t v;
                    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(at + KV_BYTES + i * 4));
                    if ((v & 0x7f80u) == 0x7f80u) v &= 0xffff0000u;
                    if ((v & 0x7f800000u) == 0x7f800000u) v &= 0xffffu;
                    asm volatile("st.shared.b32 [%0], %1;" ::"r"(at + KV_BYTES + i * 4), "r"(v) : "memory");
                }
                __syncwarp();
            }
#pragma unroll
            for (int jp = 0; jp < DH / 16; ++jp) {
                uint32_t v0, v1, v2, v3;
                ldsm_x4_t(at + v_get ^ jp << 5, v0, v1, v2, v3);
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    mma_bf16(o[t][2 * jp], pa[t][0], pa[t][1], pa[t][2], pa[t][3], v0, v1);
                    mma_bf16(o[t][2 * jp + 1], pa[t][0], pa[t][1], pa[t][2], pa[t][3], v2, v3);
                }
            }
            __syncwarp();                                                   // the stage may be refilled
        }
        // ---- the four warps' partials: outputs go to the stage that each has free (the two behind it are under way), one tile at a time ----
        const bool complete = seg_lo == now.lo && seg_hi == now.hi;
        float *slot = f.parts + ((size_t)blockIdx.x * 2 + (seg_lo == line_lo ? 0 : 1)) * slot_floats<DH, MT>();
        float *mine = reinterpret_cast<float *>(few_sm + (size_t)(warp * STAGES + (stage == 0 ? STAGES - 1 : stage - 1)) * STAGE);
        auto finish = [&](uint32_t row, uint32_t d, float4 v, float sum) {  // (a row that sees nothing is zero; a NaN stays one)
            const uint32_t t = token_of(row);
            const float inv = 1.f / sum;
            uint2 two = make_uint2(bf16x2(v.x * inv, v.y * inv), bf16x2(v.z * inv, v.w * inv));
            if (sum == 0.f) two = make_uint2(0u, 0u);
            *reinterpret_cast<uint2 *>(a.o + ((size_t)(now.s.first + t) * a.Hq + now.hk * a.G + (row - t * a.G)) * DH + d) = two;
        };
        auto add = [](float4 &v, float w, const float4 &x) { v.x += w * x.x; v.y += w * x.y; v.z += w * x.z; v.w += w * x.w; };
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            if (t && t * 16 >= rows) break;
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t row = r + 8 * e;
                if (t * 16 + row < rows) {
                    if (c == 0) { ml[(warp * 16 + row) * 2] = m[t][e]; ml[(warp * 16 + row) * 2 + 1] = l[t][2 * e]; }
#pragma unroll
                    for (int j = 0; j < DH / 8; ++j) *reinterpret_cast<float2 *>(mine + row * DH + ((j * 8 + 2 * c) ^ (row & 7) * 8)) = make_float2(o[t][j][2 * e], o[t][j][2 * e + 1]);
                }
            }
            if (tid == 0) shared_u[8] = 0;
            if (lane == 0) shared_u[warp] = (uint32_t)(reinterpret_cast<uint8_t *>(mine) - few_sm);
            __syncthreads();
            const uint32_t tile_rows = min(16u, rows - t * 16);
            const float *theirs[WARPS];
#pragma unroll
            for (uint32_t w = 0; w < WARPS; ++w) theirs[w] = reinterpret_cast<const float *>(few_sm + shared_u[w]);
            for (uint32_t i = tid; i < tile_rows * DH / 4; i += WARPS * 32) {
                const uint32_t row = i / (DH / 4), d = i % (DH / 4) * 4;
                float2 x[WARPS];
                float M = -FLT_MAX, sum = 0.f;
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (uint32_t w = 0; w < WARPS; ++w) { x[w] = *reinterpret_cast<const float2 *>(ml + (w * 16 + row) * 2); M = fmaxf(M, x[w].x); }
#pragma unroll
                for (uint32_t w = 0; w < WARPS; ++w) {
                    const float wgt = ex2(x[w].x - M);                      // (a warp without a chunk: any weight of zeros)
                    sum += wgt * x[w].y;
                    add(v, wgt, *reinterpret_cast<const float4 *>(theirs[w] + row * DH + (d ^ (row & 7) * 8)));
                }
                if (complete) finish(t * 16 + row, d, v, sum);
                else {
                    if (d == 0) *reinterpret_cast<float2 *>(slot + MT * 16 * DH + (t * 16 + row) * 2) = make_float2(M, sum);
                    *reinterpret_cast<float4 *>(slot + (t * 16 + row) * DH + d) = v;
                }
            }
            __syncthreads();
        }
        // ---- an item of several stretches: the last to arrive merges ----
        if (!complete) {
            const uint32_t item = (a.b0 + now.b) * a.Hkv + now.hk;
            // CTAs of the item's first and last chunk
            auto cta_of = [&](uint32_t g) { return g < longer * (each_cta + 1) ? g / (each_cta + 1) : longer + (g - longer * (each_cta + 1)) / each_cta; };
            const uint32_t c0 = within ? blockIdx.x - item_part : cta_of(now.lo), parts = within ? item_parts : cta_of(now.hi - 1) - c0 + 1;
            if (tid == 0) shared_u[8] = tgp_paged_arrive(f.counters + item) == parts;
            __syncthreads();
            if (shared_u[8]) {
                if (tid == 0) f.counters[item] = TGP_PAGED_COUNTS;
                // a partial: [rows][DH] outputs, [rows][2] maxima and sums
                auto part = [&](uint32_t p) { const uint32_t cta = c0 + p; return f.parts + ((size_t)cta * 2 + (within || stretch(cta) >= now.lo ? 0 : 1)) * slot_floats<DH, MT>(); };
                auto ml_of = [&](const float *from, uint32_t row) { return __ldcg(reinterpret_cast<const float2 *>(from + MT * 16 * DH + row * 2)); };
                auto four_of = [&](const float *from, uint32_t row, uint32_t d) { return __ldcg(reinterpret_cast<const float4 *>(from + row * DH + d)); };
                constexpr uint32_t SOME = MT == 1 ? 6 : 4, ROWS = DH == 128 ? (MT == 1 ? 2 : 3) : 1;     // partials, and pieces of four dimensions, that a thread asks for at a time
                for (uint32_t i0 = tid; i0 < rows * DH / 4; i0 += WARPS * 32 * ROWS) {
                    float M[ROWS], sum[ROWS];
                    float4 v[ROWS];
#pragma unroll
                    for (uint32_t k = 0; k < ROWS; ++k) { M[k] = -FLT_MAX; sum[k] = 0.f; v[k] = make_float4(0.f, 0.f, 0.f, 0.f); }
                    for (uint32_t p0 = 0; p0 < parts; p0 += SOME) {
                        float2 y[ROWS][SOME];
                        float4 x[ROWS][SOME];
#pragma unroll
                        for (uint32_t p = 0; p < SOME; ++p) {
                            const float *from = part(min(p0 + p, parts - 1));
#pragma unroll
                            for (uint32_t k = 0; k < ROWS; ++k) {
                                const uint32_t i = i0 + k * WARPS * 32, row = i / (DH / 4), d = i % (DH / 4) * 4;
                                y[k][p] = make_float2(-FLT_MAX, 0.f);
                                x[k][p] = make_float4(0.f, 0.f, 0.f, 0.f);
                                if (p0 + p < parts && row < rows) { y[k][p] = ml_of(from, row); x[k][p] = four_of(from, row, d); }
                            }
                        }
#pragma unroll
                        for (uint32_t k = 0; k < ROWS; ++k) {
                            float best = M[k];
#pragma unroll
                            for (uint32_t p = 0; p < SOME; ++p) best = fmaxf(best, y[k][p].x);
                            const float old = ex2(M[k] - best);
                            M[k] = best;
                            sum[k] *= old;
                            v[k].x *= old; v[k].y *= old; v[k].z *= old; v[k].w *= old;
#pragma unroll
                            for (uint32_t p = 0; p < SOME; ++p) { const float w = ex2(y[k][p].x - best); sum[k] += w * y[k][p].y; add(v[k], w, x[k][p]); }
                        }
                    }
#pragma unroll
                    for (uint32_t k = 0; k < ROWS; ++k) {
                        const uint32_t i = i0 + k * WARPS * 32, row = i / (DH / 4);
                        if (row < rows) finish(row, i % (DH / 4) * 4, v[k], sum[k]);
                    }
                }
            }
            __syncthreads();
        }
        seg_lo = seg_hi;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (f.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// CTAs that the GPU holds at a time, of launches of up to some 360 sequences.  Above, their 20 bytes each in shared memory leave three CTAs an SM instead of four (heads of 64, one tile of rows: from 369 sequences on), or
// one instead of two (heads of 128, two tiles: from 420 on), and the grid's stretches take two turns: 368 -> 384 single tokens over up to 600 keys, 8 heads of 64 over 2, 19.2 -> 29.8 us; 416 -> 432 of up to five drafted
// tokens, heads of 128, 45.0 -> 73.5.
template <int DH, int MT> uint32_t few_ctas() { return (uint32_t)tgpk_sms() * (DH == 128 ? 2u : MT == 1 ? 4u : 3u); }

template <int DH, int MT>
int launch_few(FewArgs f, cudaStream_t st) {
    if (!tgpk_allow_smem<tgp_attn_paged_few_kernel<DH, MT>>(fixed_smem<DH, MT>() + GROUP * 20, true)) return TGP_E_CUDA;
    const uint32_t B = f.a.B;
    for (uint32_t b0 = 0; b0 < B; b0 += GROUP) {
        f.a.b0 = b0;
        f.a.B = std::min(GROUP, B - b0);
        if (int rc = launch(tgp_attn_paged_few_kernel<DH, MT>, dim3(few_ctas<DH, MT>()), dim3(WARPS * 32), fixed_smem<DH, MT>() + f.a.B * 20, st, 1, f)) return rc;
        f.beside = false;                                                   // the next launch takes the same partials
    }
    return TGP_OK;
}

bool shapes_ok(const tgp_model_cfg *c) { return c && (c->Dh == 64 || c->Dh == 128) && c->Hkv && c->Hq && c->Hq % c->Hkv == 0 && c->Hq / c->Hkv <= 128 && c->TK && c->TK % 16 == 0 && c->max_len; }

// bytes of the counters - of each sequence and KV head, and one of tiles -, and of the partials of a launch of few rows
uint64_t counter_bytes(const tgp_model_cfg *c, uint32_t B) { return (((uint64_t)B * c->Hkv + 1) * 8 + 255) / 256 * 256; }
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
        (uint64_t)n_pages * cfg->TK * cfg->Hkv > 0x7fffff00u || (uint64_t)B * ((kv_max + 15) / 16) * cfg->Hkv > 0x7fffffffu) return TGP_E_TOO_LARGE;
    if (!B || !T || !q_max || !kv_max) return TGP_OK;
    q_max = std::min(q_max, T);
    const uint32_t G = cfg->Hq / cfg->Hkv;
    FewArgs f{};
    f.a = TgpPagedAttn{(const bf16 *)qb, (const bf16 *)k_pages, (const bf16 *)v_pages, (bf16 *)ob, table_dev, start_dev, end_dev, cfg->Hq, cfg->Hkv, G, cfg->TK,
                       cfg->max_len / cfg->TK + (cfg->max_len % cfg->TK != 0), B, T, q_max, kv_max, n_pages, window, window ? sinks : 0, 0, 1.4426950408889634f / sqrtf((float)cfg->Dh), 0};
    // with s bits for the chunks of a page, ceil(2^(27 + s) / chunks) is off by less than 2^s / 2^(27 + s) of what it multiplies
    const uint32_t chunks = cfg->TK / KEYS;
    uint32_t s = 0;
    while ((1u << s) < chunks) ++s;
    f.shift = 27 + s;
    f.magic = (uint32_t)(((1ull << f.shift) + chunks - 1) / chunks);
    f.per_token = (65536 + G - 1) / G;
    f.counters = (u64 *)scratch_dev;
    f.parts = (float *)((uint8_t *)scratch_dev + counter_bytes(cfg, B));
    // one tile of 16 rows where all sequences fit it, else two; sequences of more rows are the other kernel's
    const bool one = (uint64_t)q_max * G <= 16;
    f.a.few = one ? 16 : 32;
    f.beside = (uint64_t)q_max * G > f.a.few;
    if (f.beside)
        if (int rc = tgpk_attn_paged_many(f.a, cfg->Dh, f.counters + (uint64_t)B * cfg->Hkv, (cudaStream_t)stream)) return rc;
    return cfg->Dh == 64 ? (one ? launch_few<64, 1>(f, (cudaStream_t)stream) : launch_few<64, 2>(f, (cudaStream_t)stream))
                               : (one ? launch_few<128, 1>(f, (cudaStream_t)stream) : launch_few<128, 2>(f, (cudaStream_t)stream));
}
