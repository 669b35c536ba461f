// A KV cache in 4 bits: append (with the rotation), read back, and the attention that reads it.
//
// A page - one sequence and KV head of a tile - is TK rows of DH / 2 bytes of codes, two e2m1 numbers per byte with the lower dimension in the
// lower half, and behind them TK rows of DH / 16 bytes of scales in e4m3, one for 16 dimensions.  An element stands for code * scale * 2^exp.
// A code has two significant bits and a scale four, so code * scale is exact in fp16 and bf16, and what the kernels multiply is what the cache
// stands for, without a rounding of its own.  Roundings are those of a position that is appended (fp32, bf16, scale and code), of the softmax weights (fp16 where the codes are read,
// bf16 where the cache is unpacked for the kernels over bf16), and, where the codes are read, of a query's small numbers.
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
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
using tgp_sm100::cluster_sync_all; using tgp_sm100::ld_remote_f32x2; using tgp_sm100::smem_u32;
typedef __nv_bfloat16 bf16;
constexpr uint32_t KEYS = 16;                    // positions that an MMA of the attention takes; a tile holds whole ones
constexpr uint32_t E4M3_NAN = 0x7f;

__device__ __host__ constexpr uint32_t row_codes(uint32_t Dh) { return Dh / 2; }
__device__ __host__ constexpr uint32_t row_scales(uint32_t Dh) { return Dh / 16; }
__device__ __host__ constexpr uint64_t page_bytes(uint32_t Dh, uint32_t TK) { return (uint64_t)TK * (row_codes(Dh) + row_scales(Dh)); }

// The position of sequence b's first new token, -1 if the sequence is idle: positions on the device are not trusted beyond the bound that
// the call was checked with.
__device__ __forceinline__ int position_of(const int32_t *pos, uint32_t b, uint32_t pos0) {
    if (!pos) return (int)pos0;
    const int p = pos[b];
    return p < 0 || (uint32_t)p > pos0 ? -1 : p;
}

// ---- conversions (each two values; the lower half is the first) ----
template <int BYTE> __device__ __forceinline__ uint32_t e2m1_f16x2(uint32_t w) {
    uint32_t d;
    if (BYTE == 0) asm("{.reg .b8 p, q, r, s; mov.b32 {p, q, r, s}, %1; cvt.rn.f16x2.e2m1x2 %0, p;}" : "=r"(d) : "r"(w));
    else if (BYTE == 1) asm("{.reg .b8 p, q, r, s; mov.b32 {p, q, r, s}, %1; cvt.rn.f16x2.e2m1x2 %0, q;}" : "=r"(d) : "r"(w));
    else if (BYTE == 2) asm("{.reg .b8 p, q, r, s; mov.b32 {p, q, r, s}, %1; cvt.rn.f16x2.e2m1x2 %0, r;}" : "=r"(d) : "r"(w));
    else asm("{.reg .b8 p, q, r, s; mov.b32 {p, q, r, s}, %1; cvt.rn.f16x2.e2m1x2 %0, s;}" : "=r"(d) : "r"(w));
    return d;
}
__device__ __forceinline__ uint16_t e2m1_of(float x0, float x1, float x2, float x3) {       // four codes, the first the lowest
    uint16_t d;
    asm("{.reg .b8 p, q; cvt.rn.satfinite.e2m1x2.f32 p, %2, %1; cvt.rn.satfinite.e2m1x2.f32 q, %4, %3; mov.b16 %0, {p, q};}" : "=h"(d) : "f"(x0), "f"(x1), "f"(x2), "f"(x3));
    return d;
}
__device__ __forceinline__ uint32_t e4m3_f16x2(uint32_t two) {
    uint32_t d;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(d) : "h"((uint16_t)two));
    return d;
}
__device__ __forceinline__ uint32_t e4m3_of(float x) {                           // largest magnitude where x is beyond it
    uint16_t d;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(d) : "f"(x), "f"(0.f));
    return d & 0xffu;
}
__device__ __forceinline__ float half_lo(uint32_t h) { return __low2float(*reinterpret_cast<const __half2 *>(&h)); }
__device__ __forceinline__ float half_hi(uint32_t h) { return __high2float(*reinterpret_cast<const __half2 *>(&h)); }
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) { const __half2 h = __floats2half2_rn(lo, hi); return *reinterpret_cast<const uint32_t *>(&h); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) { const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi); return *reinterpret_cast<const uint32_t *>(&h); }
__device__ __forceinline__ uint32_t mul2(uint32_t x, uint32_t y) { uint32_t d; asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(x), "r"(y)); return d; }
__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// ---- append ---------------------------------------------------------------------------------------------------------------------

// x * c + y * s, rounded to fp32 once (and to bf16 by the caller): the products' own roundings are found by fused multiply-adds and the sum's by the difference of what it
// should be (Knuth's sum of two numbers), and added back.  The cache's values then do not depend on the order of a multiplication and an addition, at a border of two
// 4-bit codes least of all.
__device__ __forceinline__ float two_products(float x, float c, float y, float s) {
    const float p = __fmul_rn(x, c), q = __fmul_rn(y, s), sum = __fadd_rn(p, q);
    const float t = __fsub_rn(sum, p), lost = __fadd_rn(__fsub_rn(p, __fsub_rn(sum, t)), __fsub_rn(q, t));
    const float rest = __fadd_rn(lost, __fadd_rn(__fmaf_rn(x, c, -p), __fmaf_rn(y, s, -q)));
    return rest != 0.f && fabsf(sum) < INFINITY ? __fadd_rn(sum, rest) : sum;       // (a zero keeps its sign; an infinity's rest is NaN)
}

// Codes and scale of a group of 16 dimensions of which this thread and its three neighbours hold four each, bf16 values; the codes are 16 bits.
// The quotient is never near a border without being on it (a border times the scale has seven bits, the value eight), so both roundings
// are those of the exact quotients.
__device__ __forceinline__ uint32_t quantise(const float (&x)[4], float down, uint32_t quad, uint32_t &scale) {
    uint32_t top = 0;                                            // the largest magnitude as its bits: ordered like the numbers, infinity and NaN above all of them
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = max(top, __shfl_xor_sync(quad, top, 1));
    top = max(top, __shfl_xor_sync(quad, top, 2));
    if (top >= 0x7f800000u) { scale = E4M3_NAN; return 0; }      // the group stands for NaN
    scale = e4m3_of(__fdiv_rn(__uint_as_float(top) * down, 6.f));
    const float s = half_lo(e4m3_f16x2(scale));
    if (s == 0.f) return 0;
    return e2m1_of(__fdiv_rn(x[0] * down, s), __fdiv_rn(x[1] * down, s), __fdiv_rn(x[2] * down, s), __fdiv_rn(x[3] * down, s));
}

struct AppendArgs {
    const float *q32, *k32, *v32; bf16 *qb; const float *cos_t, *sin_t; const int32_t *pos;
    uint32_t Hq, Hkv, TK, q_len, pos0;
    float k_down, v_down;                                        // 2^-exp
    TgpTilePtrs tiles;
};

// A thread takes four neighbouring dimensions of a head and their partners half a head away, as in tgp_rope_kv_vec_kernel: 16-byte loads, and the
// four threads of a group of 16 dimensions are neighbours.  8192 positions of 64 + 2 x 8 heads of 128 (479 MB) take 93 us with a cold L2, 5.1 TB/s,
// with the issue slots 78 % busy (100 us with the read back right behind it): a rotated value costs 13 instructions, three without the exact sum.  (An estimate with an error bound
// first, the exact sum where the bound does not settle the rounding, would leave no warp of 256 values without such a one.)  Eight single tokens, read back: 3.9 us, which is the launches.
template <int DH>
__global__ void __launch_bounds__(256) tgp_rope_kv_q4_kernel(const AppendArgs a) {
    pdl_enter();
    constexpr uint32_t HALF = DH / 2, V = HALF / 4;
    const uint32_t m = blockIdx.x, b = m / a.q_len, quad = 0xfu << (threadIdx.x & 28u);
    const int first = position_of(a.pos, b, a.pos0);
    if (first < 0) return;
    const uint32_t pos = (uint32_t)first + (m - b * a.q_len), tile = pos / a.TK, slot = pos - tile * a.TK;
    for (uint32_t idx = blockIdx.y * blockDim.x + threadIdx.x; idx < (a.Hq + 2 * a.Hkv) * V; idx += gridDim.y * blockDim.x) {
        const uint32_t h = idx / V, i = idx % V * 4;
        const bool rot = h < a.Hq + a.Hkv;
        const uint32_t hk = h < a.Hq ? h : rot ? h - a.Hq : h - a.Hq - a.Hkv;
        const float *s = (h < a.Hq ? a.q32 + (size_t)m * a.Hq * DH : (rot ? a.k32 : a.v32) + (size_t)m * a.Hkv * DH) + hk * DH + i;
        const float4 y0 = *reinterpret_cast<const float4 *>(s), y1 = *reinterpret_cast<const float4 *>(s + HALF);
        float x0[4] = {y0.x, y0.y, y0.z, y0.w}, x1[4] = {y1.x, y1.y, y1.z, y1.w};
        if (rot) {
            const float4 c4 = *reinterpret_cast<const float4 *>(a.cos_t + (size_t)pos * HALF + i), s4 = *reinterpret_cast<const float4 *>(a.sin_t + (size_t)pos * HALF + i);
            const float c[4] = {c4.x, c4.y, c4.z, c4.w}, sn[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float lo = x0[e], hi = x1[e];
                x0[e] = two_products(lo, c[e], -hi, sn[e]);
                x1[e] = two_products(hi, c[e], lo, sn[e]);
            }
        }
        const uint2 p0 = make_uint2(pack_bf16(x0[0], x0[1]), pack_bf16(x0[2], x0[3])), p1 = make_uint2(pack_bf16(x1[0], x1[1]), pack_bf16(x1[2], x1[3]));
        if (h < a.Hq) {
            bf16 *o = a.qb + (size_t)m * a.Hq * DH + hk * DH + i;
            *reinterpret_cast<uint2 *>(o) = p0;
            *reinterpret_cast<uint2 *>(o + HALF) = p1;
            continue;
        }
        uint8_t *page = reinterpret_cast<uint8_t *>(rot ? a.tiles.k[tile] : a.tiles.v[tile]) + ((size_t)b * a.Hkv + hk) * page_bytes(DH, a.TK);
        uint8_t *codes = page + slot * row_codes(DH) + i / 2, *scales = page + a.TK * row_codes(DH) + slot * row_scales(DH) + i / 16;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            const uint2 p = part ? p1 : p0;
            const float x[4] = {__uint_as_float(p.x << 16), __uint_as_float(p.x & 0xffff0000u), __uint_as_float(p.y << 16), __uint_as_float(p.y & 0xffff0000u)};
            uint32_t scale;
            const uint32_t code = quantise(x, rot ? a.k_down : a.v_down, quad, scale);
            *reinterpret_cast<uint16_t *>(codes + part * (HALF / 2)) = (uint16_t)code;
            if ((i & 15u) == 0) scales[part * (HALF / 16)] = (uint8_t)scale;
        }
    }
}

// ---- read back -------------------------------------------------------------------------------------------------------------------

struct UnpackArgs {
    bf16 *kb, *vb; const int32_t *pos;
    uint32_t Hkv, TK, count, pos0, ld, no_nan;                   // rows of a head in kb and vb are ld apart from head to head; values of positions from no_nan on that stand for NaN are zeros
    float k_up, v_up;                                            // 2^exp
    TgpTilePtrs tiles;
};

// A thread takes a group of 16 dimensions: 8 bytes of codes and a scale, 32 bytes of bf16.  8192 positions of 2 x 8 heads of 128 (9 MB of codes, 34 MB of bf16) take
// 13 us with a cold L2, 3.3 TB/s, twice what HBM needs: a thread's 9 bytes are all that it has requested while it waits (memory is what warps wait for most,
// 58 % of the issue slots are busy).
template <int DH>
__global__ void __launch_bounds__(256) tgp_kv_unpack_q4_kernel(const UnpackArgs a) {
    pdl_enter();
    constexpr uint32_t GROUPS = DH / 16;
    const uint32_t hk = blockIdx.y % a.Hkv, b = blockIdx.y / a.Hkv, is_v = blockIdx.z;
    const int first = position_of(a.pos, b, a.pos0);
    if (first < 0) return;
    const float up = is_v ? a.v_up : a.k_up;
    bf16 *out = (is_v ? a.vb : a.kb) + (size_t)blockIdx.y * a.ld * DH;
    for (uint32_t idx = blockIdx.x * blockDim.x + threadIdx.x; idx < a.count * GROUPS; idx += gridDim.x * blockDim.x) {
        const uint32_t t = idx / GROUPS, g = idx % GROUPS, pos = (uint32_t)first + t, tile = pos / a.TK, slot = pos - tile * a.TK;
        const uint8_t *page = reinterpret_cast<const uint8_t *>(is_v ? a.tiles.v[tile] : a.tiles.k[tile]) + ((size_t)b * a.Hkv + hk) * page_bytes(DH, a.TK);
        const uint2 w = *reinterpret_cast<const uint2 *>(page + slot * row_codes(DH) + g * 8);
        uint32_t scale = page[a.TK * row_codes(DH) + slot * row_scales(DH) + g];
        if (is_v && pos >= a.no_nan && (scale & 0x7fu) == E4M3_NAN) scale = 0;
        const float s = half_lo(e4m3_f16x2(scale)) * up;
        const uint32_t h[8] = {e2m1_f16x2<0>(w.x), e2m1_f16x2<1>(w.x), e2m1_f16x2<2>(w.x), e2m1_f16x2<3>(w.x),
                               e2m1_f16x2<0>(w.y), e2m1_f16x2<1>(w.y), e2m1_f16x2<2>(w.y), e2m1_f16x2<3>(w.y)};
        uint32_t o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = pack_bf16(half_lo(h[i]) * s, half_hi(h[i]) * s);
        uint4 *dst = reinterpret_cast<uint4 *>(out + (size_t)t * DH + g * 16);
        dst[0] = make_uint4(o[0], o[1], o[2], o[3]);
        dst[1] = make_uint4(o[4], o[5], o[6], o[7]);
    }
}

// A value that stands for NaN makes NaN of the queries that see it, and of no other.  The attention kernels over bf16 multiply values by weights of 0 where a query does
// not see them, so those of a call's own positions, which only its later queries see, are unpacked as zeros (no_nan), and this kernel writes what they make of
// the outputs: a thread looks at the scales of one new position, and as a rule nobody finds anything.
struct NanArgs {
    bf16 *ob;
    uint32_t Hq, Hkv, G, TK, q_len, pos0;
    TgpTilePtrs tiles;
};
template <int DH>
__global__ void __launch_bounds__(256) tgp_attn_q4_nan_kernel(const NanArgs a) {
    pdl_enter();
    constexpr uint32_t GROUPS = DH / 16;
    __shared__ uint32_t first[GROUPS];                           // the first query that sees a NaN in a group of dimensions
    const uint32_t hk = blockIdx.x % a.Hkv, b = blockIdx.x / a.Hkv;
    if (threadIdx.x < GROUPS) first[threadIdx.x] = a.q_len;
    __syncthreads();
    const uint32_t t = blockIdx.y * blockDim.x + threadIdx.x;
    if (t < a.q_len) {
        const uint32_t pos = a.pos0 + t, tile = pos / a.TK, slot = pos - tile * a.TK;
        const uint32_t *row = reinterpret_cast<const uint32_t *>(reinterpret_cast<const uint8_t *>(a.tiles.v[tile]) + ((size_t)b * a.Hkv + hk) * page_bytes(DH, a.TK) + a.TK * row_codes(DH) + slot * row_scales(DH));
#pragma unroll
        for (uint32_t w = 0; w < GROUPS / 4; ++w) {
            const uint32_t nan = __vcmpeq4(row[w] & 0x7f7f7f7fu, 0x7f7f7f7fu);
            if (nan)
                for (uint32_t i = 0; i < 4; ++i) if (nan >> (8 * i) & 1) atomicMin(&first[4 * w + i], t);
        }
    }
    __syncthreads();
    for (uint32_t g = 0; g < GROUPS; ++g)
        for (uint32_t i = first[g] * a.G * 16 + threadIdx.x; i < a.q_len * a.G * 16; i += blockDim.x) {
            const uint32_t t = i / 16 / a.G, h = i / 16 - t * a.G;
            a.ob[((size_t)(b * a.q_len + t) * a.Hq + hk * a.G + h) * DH + g * 16 + i % 16] = __float2bfloat16_rn(NAN);
        }
}

// ---- attention of a few query rows ------------------------------------------------------------------------------------------------
// The rows that share a KV head - the G query heads of the group, at each of the call's positions - are the eight columns of an mma.sync m16n8k16 tile, 16
// keys its rows.  Both products take the cache as the 16-row operand, so a step of eight rows costs half the MMAs that rows of their own would:
//   S [16 keys x 8 rows]      = K Q^T       DH / 16 MMAs, the sum runs over dimensions;
//   O^T [DH dimensions x 8 rows] += V^T P^T DH / 16 MMAs of 16 dimensions each, the sum runs over the keys.
// The order of a sum is free, and of the rows of a tile too, as long as both operands keep to it.  So a lane (r = lane / 4, c = lane % 4) takes whatever
// is contiguous in memory:
//   K: of the keys that rows r and r + 8 stand for, dimensions [c DH / 4, (c + 1) DH / 4) - one load of 16 bytes each (8 at DH = 64);
//   V: of its four keys, dimensions [r DH / 8, (r + 1) DH / 8) - four loads of 8 bytes (4 at DH = 64).
// and converts it to the registers the MMA reads: two codes to two fp16 per instruction, and a multiplication of both by their scales.
// Row r of a chunk stands for key (r % 2) * 4 + r / 2, and row r + 8 for the key 8 further on: the four keys of a lane's V are then
// c, c + 4, c + 8, c + 12, and each of those loads reads four neighbouring rows.
// S leaves the MMA with a key per lane row, P enters the next with a key per register pair: two 8 x 8 transposes (movmatrix) of P in fp16.
// Bound by the chain of a warp's steps - conversion, S, vote, exponentials, transpose, O, chunk after chunk - at four warps a scheduler: 16 keys of 128 dimensions (2.3 KB of K and
// V) take about 290 instructions, most of them conversions and the products with the scales, which the issue slots (61 % busy) would do in half of the time; a warp waits for its
// own last instruction's result or for the pipe of the conversions twice as long as it issues.  Calls in a row, whose cache may lie in L2 / behind an L2 flush: 24 sequences of 12001 keys, 64 heads over 8 x 128
// 71 / 84 - 86 us (333 MB, which HBM would move in 51); 61 of up to 2501 keys at positions of their own, 32 heads over 8 27.5 - 29 / 37 (12; 41 us when the host waits for each call); one of 701 keys 4.1 / 10, a launch and
// its ramp.  Scales after the MMAs instead of on the codes would need an MMA per group of 16 dimensions with sums of its own; 128 registers and four CTAs an SM are faster than five, which
// spill (with 16 rows three CTAs of 168 registers, where chunks of 32 keys of 128 dimensions spill 8 to 20 bytes).
struct AttnQ4Args {
    const bf16 *qb; bf16 *ob; float *scratch; const int32_t *pos;
    uint32_t Hq, Hkv, G, TK, q_len, pos0, rows, row_blocks, parts, per_part, chunk, B;      // chunk: keys of one, 16 or 32; per_part: chunks
    float qk, v_up;                                              // score = q k * qk in units of log2; 2^v_exp
    TgpTilePtrs tiles;
};
constexpr int WARPS = 4;
constexpr uint32_t CLUSTER_MAX = 8;
constexpr float BELOW = 6.f, ABOVE = 14.f;

// A chunk in shared memory: codes of its keys, codes of its values, scales of both.  A 16-byte piece of a row lies where neither the copies in nor the loads of
// eight lanes at a time meet another in a bank: K is read four pieces of rows q and q + 4 at a time, V two pieces of four neighbouring rows.
template <int DH, int U> struct Stage {
    static constexpr uint32_t CODES = row_codes(DH), SCALES = row_scales(DH), V = U * KEYS * CODES, KS = 2 * V, VS = KS + U * KEYS * SCALES, BYTES = VS + U * KEYS * SCALES;
    static __device__ __forceinline__ uint32_t at(uint32_t row, uint32_t piece) {
        if constexpr (DH == 128) return (row >> 1) * 128 + (((row ^ row >> 2) & 1) * 4 + (piece ^ (row & 2))) * 16;
        else return (row >> 2) * 128 + (((row & 3) * 2 + piece) ^ (row & 4)) * 16;
    }
};
template <int DH, int U> constexpr int STAGES = U == 2 ? (DH == 128 ? 3 : 4) : DH == 128 ? 5 : 6;
template <int DH, int NT, int U> constexpr uint32_t attn_smem() {
    const uint32_t ring = WARPS * STAGES<DH, U> * Stage<DH, U>::BYTES, partial = 8 * NT * (WARPS * (DH + 8 + 2) + 2) * 4;
    return ring > partial ? ring : partial;
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(x));
    return d;
}

// One unit - a sequence, a KV head and a block of rows - or some of its chunks, [c_lo, c_lo + c_n): by all warps of the CTA.  The result goes to the output, with `partial` to that array,
// per row a reference and a sum, in four numbers, and the outputs before the division.  In a cluster (CTAs of the grid's x) the parts are merged.
template <int DH, int NT, int U, bool CLUSTER>
__device__ __forceinline__ void attend_unit(const AttnQ4Args &a, uint8_t *q4_sm, uint32_t b, uint32_t hk, uint32_t row0, int first, uint32_t c_lo, uint32_t c_n, float *partial) {
    constexpr int KS = DH / 16;                                   // MMAs of either product
    constexpr uint32_t RB = 8 * NT, LD = DH + 8, CODES = row_codes(DH), SCALES = row_scales(DH), CHUNK = U * KEYS;
    using St = Stage<DH, U>;
    constexpr uint32_t RING = STAGES<DH, U> * St::BYTES;
    float (*part_o)[RB][LD] = reinterpret_cast<float (*)[RB][LD]>(q4_sm);                                  // (of the warps, when the chunks are done)
    float (*part_ml)[RB][2] = reinterpret_cast<float (*)[RB][2]>(q4_sm + sizeof(float) * WARPS * RB * LD);
    float2 *cta_ml = reinterpret_cast<float2 *>(q4_sm + sizeof(float) * WARPS * RB * (LD + 2));
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3, part = blockIdx.x;
    const uint32_t nrows = min(RB, a.rows - row0);
    auto out_row = [&](uint32_t row) {
        const uint32_t t = (row0 + row) / a.G;
        return ((size_t)(b * a.q_len + t) * a.Hq + hk * a.G + (row0 + row - t * a.G)) * DH;
    };
    // keys that this block's rows see: the last row's; the first row's tells from where on a chunk has masked ones
    const uint32_t lim_first = (uint32_t)first + row0 / a.G, kvlen = (uint32_t)first + (row0 + nrows - 1) / a.G + 1;
    const uint32_t nchunks = (kvlen + CHUNK - 1) / CHUNK, p_lo = min(nchunks, c_lo), p_n = min(nchunks - p_lo, c_n);
    const uint32_t q_lo = p_lo + p_n * warp / WARPS, q_hi = p_lo + p_n * (warp + 1) / WARPS;          // this warp's chunks

    // ---- chunks of 16 or 32 keys (32 where a tile holds whole ones), requested STAGES - 1 ahead; the addresses of a lane's pieces run along a tile ----
    const uint64_t page = ((uint64_t)b * a.Hkv + hk) * page_bytes(DH, a.TK);
    const uint32_t krow = (r & 1) * 4 + (r >> 1), ring = (uint32_t)__cvta_generic_to_shared(q4_sm) + warp * RING;
    constexpr uint32_t SC = U * SCALES;                          // 16-byte pieces of a chunk's scales, for the keys; as many lanes bring them, and as many those of the values
    const uint32_t lane_at = St::at(lane / (CODES / 16), lane % (CODES / 16)), lane_scale = St::KS + lane * 16;
    uint32_t left = q_hi - q_lo, tile = q_lo * CHUNK / a.TK, off = q_lo * CHUNK - tile * a.TK, fill = ring;
    const uint8_t *kp = nullptr, *vp = nullptr, *sp = nullptr;
    auto enter = [&]() {                                          // the lane's pieces of the chunk at `off` in `tile`
        const uint8_t *k = reinterpret_cast<const uint8_t *>(a.tiles.k[tile]) + page, *v = reinterpret_cast<const uint8_t *>(a.tiles.v[tile]) + page;
        kp = k + off * CODES + lane * 16;
        vp = v + off * CODES + lane * 16;
        sp = (lane < SC ? k : v) + a.TK * CODES + off * SCALES + (lane % SC) * 16;
    };
    if (left) enter();
    auto request = [&]() {
        if (left) {
#pragma unroll
            for (uint32_t i = 0; i < CHUNK * CODES / 512; ++i) {      // (512 bytes are a multiple of eight rows, which the swizzle does not look at)
                cp_async16(fill + lane_at + i * 512, kp + i * 512);
                cp_async16(fill + St::V + lane_at + i * 512, vp + i * 512);
            }
            if (lane < 2 * SC) cp_async16(fill + lane_scale, sp);
            off += CHUNK;
            if (--left) {
                if (off < a.TK) { kp += CHUNK * CODES; vp += CHUNK * CODES; sp += CHUNK * SCALES; }
                else { off = 0; ++tile; enter(); }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        fill = fill + St::BYTES == ring + RING ? ring : fill + St::BYTES;
    };
#pragma unroll
    for (int i = 0; i < STAGES<DH, U> - 1; ++i) request();

    // ---- the rows of Q: fp16 has fewer exponents than bf16, so each row is scaled to [1, 2) by a power of two, which its scores get back.  Numbers down to 2^-17 of the largest
    // keep their bits, smaller ones are off by 2^-25 of it: what an fp32 sum loses next to a product of the largest, but more where the keys are zero there.  (Codes as bf16
    // instead take another conversion and multiplication for two of them, a second fp16 part of Q as many MMAs again) ----
    uint32_t qf[NT][KS][2];
    float fix[NT][2];                                             // of the rows 2c and 2c + 1, which this lane's scores belong to
    uint32_t lim[NT][2];                                          // the last key that these rows see
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const uint32_t row = nt * 8 + r;
        uint4 w[DH / 32];
#pragma unroll
        for (int i = 0; i < DH / 32; ++i) w[i] = row < nrows ? reinterpret_cast<const uint4 *>(a.qb + out_row(row) + c * (DH / 4))[i] : make_uint4(0, 0, 0, 0);
        const uint32_t *x = reinterpret_cast<const uint32_t *>(w);
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < DH / 8; ++i) top = __vmaxu2(top, x[i] & 0x7fff7fffu);
        top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 2));
        top = max(top << 16, top & 0x7fff0000u);
        uint32_t e = top >> 23;                                   // exponent of the largest; 0 (nothing but zeros and subnormals) and 255 (not finite) leave the row as it is
        if (e == 0 || e == 255) e = 127;
        const float f = __uint_as_float(e == 254 ? 0x00400000u : (254 - e) << 23);          // 2^(127 - e), subnormal at the end
#pragma unroll
        for (int i = 0; i < DH / 8; ++i) qf[nt][i / 2][i & 1] = pack_f16(__uint_as_float(x[i] << 16) * f, __uint_as_float(x[i] & 0xffff0000u) * f);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t ee = __shfl_sync(0xffffffffu, e, (2 * c + i) * 4);
            fix[nt][i] = fminf(fmaxf(a.qk * __uint_as_float(ee << 23), FLT_MIN), FLT_MAX);      // (neither 0 nor infinite: a masked score is -inf, a zero one 0)
            lim[nt][i] = (uint32_t)first + min(row0 + nt * 8 + 2 * c + i, a.rows - 1) / a.G;
        }
    }

    float o[NT][KS][4], m_ref[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int j = 0; j < KS; ++j) o[nt][j][0] = o[nt][j][1] = o[nt][j][2] = o[nt][j][3] = 0.f;
        m_ref[nt][0] = m_ref[nt][1] = -FLT_MAX;                   // finite: keys of score -inf weigh nothing, wherever they lie
        l[nt][0] = l[nt][1] = 0.f;
    }
    auto attend = [&](uint32_t at, uint32_t key0) {
        const uint8_t *st = q4_sm + (at - (uint32_t)__cvta_generic_to_shared(q4_sm));
        const bool masked = key0 + CHUNK - 1 > lim_first;         // some row does not see all of the chunk
        float s[U][NT][4];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // ---- S = K Q^T ----
            uint32_t kw[2][DH / 32];
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) {
                const uint8_t *from = st + (u * 2 + h) * 8 * CODES + (DH == 128 ? St::at(krow, c) : St::at(krow, c >> 1) + (c & 1) * 8);
                if constexpr (DH == 128) { const uint4 w = *reinterpret_cast<const uint4 *>(from); kw[h][0] = w.x; kw[h][1] = w.y; kw[h][2] = w.z; kw[h][3] = w.w; }
                else { const uint2 w = *reinterpret_cast<const uint2 *>(from); kw[h][0] = w.x; kw[h][1] = w.y; }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[u][nt][0] = s[u][nt][1] = s[u][nt][2] = s[u][nt][3] = 0.f;
            uint32_t sc[2][2];                                    // scales of the two keys, of the first and the second half of the lane's dimensions
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint8_t *from = st + St::KS + ((u * 2 + h) * 8 + krow) * SCALES;
                if constexpr (DH == 128) {
                    const uint32_t f = e4m3_f16x2(*reinterpret_cast<const uint16_t *>(from + 2 * c));
                    sc[h][0] = __byte_perm(f, f, 0x1010);
                    sc[h][1] = __byte_perm(f, f, 0x3232);
                } else sc[h][0] = sc[h][1] = e4m3_f16x2(from[c] * 0x101u);
            }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int half = DH == 128 ? ks / 4 : 0;
                const uint32_t w0 = kw[0][ks / 2], w1 = kw[1][ks / 2];
                const uint32_t a0 = mul2(ks & 1 ? e2m1_f16x2<2>(w0) : e2m1_f16x2<0>(w0), sc[0][half]), a1 = mul2(ks & 1 ? e2m1_f16x2<2>(w1) : e2m1_f16x2<0>(w1), sc[1][half]);
                const uint32_t a2 = mul2(ks & 1 ? e2m1_f16x2<3>(w0) : e2m1_f16x2<1>(w0), sc[0][half]), a3 = mul2(ks & 1 ? e2m1_f16x2<3>(w1) : e2m1_f16x2<1>(w1), sc[1][half]);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma_f16(s[u][nt], a0, a1, a2, a3, qf[nt][ks][0], qf[nt][ks][1]);
            }
            if (masked) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) if (key0 + u * KEYS + krow + (i & 2) * 4 > lim[nt][i & 1]) s[u][nt][i] = -INFINITY;       // (fix > 0)
            }
        }
        // ---- softmax weights: the reference of a row lies BELOW under its largest score when it moves, and moves when a score is more than ABOVE over it.  Weights
        // are below 2^ABOVE then, which fp16 holds, and what it rounds to multiples of 2^-24 is less than 2^-(BELOW + 14) of the largest ----
        uint32_t pb[U][NT][2];
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaf(s[u][nt][i], fix[nt][i & 1], -m_ref[nt][i & 1]));
        if (__any_sync(0xffffffffu, top > ABOVE)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float mx = fmaxf(s[0][nt][i], s[0][nt][i + 2]);
                    if constexpr (U == 2) mx = fmaxf(mx, fmaxf(s[U - 1][nt][i], s[U - 1][nt][i + 2]));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                    const float m_new = fmaxf(m_ref[nt][i], mx * fix[nt][i] - BELOW), alpha = ex2(m_ref[nt][i] - m_new);
                    m_ref[nt][i] = m_new;
                    l[nt][i] *= alpha;
#pragma unroll
                    for (int j = 0; j < KS; ++j) { o[nt][j][i] *= alpha; o[nt][j][i + 2] *= alpha; }
                }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float p[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] = ex2(fmaf(s[u][nt][i], fix[nt][i & 1], -m_ref[nt][i & 1]));
                l[nt][0] += p[0] + p[2];
                l[nt][1] += p[1] + p[3];
                pb[u][nt][0] = transpose8(pack_f16(p[0], p[1]));
                pb[u][nt][1] = transpose8(pack_f16(p[2], p[3]));
            }
        // ---- O^T += V^T P^T ----
#pragma unroll
        for (int u = 0; u < U; ++u) {
            uint32_t vw[4][DH / 64], vs[4], nans = 0;             // nans: keys whose group of this lane's dimensions stands for NaN
            const uint32_t base = key0 + u * KEYS;
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                const uint8_t *from = st + St::V + u * KEYS * CODES + (DH == 128 ? St::at(4 * i + c, r >> 1) + (r & 1) * 8 : St::at(4 * i + c, r >> 2) + (r & 3) * 4);
                if constexpr (DH == 128) { const uint2 w = *reinterpret_cast<const uint2 *>(from); vw[i][0] = w.x; vw[i][1] = w.y; }
                else vw[i][0] = *reinterpret_cast<const uint32_t *>(from);
                vs[i] = st[St::VS + (u * KEYS + 4 * i + c) * SCALES + (DH == 128 ? r : r / 2)];
            }
            if (masked) {                                         // behind the sequence: whatever the tile holds there; a row that does not see a NaN must not multiply it by 0
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t key = 4 * i + c;
                    const bool nan = (vs[i] & 0x7fu) == E4M3_NAN;
                    if (base + key < kvlen && nan) nans |= 1u << key;
                    if (base + key >= kvlen || nan) vs[i] = 0;
                }
                nans |= __shfl_xor_sync(0xffffffffu, nans, 1);
                nans |= __shfl_xor_sync(0xffffffffu, nans, 2);
            }
            const uint32_t vs01 = e4m3_f16x2(vs[0] | vs[1] << 8), vs23 = e4m3_f16x2(vs[2] | vs[3] << 8);
#pragma unroll
            for (int w = 0; w < KS / 4; ++w) {
                // bytes that hold the same dimension of two keys, of even dimensions and of odd ones
                constexpr uint32_t LO = 0x0f0f0f0fu;
                const uint32_t e01 = (vw[0][w] & LO) | (vw[1][w] << 4 & ~LO), d01 = (vw[0][w] >> 4 & LO) | (vw[1][w] & ~LO);
                const uint32_t e23 = (vw[2][w] & LO) | (vw[3][w] << 4 & ~LO), d23 = (vw[2][w] >> 4 & LO) | (vw[3][w] & ~LO);
#define TGP_Q4_PV(I) do { \
                    const uint32_t a0 = mul2(e2m1_f16x2<I>(e01), vs01), a1 = mul2(e2m1_f16x2<I>(d01), vs01), a2 = mul2(e2m1_f16x2<I>(e23), vs23), a3 = mul2(e2m1_f16x2<I>(d23), vs23); \
                    _Pragma("unroll") for (int nt = 0; nt < NT; ++nt) mma_f16(o[nt][4 * w + I], a0, a1, a2, a3, pb[u][nt][0], pb[u][nt][1]); } while (0)
                TGP_Q4_PV(0); TGP_Q4_PV(1); TGP_Q4_PV(2); TGP_Q4_PV(3);
#undef TGP_Q4_PV
            }
            if (masked && __any_sync(0xffffffffu, nans != 0)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t seen = lim[nt][i] < base ? 0u : lim[nt][i] - base >= KEYS - 1 ? 0xffffu : (2u << (lim[nt][i] - base)) - 1;
                        if (nans & seen)
#pragma unroll
                            for (int j = 0; j < KS; ++j) o[nt][j][i] = o[nt][j][i + 2] = NAN;
                    }
            }
        }
    };
    uint32_t at = ring;
    for (uint32_t q = q_lo; q < q_hi; ++q) {
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES<DH, U> - 2) : "memory");
        __syncwarp();                                             // this chunk has landed, and every lane is done with the one before, whose stage is filled next
        request();
        attend(at, q * CHUNK);
        at = at + St::BYTES == ring + RING ? ring : at + St::BYTES;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();

    // ---- the warps' partial results meet ----
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float sum = l[nt][i];
            sum += __shfl_xor_sync(0xffffffffu, sum, 4);
            sum += __shfl_xor_sync(0xffffffffu, sum, 8);
            sum += __shfl_xor_sync(0xffffffffu, sum, 16);
            const uint32_t row = nt * 8 + 2 * c + i;
            if (r == 0) { part_ml[warp][row][0] = m_ref[nt][i]; part_ml[warp][row][1] = sum; }
#pragma unroll
            for (int j = 0; j < KS; ++j) *reinterpret_cast<float2 *>(&part_o[warp][row][(j * 8 + r) * 2]) = make_float2(o[nt][j][i], o[nt][j][i + 2]);        // (without bank conflicts)
        }
    __syncthreads();
    // what a row's partial of each warp counts, and the row's reference and sum in this CTA
    if (threadIdx.x < RB) {
        const uint32_t row = threadIdx.x;
        float m[WARPS], M = -FLT_MAX, sum = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) { m[w] = part_ml[w][row][0]; M = fmaxf(M, m[w]); }
#pragma unroll
        for (int w = 0; w < WARPS; ++w) { const float f = ex2(m[w] - M); sum += f * part_ml[w][row][1]; part_ml[w][row][0] = f; }
        cta_ml[row] = make_float2(M, sum);
    }
    __syncthreads();
    constexpr uint32_t QUADS = DH / 4;
    // four neighbouring dimensions d of a row: two pairs, 16 apart in shared memory
    for (uint32_t e = threadIdx.x; e < nrows * QUADS; e += WARPS * 32) {
        const uint32_t row = e / QUADS, q = e % QUADS, d = (q & 7) * (DH / 8) + (q >> 3) * 4, at0 = ((q >> 3) * 16 + (q & 7)) * 2;
        float4 x[WARPS], acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float2 lo = *reinterpret_cast<const float2 *>(&part_o[w][row][at0]), hi = *reinterpret_cast<const float2 *>(&part_o[w][row][at0 + 16]);
            x[w] = make_float4(lo.x, lo.y, hi.x, hi.y);
        }
#pragma unroll
        for (int w = 0; w < WARPS; ++w) { const float f = part_ml[w][row][0]; acc.x += f * x[w].x; acc.y += f * x[w].y; acc.z += f * x[w].z; acc.w += f * x[w].w; }
        const float2 ml = cta_ml[row];
        if (!CLUSTER && !partial) {
            const float f = a.v_up / ml.y;
            *reinterpret_cast<uint2 *>(a.ob + out_row(row) + d) = make_uint2(pack_bf16(acc.x * f, acc.y * f), pack_bf16(acc.z * f, acc.w * f));
        } else if (!CLUSTER) {
            float *to = partial + row * (DH + 4);
            if (d == 0) *reinterpret_cast<float2 *>(to) = ml;
            *reinterpret_cast<float4 *>(to + 4 + d) = acc;
        } else {                                                  // (over what this thread has read)
            *reinterpret_cast<float2 *>(&part_o[0][row][at0]) = make_float2(acc.x, acc.y);
            *reinterpret_cast<float2 *>(&part_o[0][row][at0 + 16]) = make_float2(acc.z, acc.w);
        }
    }
    if constexpr (!CLUSTER) return;
    // the CTAs of a cluster are the parts of one unit: each takes a share of the outputs and reads all partials of it
    cluster_sync_all();
    const uint32_t share = (nrows * QUADS + a.parts - 1) / a.parts, end = min(nrows * QUADS, (part + 1) * share);
    for (uint32_t e = part * share + threadIdx.x; e < end; e += WARPS * 32) {
        const uint32_t row = e / QUADS, q = e % QUADS, d = (q & 7) * (DH / 8) + (q >> 3) * 4, at0 = ((q >> 3) * 16 + (q & 7)) * 2;
        float2 ml[CLUSTER_MAX];
        float4 x[CLUSTER_MAX];
        float M = -FLT_MAX, sum = 0.f;
#pragma unroll
        for (uint32_t p = 0; p < CLUSTER_MAX; ++p)
            if (p < a.parts) {
                ml[p] = ld_remote_f32x2(smem_u32(&cta_ml[row]), p);
                const float2 lo = ld_remote_f32x2(smem_u32(&part_o[0][row][at0]), p), hi = ld_remote_f32x2(smem_u32(&part_o[0][row][at0 + 16]), p);
                x[p] = make_float4(lo.x, lo.y, hi.x, hi.y);
            }
#pragma unroll
        for (uint32_t p = 0; p < CLUSTER_MAX; ++p) if (p < a.parts) M = fmaxf(M, ml[p].x);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (uint32_t p = 0; p < CLUSTER_MAX; ++p)
            if (p < a.parts) { const float f = ex2(ml[p].x - M); sum += f * ml[p].y; acc.x += f * x[p].x; acc.y += f * x[p].y; acc.z += f * x[p].z; acc.w += f * x[p].w; }
        const float f = a.v_up / sum;
        *reinterpret_cast<uint2 *>(a.ob + out_row(row) + d) = make_uint2(pack_bf16(acc.x * f, acc.y * f), pack_bf16(acc.z * f, acc.w * f));
    }
    cluster_sync_all();                                           // no CTA leaves while another may still read its partials
}

template <int DH, int NT, int U, bool CLUSTER>
__global__ void __launch_bounds__(WARPS * 32, NT == 1 ? 4 : 3) tgp_attn_q4_kernel(const AttnQ4Args a) {
    pdl_enter();
    extern __shared__ __align__(128) uint8_t q4_sm[];
    const uint32_t hk = blockIdx.y / a.row_blocks, row0 = (blockIdx.y - hk * a.row_blocks) * 8 * NT, b = blockIdx.z;
    const int first = position_of(a.pos, b, a.pos0);
    if (first < 0) {                                              // an idle sequence: its rows are zeros
        if (blockIdx.x == 0)
            for (uint32_t e = threadIdx.x; e < min(8u * NT, a.rows - row0) * DH; e += WARPS * 32) {
                const uint32_t row = row0 + e / DH, t = row / a.G;
                a.ob[((size_t)(b * a.q_len + t) * a.Hq + hk * a.G + (row - t * a.G)) * DH + e % DH] = __float2bfloat16_rn(0.f);
            }
        return;
    }
    attend_unit<DH, NT, U, CLUSTER>(a, q4_sm, b, hk, row0, first, blockIdx.x * a.per_part, a.per_part, nullptr);
}

// Contexts longer than a CTA should have to itself, and of any lengths: all chunks of all units lie in a row - sequence by sequence, in it unit by unit - and every CTA of one
// wave takes an equal stretch of it.  What a unit costs besides its chunks, queries and merging, is as long as SETUP chunks take, and lies before them in the row (61 sequences of up
// to 2500 keys, some of a few: 45 us without).  A unit that lies in one stretch is finished there; of others each CTA leaves a partial in the scratch array, in its place 2 i + 1 if the unit
// goes on behind its stretch, else 2 i, which the merge kernel finds again by the same arithmetic.  The array begins with the length of a stretch and where each sequence's
// chunks begin, which the first CTA writes for it.
constexpr uint32_t SETUP = 12;
struct Stretch { uint32_t per, total; };                         // (chunks; with the sequences' beginnings behind it in the scratch array)
__device__ __host__ constexpr uint64_t stretch_bytes(uint64_t B) { return (sizeof(Stretch) + 4 * (B + 1) + 15) / 16 * 16; }

template <int DH, int NT, int U>
__global__ void __launch_bounds__(WARPS * 32, NT == 1 ? 4 : 3) tgp_attn_q4_stretch_kernel(const AttnQ4Args a) {
    pdl_enter();
    extern __shared__ __align__(128) uint8_t q4_sm[];
    __shared__ uint32_t sums[WARPS], found[2];                   // of the warps' sequences; the stretch's first sequence and where its chunks begin
    constexpr uint32_t RB = 8 * NT, CHUNK = U * KEYS;
    const uint32_t units = a.Hkv * a.row_blocks, tid = threadIdx.x;
    auto chunks_of = [&](uint32_t b) {
        const int first = position_of(a.pos, b, a.pos0);
        return first < 0 ? 0u : ((uint32_t)first + a.q_len + CHUNK - 1) / CHUNK;
    };
    // a thread adds up the chunks of neighbouring sequences, the threads' sums are added up
    const uint32_t each = (a.B + WARPS * 32 - 1) / (WARPS * 32), b_lo = min(a.B, tid * each), b_hi = min(a.B, b_lo + each);
    uint32_t mine = 0;
    auto length_of = [&](uint32_t b) { const uint32_t n = chunks_of(b); return n ? n + SETUP : 0; };
    for (uint32_t b = b_lo; b < b_hi; ++b) mine += length_of(b) * units;
    uint32_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o); if ((tid & 31) >= o) upto += v; }
    if ((tid & 31) == 31) sums[tid / 32] = upto;
    __syncthreads();
    uint32_t total = 0;
#pragma unroll
    for (uint32_t w = 0; w < WARPS; ++w) { if (w < tid / 32) upto += sums[w]; total += sums[w]; }
    uint32_t begin = upto - mine;                                // of this thread's first sequence
    const uint32_t per = max((total + gridDim.x - 1) / gridDim.x, SETUP + 2 * WARPS), w_lo = min(total, blockIdx.x * per), w_hi = min(total, w_lo + per);
    Stretch *head = reinterpret_cast<Stretch *>(a.scratch);
    uint32_t *begins = reinterpret_cast<uint32_t *>(head + 1);
    if (blockIdx.x == 0 && tid == 0) *head = {per, total};
    for (uint32_t b = b_lo; b < b_hi; ++b) {
        const uint32_t n = length_of(b) * units;
        if (blockIdx.x == 0) begins[b] = begin;
        if (w_lo >= begin && w_lo < begin + n) { found[0] = b; found[1] = begin; }
        begin += n;
    }
    __syncthreads();
    float *partials = a.scratch + stretch_bytes(a.B) / sizeof(float);
    uint32_t b = found[0], base = found[1];
    for (uint32_t w = w_lo; w < w_hi;) {
        const uint32_t n = chunks_of(b), unit = (w - base) / (n + SETUP), at = w - base - unit * (n + SETUP), end = min(n + SETUP, at + w_hi - w), hk = unit / a.row_blocks;
        const uint32_t c_lo = at > SETUP ? at - SETUP : 0, c_hi = end > SETUP ? end - SETUP : 0;
        if (c_hi > c_lo) {
            if (w != w_lo) __syncthreads();                      // (the unit before is written: its shared memory is free)
            attend_unit<DH, NT, U, false>(a, q4_sm, b, hk, (unit - hk * a.row_blocks) * RB, position_of(a.pos, b, a.pos0), c_lo, c_hi - c_lo,
                                          c_hi - c_lo == n ? nullptr : partials + (2 * (size_t)blockIdx.x + (c_hi < n)) * RB * (DH + 4));
        }
        w += end - at;
        if (w < w_hi && w == base + (n + SETUP) * units) {
            base = w;
            do ++b; while (!chunks_of(b));
        }
    }
}

// One warp per row, four or two dimensions a lane: merges what the CTAs have left of its unit, eight partials' outputs under way at a time; zeros for idle sequences.
template <int DH>
__global__ void __launch_bounds__(128) tgp_attn_q4_merge_kernel(const AttnQ4Args a) {
    pdl_enter();
    const uint32_t row = blockIdx.x * 4 + threadIdx.x / 32, lane = threadIdx.x & 31, hk = blockIdx.y, b = blockIdx.z, t = row / a.G;
    if (row >= a.rows) return;
    constexpr uint32_t LD = DH + 4, V = DH / 32;
    const Stretch head = *reinterpret_cast<const Stretch *>(a.scratch);
    const uint32_t begin = reinterpret_cast<const uint32_t *>(a.scratch)[2 + b];
    const int first = position_of(a.pos, b, a.pos0);
    bf16 *to = a.ob + ((size_t)(b * a.q_len + t) * a.Hq + hk * a.G + (row - t * a.G)) * DH + lane * V;
    if (first < 0) {
#pragma unroll
        for (uint32_t i = 0; i < V; i += 2) *reinterpret_cast<uint32_t *>(to + i) = 0;
        return;
    }
    const uint32_t RB = a.rows <= 8 ? 8 : 16, n = ((uint32_t)first + a.q_len + a.chunk - 1) / a.chunk, at = begin + (hk * a.row_blocks + row / RB) * (n + SETUP) + SETUP;
    const uint32_t i_lo = at / head.per, parts = (at + n - 1) / head.per - i_lo + 1;                   // stretches that the unit lies in
    if (parts == 1) return;
    // the partial of part p, and of the last
    const float *from = a.scratch + stretch_bytes(a.B) / sizeof(float) + ((2 * (size_t)i_lo + 1) * RB + row % RB) * LD;
    const uint32_t step = 2 * RB * LD;
    auto part = [&](uint32_t p) { return from + (size_t)p * step - (p + 1 == parts ? RB * LD : 0); };
    float M = -FLT_MAX, sum = 0.f, acc[V];
    for (uint32_t p = lane; p < parts; p += 32) M = fmaxf(M, part(p)[0]);
#pragma unroll
    for (int o = 16; o; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
#pragma unroll
    for (uint32_t i = 0; i < V; ++i) acc[i] = 0.f;
    for (uint32_t p0 = 0; p0 < parts; p0 += 8) {
        float x[8][V];
        float2 ml[8];
#pragma unroll
        for (uint32_t p = 0; p < 8; ++p)
            if (p0 + p < parts) {
                const float *src = part(p0 + p);
                ml[p] = *reinterpret_cast<const float2 *>(src);
#pragma unroll
                for (uint32_t i = 0; i < V; i += 2) { const float2 v = *reinterpret_cast<const float2 *>(src + 4 + lane * V + i); x[p][i] = v.x; x[p][i + 1] = v.y; }
            }
#pragma unroll
        for (uint32_t p = 0; p < 8; ++p)
            if (p0 + p < parts) {
                const float f = ex2(ml[p].x - M);
                sum += f * ml[p].y;
#pragma unroll
                for (uint32_t i = 0; i < V; ++i) acc[i] += f * x[p][i];
            }
    }
    const float f = a.v_up / sum;
#pragma unroll
    for (uint32_t i = 0; i < V; i += 2) *reinterpret_cast<uint32_t *>(to + i) = pack_bf16(acc[i] * f, acc[i + 1] * f);
}

// ---- host side ---------------------------------------------------------------------------------------------------------------------

constexpr uint32_t UNPACK_FROM = 32;                             // queries from which on the cache may be unpacked and the tcgen05 kernel run on it

bool q4_geometry(const tgp_model_cfg *c) {
    return c && (c->Dh == 64 || c->Dh == 128) && c->Hkv && c->Hq && c->Hq % c->Hkv == 0 && c->TK && c->TK % KEYS == 0 && c->TK <= (1u << 20);
}

// positions [pos0, pos0 + q_len) of B sequences, in tiles that hold them
bool q4_call(const tgp_model_cfg *c, uint32_t n_tiles, uint32_t B, uint32_t q_len, uint32_t pos0, const int32_t *pos, int k_exp, int v_exp) {
    if (!q4_geometry(c) || B > c->B || (pos && q_len > 1) || k_exp < -TGP_Q4_EXP_MAX || k_exp > TGP_Q4_EXP_MAX || v_exp < -TGP_Q4_EXP_MAX || v_exp > TGP_Q4_EXP_MAX) return false;
    return (uint64_t)pos0 + q_len <= c->max_len && (uint64_t)pos0 + q_len <= (uint64_t)n_tiles * c->TK;
}

// tiles first <= i < end are used; they begin on 16 bytes
int q4_tiles(TgpTilePtrs &t, void *const *k, void *const *v, uint32_t n, uint32_t first, uint32_t end) {
    if (n > TGP_MAX_TILES) return TGP_E_TOO_LARGE;
    if (!k || !v) return TGP_E_INVAL;
    t = TgpTilePtrs{};
    for (uint32_t i = first; i < end && i < n; ++i) {
        t.k[i] = k[i]; t.v[i] = v[i];
        if (!k[i] || !v[i] || ((reinterpret_cast<uintptr_t>(k[i]) | reinterpret_cast<uintptr_t>(v[i])) & 15u)) return TGP_E_INVAL;
    }
    return TGP_OK;
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// How the CTAs share the work: 1, a CTA per unit; 2 - 8, a cluster of as many per unit; 0, stretches of all units' chunks.  By what each is expected to take, in chunks of a CTA on a full SM:
// what a unit costs besides its chunks (SETUP), a cluster's barriers and that its parts do not end together, a second kernel.  The ways' times (us, 32-key chunks, one CTA / cluster / stretches):
// 61 sequences of 701 keys, 32 heads over 8 x 128 15.2 / - / 20.0; 200 of 601, x 64 22.8 / - / 29.7; 16 of 2112, 64 over 8 x 128 25.7 / 14.7 (four) / 18.4; one of 4001, 32 over 8 x 64
// 21 / 6.1 (eight) / 9.8; one of 16001, x 128 108 / 17.5 (eight) / 15.8; four of these 109 / 32.4 (eight) / 25.2; 24 of 12001, 64 over 8 109 / 88 (three) / 71; 61 of up to 2500 at positions of their
// own 35 / 38 (two) / 27.4.  CTAs of a wave: four fit an SM, three with 16 rows.
uint32_t wave(uint32_t rb) { return (uint32_t)tgpk_sms() * (rb == 8 ? 4 : 3); }
uint32_t few_parts(uint32_t units, uint32_t rb, uint32_t n, bool ragged) {
    const uint32_t slots = wave(rb);
    const float mean = ragged ? 0.5f * (float)n : (float)n;      // positions of their own: the longest is known, not the mean
    float best = std::max((float)(SETUP + 2 * WARPS), (mean + SETUP) * (float)units / (float)slots) + 32.f;
    uint32_t way = 0;
    const float alone = (float)((units + slots - 1) / slots) * (float)(SETUP + n);
    if (alone <= best) { best = alone; way = 1; }
    for (uint32_t p = 2; p <= CLUSTER_MAX && p <= (n + WARPS - 1) / WARPS && (uint64_t)units * p <= slots; ++p) {
        const float together = (float)(SETUP + 5) + 1.3f * (float)((n + p - 1) / p);
        if (together < best) { best = together; way = p; }
    }
    return way;
}

template <int DH, int NT, int U>
int launch_attn(const AttnQ4Args &a, cudaStream_t st) {
    constexpr uint32_t smem = attn_smem<DH, NT, U>();
    const dim3 grid(a.parts, a.Hkv * a.row_blocks, a.B), block(WARPS * 32);
    if (a.parts > 1) {
        if (!tgpk_allow_smem<tgp_attn_q4_kernel<DH, NT, U, true>>(smem, true)) return TGP_E_CUDA;
        return launch(tgp_attn_q4_kernel<DH, NT, U, true>, grid, block, smem, st, a.parts, a);
    }
    if (a.parts == 1) {
        if (!tgpk_allow_smem<tgp_attn_q4_kernel<DH, NT, U, false>>(smem, true)) return TGP_E_CUDA;
        return launch(tgp_attn_q4_kernel<DH, NT, U, false>, grid, block, smem, st, 1, a);
    }
    if (!tgpk_allow_smem<tgp_attn_q4_stretch_kernel<DH, NT, U>>(smem, true)) return TGP_E_CUDA;
    if (int rc = launch(tgp_attn_q4_stretch_kernel<DH, NT, U>, dim3(wave(8 * NT)), block, smem, st, 1, a)) return rc;
    return launch(tgp_attn_q4_merge_kernel<DH>, dim3((a.rows + 3) / 4, a.Hkv, a.B), dim3(128), 0, st, 1, a);
}

template <int DH>
int launch_attn(const AttnQ4Args &a, cudaStream_t st) {
    if (a.chunk == 2 * KEYS) return a.rows <= 8 ? launch_attn<DH, 1, 2>(a, st) : launch_attn<DH, 2, 2>(a, st);
    return a.rows <= 8 ? launch_attn<DH, 1, 1>(a, st) : launch_attn<DH, 2, 1>(a, st);
}

uint32_t rows_of_block(const tgp_model_cfg *c, uint32_t q_len) { return (uint64_t)q_len * (c->Hq / c->Hkv) <= 8 ? 8 : 16; }

// Does a call read the codes itself?  Below 32 queries always.  From there on each block of 16 rows converts the cache again, while the tcgen05 kernel's time, on the unpacked cache, is a chain of its
// blocks of 64 keys, or the GPU's rate where its CTAs of 128 queries are many.  Both times (us) as straight lines through 300 measured shapes (8 - 256 queries of 1 - 24 sequences, 100 - 8000 keys, 8 heads over
// 1 to 64 over 8), off by an eighth as a rule; the choice costs 0.4 % on average over the better of the two, where reading the codes up to 127 queries cost 10 (us, codes / unpacked: 3 sequences of
// 2000 keys, 32 heads over 8 x 128, 32 queries 24.5 / 30.9, 64 39.5 / 31.7, 127 74.9 / 33.7; 64 heads, 8 sequences, 127 366 / 99; 24 of 500 365 / 104; one of 8000, 8 heads x 128, 127 30.9 / 60.4).
// The codes' weights keep fp16's eleven bits, the others' bf16's eight: unpacking has to gain a tenth.
bool reads_codes(const tgp_model_cfg *c, uint32_t B, uint32_t q_len, uint32_t kvlen) {
    if (q_len < UNPACK_FROM || (uint64_t)B * c->Hkv > 65535u) return true;             // (the unpacking's grid)
    const float wide = c->Dh == 128 ? 1.f : 0.f, chunks = (float)kvlen / 32.f, blocks = (float)kvlen / 64.f, pages = (float)B * (float)c->Hkv;
    const float units = pages * (float)(((uint64_t)q_len * (c->Hq / c->Hkv) + 15) / 16), ctas = (float)B * (float)c->Hq * (float)((q_len + 127) / 128);
    const float codes = 4.6f + 0.035f * chunks + 1.02e-3f * units * (chunks + 12.f) * (0.65f + 0.35f * wide);
    const float unpacked = 7.5f + 0.26f * blocks + 3.6e-3f * ctas * blocks * (0.7f + 0.3f * wide) + 6.2e-5f * pages * (float)kvlen * (1.f + wide);
    return codes * 0.9f <= unpacked;
}

uint64_t unpacked_rows(uint32_t kvlen) { return ((uint64_t)kvlen + 63) / 64 * 64; }
uint64_t unpacked_bytes(const tgp_model_cfg *c, uint32_t kvlen) { return 2 * (uint64_t)c->Hkv * unpacked_rows(kvlen) * c->Dh * sizeof(bf16); }     // of a sequence

// The part of the scratch array that holds an unpacked cache: of all sequences if that is no more than UNPACK_MOST, else of as many as fit (one at least), and a call takes
// them group by group.  Bytes in bf16 are 3.6 times those of the tiles, which are small because memory is short; a group of 4 GB fills the GPU (64 heads over 8 x 128, 131072 keys: eight
// sequences, at 32 queries 512 CTAs).
constexpr uint64_t UNPACK_MOST = 4ull << 30;
uint64_t unpacked_capacity(const tgp_model_cfg *c) {
    const uint64_t one = unpacked_bytes(c, c->max_len);
    return one * std::max<uint64_t>(1, std::min<uint64_t>(c->B, UNPACK_MOST / one));
}

int launch_unpack(const UnpackArgs &a, const tgp_model_cfg *c, uint32_t B, cudaStream_t st) {
    const dim3 grid(std::min<uint64_t>(((uint64_t)a.count * (c->Dh / 16) + 255) / 256, 1u << 20), B * c->Hkv, 2);
    return c->Dh == 64 ? launch(tgp_kv_unpack_q4_kernel<64>, grid, dim3(256), 0, st, 1, a) : launch(tgp_kv_unpack_q4_kernel<128>, grid, dim3(256), 0, st, 1, a);
}

}  // namespace

extern "C" {

int tgp_k_kv_q4_tile_bytes(const tgp_model_cfg *cfg, uint64_t *bytes) {
    if (!bytes || !q4_geometry(cfg)) return TGP_E_INVAL;
    *bytes = (uint64_t)cfg->B * cfg->Hkv * page_bytes(cfg->Dh, cfg->TK);
    return TGP_OK;
}

int tgp_k_rope_kv_q4(const float *q32, const float *k32, const float *v32, void *qb, void *const *k_tiles, void *const *v_tiles, uint32_t n_tiles, const float *cos_dev,
                     const float *sin_dev, const tgp_model_cfg *cfg, uint32_t B, uint32_t q_len, uint32_t pos0, int k_exp, int v_exp, const int32_t *pos_dev, void *stream) {
    if (!q32 || !k32 || !v32 || !qb || !cos_dev || !sin_dev || !q4_call(cfg, n_tiles, B, q_len, pos0, pos_dev, k_exp, v_exp)) return TGP_E_INVAL;
    if (!aligned16(q32) || !aligned16(k32) || !aligned16(v32) || !aligned16(qb) || !aligned16(cos_dev) || !aligned16(sin_dev)) return TGP_E_INVAL;
    AppendArgs a{q32, k32, v32, (bf16 *)qb, cos_dev, sin_dev, pos_dev, cfg->Hq, cfg->Hkv, cfg->TK, q_len, pos0, ldexpf(1.f, -k_exp), ldexpf(1.f, -v_exp), {}};
    const uint32_t end = B && q_len ? (pos0 + q_len - 1) / cfg->TK + 1 : 0;
    if (int rc = q4_tiles(a.tiles, k_tiles, v_tiles, n_tiles, pos_dev ? 0 : pos0 / cfg->TK, end)) return rc;
    if (!B || !q_len) return TGP_OK;
    if ((uint64_t)B * q_len > 0x7fffffffu) return TGP_E_TOO_LARGE;
    const uint32_t items = (cfg->Hq + 2 * cfg->Hkv) * (cfg->Dh / 8);
    const uint32_t split = std::max(1u, std::min((items + 255) / 256, 4u * (uint32_t)tgpk_sms() / (B * q_len)));
    const dim3 grid(B * q_len, split);
    return cfg->Dh == 64 ? launch(tgp_rope_kv_q4_kernel<64>, grid, dim3(256), 0, (cudaStream_t)stream, 1, a) : launch(tgp_rope_kv_q4_kernel<128>, grid, dim3(256), 0, (cudaStream_t)stream, 1, a);
}

int tgp_k_kv_unpack_q4(void *const *k_tiles, void *const *v_tiles, uint32_t n_tiles, void *kb, void *vb, const tgp_model_cfg *cfg, uint32_t B, uint32_t q_len, uint32_t pos0,
                       int k_exp, int v_exp, const int32_t *pos_dev, void *stream) {
    if (!kb || !vb || !aligned16(kb) || !aligned16(vb) || !q4_call(cfg, n_tiles, B, q_len, pos0, pos_dev, k_exp, v_exp)) return TGP_E_INVAL;
    UnpackArgs a{(bf16 *)kb, (bf16 *)vb, pos_dev, cfg->Hkv, cfg->TK, q_len, pos0, q_len, 0xffffffffu, ldexpf(1.f, k_exp), ldexpf(1.f, v_exp), {}};
    const uint32_t end = B && q_len ? (pos0 + q_len - 1) / cfg->TK + 1 : 0;
    if (int rc = q4_tiles(a.tiles, k_tiles, v_tiles, n_tiles, pos_dev ? 0 : pos0 / cfg->TK, end)) return rc;
    if (!B || !q_len) return TGP_OK;
    if ((uint64_t)B * cfg->Hkv > 65535u) return TGP_E_TOO_LARGE;
    return launch_unpack(a, cfg, B, (cudaStream_t)stream);
}

int tgp_k_attn_q4_scratch_bytes(const tgp_model_cfg *cfg, uint32_t q_len, uint64_t *bytes) {
    if (!bytes || !q4_geometry(cfg) || !cfg->B || !q_len || q_len > cfg->max_len) return TGP_E_INVAL;
    const uint64_t rb = rows_of_block(cfg, q_len);                // two partial results for each CTA of a wave; keys and values as bf16
    *bytes = stretch_bytes(cfg->B) + 2ull * wave((uint32_t)rb) * rb * (cfg->Dh + 4) * sizeof(float);
    if (q_len >= UNPACK_FROM) *bytes = std::max(*bytes, unpacked_capacity(cfg));
    return TGP_OK;
}

int tgp_k_attn_q4(const void *qb, void *const *k_tiles, void *const *v_tiles, uint32_t n_tiles, void *ob, const tgp_model_cfg *cfg, uint32_t B, uint32_t q_len, uint32_t pos0,
                  int k_exp, int v_exp, const int32_t *pos_dev, void *scratch_dev, void *stream) {
    if (!qb || !ob || !scratch_dev || !aligned16(qb) || !aligned16(ob) || !aligned16(scratch_dev) || !q4_call(cfg, n_tiles, B, q_len, pos0, pos_dev, k_exp, v_exp)) return TGP_E_INVAL;
    const uint32_t kvlen = pos0 + q_len, G = cfg->Hq / cfg->Hkv;
    TgpTilePtrs tiles;
    if (int rc = q4_tiles(tiles, k_tiles, v_tiles, n_tiles, 0, B && q_len ? (kvlen - 1) / cfg->TK + 1 : 0)) return rc;
    if (!B || !q_len) return TGP_OK;
    cudaStream_t st = (cudaStream_t)stream;
    if (reads_codes(cfg, B, q_len, kvlen)) {
        if ((uint64_t)q_len * G > 1u << 20) return TGP_E_TOO_LARGE;
        const uint32_t rows = q_len * G, rb = rows_of_block(cfg, q_len), row_blocks = (rows + rb - 1) / rb;
        if ((uint64_t)cfg->Hkv * row_blocks > 65535u || B > 65535u) return TGP_E_TOO_LARGE;
        const uint32_t chunk = cfg->TK % (2 * KEYS) ? KEYS : 2 * KEYS, nchunks = (kvlen + chunk - 1) / chunk;
        if ((uint64_t)B * cfg->Hkv * row_blocks * (nchunks + SETUP) > 0x7fffffffu) return TGP_E_TOO_LARGE;
        const uint32_t parts = few_parts(B * cfg->Hkv * row_blocks, rb, nchunks, pos_dev != nullptr);
        AttnQ4Args a{(const bf16 *)qb, (bf16 *)ob, (float *)scratch_dev, pos_dev, cfg->Hq, cfg->Hkv, G, cfg->TK, q_len, pos0, rows, row_blocks, parts, parts ? (nchunks + parts - 1) / parts : 0,
                     chunk, B, ldexpf(1.4426950408889634f / sqrtf((float)cfg->Dh), k_exp), ldexpf(1.f, v_exp), tiles};
        return cfg->Dh == 64 ? launch_attn<64>(a, st) : launch_attn<128>(a, st);
    }
    // more rows: keys and values once as bf16, exactly what the cache stands for, and the attention over a bf16 cache of one tile
    if ((uint64_t)B * cfg->Hkv > 65535u || q_len > 65535u * 256 || (uint64_t)q_len * G > (1u << 27)) return TGP_E_TOO_LARGE;
    const uint64_t ld = unpacked_rows(kvlen);
    const uint32_t fit = (uint32_t)std::min<uint64_t>(B, unpacked_capacity(cfg) / unpacked_bytes(cfg, kvlen)), groups = (B + fit - 1) / fit, most = (B + groups - 1) / groups;
    for (uint32_t b0 = 0; b0 < B; b0 += most) {
        const uint32_t n = std::min(most, B - b0);
        TgpTilePtrs part{};                                       // the group's pages, queries and outputs
        for (uint32_t t = 0; t <= (kvlen - 1) / cfg->TK; ++t) {
            part.k[t] = (uint8_t *)tiles.k[t] + b0 * cfg->Hkv * page_bytes(cfg->Dh, cfg->TK);
            part.v[t] = (uint8_t *)tiles.v[t] + b0 * cfg->Hkv * page_bytes(cfg->Dh, cfg->TK);
        }
        const bf16 *q = (const bf16 *)qb + (uint64_t)b0 * q_len * cfg->Hq * cfg->Dh;
        bf16 *o = (bf16 *)ob + (uint64_t)b0 * q_len * cfg->Hq * cfg->Dh, *kb = (bf16 *)scratch_dev, *vb = kb + (uint64_t)n * cfg->Hkv * ld * cfg->Dh;
        UnpackArgs u{kb, vb, nullptr, cfg->Hkv, cfg->TK, kvlen, 0, (uint32_t)ld, pos0, ldexpf(1.f, k_exp), ldexpf(1.f, v_exp), part};
        if (int rc = launch_unpack(u, cfg, n, st)) return rc;
        tgp_model_cfg one = *cfg;
        one.TK = (uint32_t)ld;
        TgpTilePtrs whole{};
        whole.k[0] = kb; whole.v[0] = vb;
        // (tgpk_attn() would take the mma.sync kernel below 128 queries: 92 us for 32 of the three sequences above)
        if (int rc = q_len < 128 ? tgpk_attn_prefill_tc5(q, whole, o, &one, n, q_len, pos0, st) : tgpk_attn(q, whole, 1, o, &one, n, q_len, pos0, nullptr, st)) return rc;
        const dim3 grid(n * cfg->Hkv, (q_len + 255) / 256);
        const NanArgs nan{o, cfg->Hq, cfg->Hkv, G, cfg->TK, q_len, pos0, part};
        if (int rc = cfg->Dh == 64 ? launch(tgp_attn_q4_nan_kernel<64>, grid, dim3(256), 0, st, 1, nan) : launch(tgp_attn_q4_nan_kernel<128>, grid, dim3(256), 0, st, 1, nan)) return rc;
    }
    return TGP_OK;
}

}  // extern "C"
