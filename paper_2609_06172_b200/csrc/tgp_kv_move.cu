// Sequences of a batch copied, forked, compacted and freed inside the KV tiles.
//
// A call is a set of pairs (from, to) over the B places of every tile, all sources read before any destination is written.  The host puts them into an
// order in which that comes by itself: a place is written once nobody still has to read it, and what is left then are cycles, which are
// swapped along.  On the device a thread owns the same bytes of every place and walks the list, so no thread waits for another; the
// threads' bytes are neighbours.  Bound by HBM: each source is read once, each destination written once (one sequence of 2111 positions of 2 x 8 heads of 128 in bf16
// to fifteen others: 138 MB in 23 us, 6.0 TB/s; 20 of 700 positions in 4 bits to other places: 7 us, of which HBM needs 3.5).
#include <cuda_runtime.h>
#include <algorithm>
#include <cstdint>
#include <new>
#include <vector>
#include "tgp.h"
#include "tgp_kernels.h"
#include "tgp_launch.cuh"

namespace {

using namespace tgp_launch;

constexpr uint32_t STEPS_MAX = 256, ZERO = 0xffffu;                      // steps of a launch; a source that is zeros
struct Step { uint16_t from, to; };
struct MoveArgs {
    uint32_t n_copies, n_steps, TK, len, heads, row, row2;                // heads of a page; bytes of a position: codes or bf16 values, scales.  Steps from n_copies on swap
    uint64_t head_bytes;
    Step steps[STEPS_MAX];
    TgpTilePtrs tiles;
};

// Takes the steps for U pieces of type T at at[] in place 0; places are `place` bytes apart.  No place that a step before the swaps reads has been written by an earlier
// step, so the sources of G steps are read together, before any of them is written: a list of copies waits for memory once in G steps, not in each
// (20 sequences of 700 positions in 4 bits moved in one batch of 61: 14 us step by step).
template <typename T, int U, int G>
__device__ __forceinline__ void walk(const MoveArgs &a, uint8_t *(&at)[U], const bool (&ok)[U], uint64_t place) {
    T x[G][U];
    for (uint32_t s = 0; s < a.n_copies; s += G) {
#pragma unroll
        for (uint32_t g = 0; g < G; ++g)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t from = s + g < a.n_copies ? a.steps[s + g].from : ZERO;
                x[g][u] = T{};
                if (ok[u] && from != ZERO) x[g][u] = *reinterpret_cast<const T *>(at[u] + from * place);
            }
#pragma unroll
        for (uint32_t g = 0; g < G; ++g)
#pragma unroll
            for (int u = 0; u < U; ++u) if (ok[u] && s + g < a.n_copies) *reinterpret_cast<T *>(at[u] + a.steps[s + g].to * place) = x[g][u];
    }
    for (uint32_t s = a.n_copies; s < a.n_steps; ++s) {
        const uint64_t p = a.steps[s].from * place, q = a.steps[s].to * place;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (ok[u]) { x[0][u] = *reinterpret_cast<const T *>(at[u] + p); x[1][u] = *reinterpret_cast<const T *>(at[u] + q); }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (ok[u]) { *reinterpret_cast<T *>(at[u] + q) = x[0][u]; *reinterpret_cast<T *>(at[u] + p) = x[1][u]; }
    }
}

// Of a tile's positions in use: the 16-byte pieces of the first kind of row, head by head, then the rows of scales, one per position.
template <int U, int G>
__global__ void __launch_bounds__(256) tgp_kv_move_kernel(const __grid_constant__ MoveArgs a) {
    pdl_enter();
    const uint32_t tile = blockIdx.y >> 1, used = min(a.TK, a.len - tile * a.TK);
    uint8_t *base = reinterpret_cast<uint8_t *>(blockIdx.y & 1 ? a.tiles.v[tile] : a.tiles.k[tile]);
    const uint64_t place = a.head_bytes * a.heads;
    const uint32_t per_head = used * (a.row / 16), wide = per_head * a.heads, narrow = a.row2 ? used * a.heads : 0;
    const uint32_t stride = gridDim.x * blockDim.x;
    uint8_t *at[U];
    bool ok[U];
    for (uint32_t i0 = blockIdx.x * blockDim.x + threadIdx.x; i0 < wide; i0 += U * stride) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t i = i0 + u * stride, h = i / per_head;
            ok[u] = i < wide;
            at[u] = base + h * a.head_bytes + (uint64_t)(i - h * per_head) * 16;
        }
        walk<uint4, U, G>(a, at, ok, place);
    }
    for (uint32_t i0 = blockIdx.x * blockDim.x + threadIdx.x; i0 < narrow; i0 += U * stride) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t i = i0 + u * stride, h = i / used;
            ok[u] = i < narrow;
            at[u] = base + h * a.head_bytes + (uint64_t)a.TK * a.row + (uint64_t)(i - h * used) * a.row2;
        }
        if (a.row2 == 8) walk<uint2, U, G>(a, at, ok, place);
        else walk<uint32_t, U, G>(a, at, ok, place);
    }
}

// The pairs as steps that may be taken one after the other; false where they are no map of places.
// First copies, none of which reads what one before it has written, then swaps.
bool in_order(const int32_t *src, const int32_t *dst, uint32_t n, uint32_t B, std::vector<Step> &steps, size_t &n_copies) {
    std::vector<int32_t> from(B, -2);                            // source of a place that is written; -2: none, or itself
    std::vector<uint32_t> readers(B, 0), next;
    for (uint32_t i = 0; i < n; ++i) {
        if (dst[i] < 0 || (uint32_t)dst[i] >= B || src[i] < -1 || src[i] >= (int32_t)B || from[dst[i]] != -2) return false;
        from[dst[i]] = src[i];
    }
    for (uint32_t b = 0; b < B; ++b) {
        if (from[b] == (int32_t)b) from[b] = -2;
        if (from[b] >= 0) ++readers[from[b]];
    }
    for (uint32_t b = 0; b < B; ++b) if (from[b] != -2 && !readers[b]) next.push_back(b);
    // (by source, so that a source that goes to several places is read once)
    std::stable_sort(next.begin(), next.end(), [&](uint32_t x, uint32_t y) { return from[x] < from[y]; });
    for (size_t i = 0; i < next.size(); ++i) {
        const uint32_t to = next[i];
        const int32_t s = from[to];
        steps.push_back({s < 0 ? (uint16_t)ZERO : (uint16_t)s, (uint16_t)to});
        from[to] = -2;
        if (s >= 0 && !--readers[s] && from[s] != -2) next.push_back((uint32_t)s);
    }
    n_copies = steps.size();
    for (uint32_t b = 0; b < B; ++b)                             // what is left are cycles: b takes from[b], which takes ... , which takes b
        for (uint32_t at = b; from[at] != -2;) {
            const uint32_t s = (uint32_t)from[at];
            from[at] = -2;
            if (from[s] == -2) break;                            // back at b, which holds what the last one is to have
            steps.push_back({(uint16_t)s, (uint16_t)at});
            at = s;
        }
    return true;
}

}  // namespace

extern "C" int tgp_k_kv_move(void *const *k_tiles, void *const *v_tiles, uint32_t n_tiles, const int32_t *src, const int32_t *dst, uint32_t n, const tgp_model_cfg *cfg, uint32_t form,
                             uint32_t B, uint32_t len, void *stream) try {
    if (!cfg || !cfg->TK || !cfg->Hkv || !cfg->Dh || (form != TGP_KV_BF16 && form != TGP_KV_Q4) || B > cfg->B || (n && (!src || !dst)) || n > B) return TGP_E_INVAL;
    if (form == TGP_KV_Q4 ? ((cfg->Dh != 64 && cfg->Dh != 128) || cfg->TK % 16) : cfg->Dh % 8 != 0) return TGP_E_INVAL;
    if (len > cfg->max_len || (uint64_t)n_tiles * cfg->TK < len) return TGP_E_INVAL;
    if (n_tiles > TGP_MAX_TILES || B > 32768) return TGP_E_TOO_LARGE;
    if (!k_tiles || !v_tiles) return TGP_E_INVAL;
    MoveArgs a{};
    const uint32_t tiles = len / cfg->TK + (len % cfg->TK != 0);
    a.TK = cfg->TK; a.len = len; a.heads = cfg->Hkv;
    a.row = form == TGP_KV_Q4 ? cfg->Dh / 2 : cfg->Dh * 2;
    a.row2 = form == TGP_KV_Q4 ? cfg->Dh / 16 : 0;
    a.head_bytes = (uint64_t)cfg->TK * (a.row + a.row2);
    if (cfg->Dh > (1u << 20) || cfg->TK > (1u << 26) || cfg->Hkv > (1u << 20)) return TGP_E_TOO_LARGE;
    const uint64_t columns = (uint64_t)std::min(cfg->TK, len) * (a.row / 16);
    if (columns > (1u << 29) || columns * cfg->Hkv > (1u << 29)) return TGP_E_TOO_LARGE;
    for (uint32_t t = 0; t < tiles; ++t) {
        a.tiles.k[t] = k_tiles[t]; a.tiles.v[t] = v_tiles[t];
        if (!k_tiles[t] || !v_tiles[t] || ((reinterpret_cast<uintptr_t>(k_tiles[t]) | reinterpret_cast<uintptr_t>(v_tiles[t])) & 15u)) return TGP_E_INVAL;
    }
    std::vector<Step> steps;
    size_t n_copies = 0;
    if (!in_order(src, dst, n, B, steps, n_copies)) return TGP_E_INVAL;
    if (!len) return TGP_OK;
    for (size_t at = 0; at < steps.size(); at += STEPS_MAX) {
        a.n_steps = (uint32_t)std::min<size_t>(STEPS_MAX, steps.size() - at);
        a.n_copies = (uint32_t)std::min<size_t>(a.n_steps, n_copies > at ? n_copies - at : 0);
        std::copy(steps.begin() + at, steps.begin() + at + a.n_steps, a.steps);
        // one piece a thread, four steps at a time (20 sequences of 700 positions in 4 bits 7.0 us, 8.7 with two pieces); with one or two steps, four pieces
        const uint32_t U = a.n_copies > 2 ? 1 : 4;
        const dim3 grid((uint32_t)std::min<uint64_t>((columns * cfg->Hkv + 256 * U - 1) / (256 * U), 1u << 16), 2 * tiles);
        if (int rc = U == 1 ? launch(tgp_kv_move_kernel<1, 4>, grid, dim3(256), 0, (cudaStream_t)stream, 1, a) : launch(tgp_kv_move_kernel<4, 2>, grid, dim3(256), 0, (cudaStream_t)stream, 1, a)) return rc;
    }
    return TGP_OK;
} catch (const std::bad_alloc &) { return TGP_E_TOO_LARGE; }
