// What the attention kernels over a cache in pages share: a sequence's rows and the keys that they see.
#pragma once
#include <cuda_bf16.h>
#include <cstdint>

struct TgpPagedAttn {
    const __nv_bfloat16 *q, *k, *v; __nv_bfloat16 *o; const int32_t *table, *start, *end;
    uint32_t Hq, Hkv, G, P, W;                                   // query heads, KV heads, query heads of one, positions of a page, pages of a table's row
    uint32_t B, T, q_max, kv_max, n_pages, window, sinks;
    uint32_t few;                                                // a sequence of up to so many rows * G is the few-rows kernel's
    float sl2;                                                   // log2(e) / sqrt(Dh)
    uint32_t b0;                                                 // first sequence of this launch (few rows)
};

// Rows first ... first + n - 1 of q and o, at positions end - n ... end - 1.  n == 0: nothing to do.  What is on the device is not trusted beyond the bounds that the
// call was checked with: with rows outside the arrays a sequence has none, with a length or a number of rows outside the bounds it is idle, its rows zero.
struct TgpPagedSeq { uint32_t first, n, end; bool idle; };

__device__ __forceinline__ TgpPagedSeq tgp_paged_seq(const TgpPagedAttn &a, uint32_t b) {
    const int s0 = a.start[b], s1 = a.start[b + 1], e = a.end[b];
    TgpPagedSeq s{(uint32_t)s0, 0, (uint32_t)e, false};
    if (s0 < 0 || s1 <= s0 || (uint32_t)s1 > a.T) return s;
    s.n = (uint32_t)(s1 - s0);
    s.idle = s.n > a.q_max || e < (int)s.n || (uint32_t)e > a.kv_max;
    return s;
}

// Keys are visited in chunks of C: those of the first `sinks` positions that lie before the window of every row (from chunk 0 on), then from the first row's window to the last position.
struct TgpPagedKeys {
    uint32_t low, head, skip, chunks;                            // lowest position in the first row's window; chunks of first positions; chunks between them and the others; chunks in all
    __device__ __forceinline__ uint32_t chunk(uint32_t i) const { return i < head ? i : i + skip; }
};

template <uint32_t C>
__device__ __forceinline__ TgpPagedKeys tgp_paged_keys(const TgpPagedAttn &a, uint32_t first_pos, uint32_t last_pos) {
    TgpPagedKeys k;
    k.low = a.window && first_pos >= a.window ? first_pos - a.window + 1 : 0;
    const uint32_t sinks = a.sinks < k.low ? a.sinks : k.low;
    k.head = (sinks + C - 1) / C;
    const uint32_t from = k.low / C > k.head ? k.low / C : k.head, to = last_pos / C + 1;
    k.head = k.head < to ? k.head : to;
    k.skip = from > k.head ? from - k.head : 0;
    k.chunks = to > from ? k.head + (to - from) : k.head;
    return k;
}

// is the key at position j visible to the row at position p?
__device__ __forceinline__ bool tgp_paged_sees(const TgpPagedAttn &a, uint32_t p, uint32_t j) { return j <= p && (!a.window || p - j < a.window || j < a.sinks); }

// Counters in a scratch of any contents: a word is a number of arrivals only with this in its upper half - a NaN that no arithmetic gives, so whatever else the memory held, partials of an earlier call
// among it, counts as 0.  The last arrival puts 0 back.
constexpr unsigned long long TGP_PAGED_COUNTS = 0xffa5c3d1ull << 32;

// How many have arrived at a counter, this one included.  What the CTA has written before its last barrier is seen by who arrives later.
__device__ __forceinline__ uint32_t tgp_paged_arrive(unsigned long long *counter) {
    asm volatile("fence.acq_rel.gpu;" ::: "memory");
    unsigned long long was = atomicAdd(counter, 1ull);
    // Not a number of arrivals yet: the first that replaces it is the first to have arrived.  Others may have added to it meanwhile; they have seen so, too, and arrive here.
    while ((was & ~0xffffffffull) != TGP_PAGED_COUNTS) {
        const unsigned long long now = atomicAdd(counter, 0ull);
        if ((now & ~0xffffffffull) == TGP_PAGED_COUNTS) was = atomicAdd(counter, 1ull);
        else if (atomicCAS(counter, now, TGP_PAGED_COUNTS + 1) == now) was = TGP_PAGED_COUNTS;
    }
    asm volatile("fence.acq_rel.gpu;" ::: "memory");
    return (uint32_t)was + 1;
}

// sequences of more than a.few rows * G, on tcgen05 (tgp_attn_paged_sm100.cu); counter: as above, of tiles begun.  Its successor on the stream is launched when what the kernel waits for has completed.
int tgpk_attn_paged_many(const TgpPagedAttn &a, uint32_t Dh, unsigned long long *counter, cudaStream_t st);
