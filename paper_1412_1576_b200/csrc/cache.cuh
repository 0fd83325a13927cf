// Shared pieces of the operators on a paged cache of keys and values (cache.cu, attend.cu).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/lda_b200.h"

namespace lda {

// Division of numbers below 2^31 by a number that a launch knows, after Granlund and Montgomery (Division by invariant integers using
// multiplication, 1994): n d^-1 as a product by a 33-bit reciprocal rounded up (off by less than 2^-31 / d, which no quotient of such numbers notices).
struct Divider {
    uint32_t d, magic, shift;
    Divider() = default;
    explicit Divider(uint32_t by) : d(by), shift(0)
    {
        while (shift < 31 && (1u << shift) < by) ++shift;
        magic = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << shift) - by)) / by + 1);
    }
    __device__ __forceinline__ uint32_t quotient(uint32_t n) const { return (uint32_t)(((uint64_t)__umulhi(n, magic) + n) >> shift); }
};

// A sequence's part of the call: its new tokens' first row, their number, and the keys in the cache before them.
struct CacheSeq {
    int64_t first;
    int n, start;
};

struct CacheView {
    char *keys, *values;
    int64_t k_page, k_slot, k_head, v_page, v_slot, v_head;  // strides in elements
    const int32_t* table;
    int64_t table_stride, pages, tokens;
    const int32_t* starts;
    const int64_t* offsets;
    int32_t seqs, width, kv_heads, dim;
    Divider page_size;

    // Offsets that do not run upwards inside [0, tokens] leave the sequence out; a start below 0 counts as 0.
    __device__ __forceinline__ CacheSeq seq(int b) const
    {
        const int64_t lo = offsets[b], hi = offsets[b + 1];
        const int start = starts[b];
        const bool ok = lo >= 0 && hi >= lo && hi <= tokens;
        return CacheSeq{lo, ok ? (int)(hi - lo) : 0, start > 0 ? start : 0};
    }
    // The page of a slot of sequence b, or -1 where the table has none, and the slot's place in it.
    __device__ __forceinline__ int page(int b, uint32_t slot, int& place) const
    {
        const uint32_t i = page_size.quotient(slot);
        place = (int)(slot - i * page_size.d);
        if (i >= (uint32_t)width) return -1;
        const int p = table[b * table_stride + i];
        return p >= 0 && p < pages ? p : -1;
    }
};

// What both entry points refuse of a cache, and its view.
int cache_view(const lda_paged_cache* cache, int64_t tokens, CacheView& view);

// Strides of rows of heads in elements, and where they start: multiples of 16 bytes.
inline bool heads_ok(const void* p, int64_t token_stride, int64_t head_stride)
{
    return p && (uintptr_t)p % 16 == 0 && token_stride % 8 == 0 && head_stride % 8 == 0 && token_stride >= 0 && head_stride >= 0;
}

// Whether no two elements of a tensor that is written to share their place, by dimensions of n values and a stride each, `width` consecutive elements in
// the innermost: a stride passes over all that the smaller ones cover, as in any permuted or sliced tensor.
template <int N>
inline bool strides_apart(const int64_t (&n)[N], const int64_t (&stride)[N], int64_t width)
{
    uint64_t covered = (uint64_t)width;
    bool done[N] = {};
    for (int round = 0; round < N; ++round) {
        int least = -1;
        for (int i = 0; i < N; ++i)
            if (!done[i] && n[i] > 1 && (least < 0 || stride[i] < stride[least])) least = i;
        if (least < 0) break;
        done[least] = true;
        if ((uint64_t)stride[least] < covered) return false;
        covered += (uint64_t)(n[least] - 1) * (uint64_t)stride[least];
    }
    return true;
}

// Whether rows of heads that are written (of 16-bit elements) share no place with each other, and none with those that are read but for lying in their
// very places.
inline bool heads_apart(const void* q, int64_t q_token, int64_t q_head, const void* out, int64_t out_token, int64_t out_head, int64_t tokens, int64_t heads,
                        int64_t dim)
{
    if (!strides_apart({tokens, heads}, {out_token, out_head}, dim)) return false;
    if (tokens == 1) q_token = out_token = 0;  // (never taken)
    if (heads == 1) q_head = out_head = 0;
    const int64_t delta = ((intptr_t)out - (intptr_t)q) / 2;
    if (delta >= (tokens - 1) * q_token + (heads - 1) * q_head + dim || -delta >= (tokens - 1) * out_token + (heads - 1) * out_head + dim) return true;
    if (q_token != out_token || q_head != out_head) return false;
    if (delta == 0) return true;
    // two parts of the same rows: is there a token and a head with |delta + token x stride + head x stride| < dim?
    for (int64_t h = 1 - heads; h < heads; ++h) {
        const int64_t at = delta + h * q_head, near = q_token ? -at / q_token : 0;
        for (int64_t t = near - 1; t <= near + 1; ++t)
            if (t > -tokens && t < tokens && at + t * q_token < dim && at + t * q_token > -dim) return false;
    }
    return true;
}

__device__ __forceinline__ float cache_value(__half x) { return __half2float(x); }
__device__ __forceinline__ float cache_value(__nv_bfloat16 x) { return __bfloat162float(x); }

}  // namespace lda
