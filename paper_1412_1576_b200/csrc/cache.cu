// New tokens into a paged cache of keys and values, and masks of drafted trees.
#include <math.h>

#include "cache.cuh"
#include "rows.cuh"

namespace lda {

int cache_view(const lda_paged_cache* c, int64_t tokens, CacheView& v)
{
    if (!c || (c->dtype != LDA_F16 && c->dtype != LDA_BF16)) return LDA_EINVAL;
    if (tokens < 0 || c->n_seqs < 0 || c->pages < 0 || c->table_width < 0 || c->kv_heads < 1 || c->page_size < 1) return LDA_EINVAL;
    if (c->dim < 8 || c->dim % 8) return LDA_EINVAL;
    if (c->dim > LDA_HEAD_MAX_DIM || tokens > 0x7fffffffll || c->n_seqs > 0x7ffffffell || c->pages > 0x7fffffffll || c->kv_heads > LDA_HEADS_MAX)
        return LDA_ERANGE;
    if ((int64_t)c->table_width * c->page_size > 0x7fffffffll) return LDA_ERANGE;  // (a key's number stays inside 31 bits)
    if (c->table_stride < 0) return LDA_EINVAL;
    for (int i = 0; i < 3; ++i) {
        if (c->key_strides[i] < 0 || c->key_strides[i] % 8 || c->value_strides[i] < 0 || c->value_strides[i] % 8) return LDA_EINVAL;
        // an element's number stays inside 63 bits
        if (c->key_strides[i] > (1ll << 31) || c->value_strides[i] > (1ll << 31)) return LDA_ERANGE;
    }
    if (c->table_stride > (1ll << 31)) return LDA_ERANGE;
    if (c->n_seqs > 0 && (!c->starts || !c->offsets || !aligned(c->starts, 4) || !aligned(c->offsets, 8))) return LDA_EINVAL;
    if (c->n_seqs > 0 && c->table_width > 0 && (!c->table || !aligned(c->table, 4))) return LDA_EINVAL;
    if (c->pages > 0 && (!c->keys || !c->values || !aligned(c->keys, 16) || !aligned(c->values, 16))) return LDA_EINVAL;
    v.keys = (char*)c->keys, v.values = (char*)c->values;
    v.k_page = c->key_strides[0], v.k_slot = c->key_strides[1], v.k_head = c->key_strides[2];
    v.v_page = c->value_strides[0], v.v_slot = c->value_strides[1], v.v_head = c->value_strides[2];
    v.table = c->table, v.table_stride = c->table_stride, v.pages = c->pages, v.tokens = tokens;
    v.starts = c->starts, v.offsets = c->offsets;
    v.seqs = (int32_t)c->n_seqs, v.width = c->table_width, v.kv_heads = c->kv_heads, v.dim = c->dim;
    v.page_size = Divider((uint32_t)c->page_size);
    return LDA_OK;
}

struct AppendArgs {
    CacheView cache;
    const void *k, *v, *q;
    void* q_out;
    int64_t k_token, k_head, v_token, v_head, q_token, q_head, out_token, out_head;
    const int32_t* positions;  // null: the tokens' slots
    const float* inv_freq;
    int32_t heads, half;       // of the queries (0: none); rotated pairs of a head
    int32_t interleaved;
    Divider per_head, per_token;  // tasks of a rotated head, of a token
    int32_t turned;               // tasks of a token's rotated heads (the values' copies follow)
};

constexpr int APPEND_THREADS = 256, APPEND_TOKENS = 4;

// The cosine and sine of position x frequency.  The angle is a product of 64 bits, taken to [-pi, pi] there: in 32 bits a position of 10^6
// would leave 0.06 of an angle open.  What is left is rounded to 32 bits (2^-23 at most of an angle of 3).
__device__ __forceinline__ float2 turn_of(int position, float freq)
{
    constexpr double TURN = 6.283185307179586476925;
    const double angle = (double)position * (double)freq;
    const double rest = fma(-rint(angle * (1.0 / TURN)), TURN, angle);
    float2 cs;
    sincosf((float)rest, &cs.y, &cs.x);
    return cs;
}

// A CTA has up to four tokens: finds their sequences among all offsets, their pages, and the angles of every pair once for all heads;
// then a thread moves 16 bytes of a head (VEC; or one pair), and of its other half where the pairs lie apart.
// Bound by reading and writing each value once: four prompts of up to 8192 tokens, 32 query heads on 8 of 128 values, bf16: 86 us, 5.9 TB/s.  A call
// for few tokens by four reads that need each other (offsets, start, table, keys): 32 tokens 7.2 us.  As every CTA looks at all offsets, one token
// for each of 256, 1024, 4096 and 16 384 sequences takes 7.8, 9.8, 27 and 148 us.
template <typename T, bool VEC>
__global__ void __launch_bounds__(APPEND_THREADS) k_append(AppendArgs a)
{
    __shared__ float2 turns[APPEND_TOKENS][LDA_HEAD_MAX_DIM / 2];
    __shared__ int seqs[APPEND_TOKENS], s_position[APPEND_TOKENS], s_page[APPEND_TOKENS], s_place[APPEND_TOKENS];
    const CacheView& c = a.cache;
    const int tid = threadIdx.x;
    const int64_t first = (int64_t)blockIdx.x * APPEND_TOKENS;
    const int tokens = (int)min((int64_t)APPEND_TOKENS, c.tokens - first);
    if (tid < APPEND_TOKENS) seqs[tid] = -1;
    __syncthreads();
    // a token's sequence: every one is asked whether the token is its own, as offsets that run nowhere say nothing of the others
    for (int b = tid; b < c.seqs; b += APPEND_THREADS) {
        const int64_t lo = c.offsets[b], hi = c.offsets[b + 1];
        if (lo < 0 || hi > c.tokens || hi <= first || lo >= first + tokens) continue;
#pragma unroll
        for (int j = 0; j < APPEND_TOKENS; ++j)
            if (lo <= first + j && first + j < hi) atomicMax(&seqs[j], b);
    }
    __syncthreads();
    if (tid < tokens) {
        const int b = seqs[tid];
        int page = -2, place = 0, position = 0;  // -2: a token of no sequence, which is left alone
        if (b >= 0) {
            const CacheSeq s = c.seq(b);
            const int64_t slot = s.start + (first + tid - s.first);
            page = slot <= 0x7fffffffll ? c.page(b, (uint32_t)slot, place) : -1;
            position = a.positions ? a.positions[first + tid] : (int)slot;
        }
        s_page[tid] = page, s_place[tid] = place, s_position[tid] = position;
    }
    __syncthreads();
    for (int j = 0; j < tokens; ++j)
        for (int i = tid; i < a.half; i += APPEND_THREADS) turns[j][i] = turn_of(s_position[j], a.inv_freq[i]);
    __syncthreads();
    const int tasks = tokens * (int)a.per_token.d, rest0 = VEC && !a.interleaved ? a.half / 8 : VEC ? a.half / 4 : a.half;
    for (int task = tid; task < tasks; task += APPEND_THREADS) {
        const int j = (int)a.per_token.quotient((uint32_t)task), t = task - j * (int)a.per_token.d, page = s_page[j];
        if (page == -2) continue;
        const int64_t token = first + j;
        if (t >= a.turned) {  // a value's 16 bytes
            if (page < 0) continue;
            const int per = c.dim / 8, h = (t - a.turned) / per, at = (t - a.turned) % per * 8;
            T* to = (T*)c.values + page * c.v_page + s_place[j] * c.v_slot + h * c.v_head + at;
            *(uint4*)to = *(const uint4*)((const T*)a.v + token * a.v_token + h * a.v_head + at);
            continue;
        }
        int h = (int)a.per_head.quotient((uint32_t)t);
        const int i = t - h * (int)a.per_head.d;
        const T* from;
        T* to;
        if (h < c.kv_heads) {
            if (page < 0) continue;
            from = (const T*)a.k + token * a.k_token + h * a.k_head;
            to = (T*)c.keys + page * c.k_page + s_place[j] * c.k_slot + h * c.k_head;
        } else {
            h -= c.kv_heads;
            from = (const T*)a.q + token * a.q_token + h * a.q_head;
            to = (T*)a.q_out + token * a.out_token + h * a.out_head;
        }
        if (i >= rest0) {  // what is not rotated
            if constexpr (VEC) {
                const int at = 2 * a.half + (i - rest0) * 8;
                *(uint4*)(to + at) = *(const uint4*)(from + at);
            } else
                to[a.half + i] = from[a.half + i];  // (half pairs, then element 2 half + (i - half))
            continue;
        }
        if constexpr (!VEC) {
            const int x = a.interleaved ? 2 * i : i, y = a.interleaved ? x + 1 : i + a.half;
            const float2 cs = turns[j][i];
            const float p = cache_value(from[x]), r = cache_value(from[y]);
            to[x] = row_element<T>(p * cs.x - r * cs.y);
            to[y] = row_element<T>(p * cs.y + r * cs.x);
        } else if (a.interleaved) {
            float x[8];
            unpack<T>(*(const uint4*)(from + 8 * i), x);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 cs = turns[j][4 * i + e];
                const float p = x[2 * e], r = x[2 * e + 1];
                x[2 * e] = p * cs.x - r * cs.y;
                x[2 * e + 1] = p * cs.y + r * cs.x;
            }
            *(uint4*)(to + 8 * i) = pack<T>(x);
        } else {
            float x[8], y[8];
            unpack<T>(*(const uint4*)(from + 8 * i), x);
            unpack<T>(*(const uint4*)(from + a.half + 8 * i), y);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 cs = turns[j][8 * i + e];
                const float p = x[e], r = y[e];
                x[e] = p * cs.x - r * cs.y;
                y[e] = p * cs.y + r * cs.x;
            }
            *(uint4*)(to + 8 * i) = pack<T>(x);
            *(uint4*)(to + a.half + 8 * i) = pack<T>(y);
        }
    }
}

template <typename T>
static void run_append(AppendArgs a, cudaStream_t st)
{
    const int dim = a.cache.dim, rotated = a.cache.kv_heads + a.heads;
    // 16 bytes at a time where the pairs' halves, or the neighbours that make a pair, fill whole 16 bytes
    const bool vec = a.interleaved ? a.half % 4 == 0 : a.half % 8 == 0;
    const int per_head = !vec ? dim - a.half : a.interleaved ? dim / 8 : dim / 8 - a.half / 8;
    a.per_head = Divider((uint32_t)per_head);
    a.turned = per_head * rotated;
    a.per_token = Divider((uint32_t)(a.turned + a.cache.kv_heads * (dim / 8)));
    const unsigned grid = (unsigned)((a.cache.tokens + APPEND_TOKENS - 1) / APPEND_TOKENS);
    if (vec) k_append<T, true><<<grid, APPEND_THREADS, 0, st>>>(a);
    else k_append<T, false><<<grid, APPEND_THREADS, 0, st>>>(a);
}

// --- masks of trees ----------------------------------------------------------------------------------------------------------

constexpr int MASK_THREADS = 256, MASK_PARENTS = 2048;  // parents of a sequence that are held in shared memory

struct MaskArgs {
    const int32_t* parents;
    const int64_t* offsets;
    const int32_t* starts;  // null: 0
    int64_t tokens;
    int32_t words;
    int64_t* mask;
    int32_t* positions;  // may be null
};

// One tree of up to 256 nodes in W words: a thread has a node, and what it knows of the way up doubles from round to round: its bits and
// those of the node where they end, eight rounds for a chain of 256.  Shared memory bounds it, so a node's words behind its own are neither
// written nor read, a node that has reached the root is written once more and then no longer, and a node's place and count are one word.
// Rows go out by 16 bytes where they can.  2048 trees of up to 255 nodes, every fourth a chain: 10.4 us, without these 13.3, and walking
// node by node 41.  Up to 64 nodes have W = 1 (32 trees of 48 nodes: 2.8 us, with W = 4 3.1).
template <int W>
__device__ __forceinline__ void mask_doubling(const MaskArgs& a, int64_t lo, int n, int start, int32_t* near,
                                              unsigned long long (*s_bits)[MASK_THREADS])
{
    const int i = threadIdx.x;
    int up = i < n ? a.parents[lo + i] : -1, above = 1;  // where the bits end, and how many there are
    if (up < 0 || up >= i) up = -1;
    bool fresh = i < n;  // not yet as it is in shared memory
    unsigned long long bits[W];
#pragma unroll
    for (int w = 0; w < W; ++w) bits[w] = W == 1 || w == i >> 6 ? 1ull << (i & 63) : 0ull;
    while (__syncthreads_or(up >= 0)) {
        if (fresh) {
            near[i] = above << 16 | (up + 1);
#pragma unroll
            for (int w = 0; w < W; ++w)
                if (W == 1 || w <= i >> 6) s_bits[w][i] = bits[w];
        }
        __syncthreads();
        fresh = up >= 0;
        if (fresh) {
#pragma unroll
            for (int w = 0; w < W; ++w)
                if (W == 1 || w <= up >> 6) bits[w] |= s_bits[w][up];
            const int there = near[up];
            above += there >> 16, up = (there & 0xffff) - 1;
        }
    }
    if (i >= n) return;
    int64_t* row = a.mask + (lo + i) * a.words;
    if (W > 1 && a.words % 2 == 0 && (uintptr_t)a.mask % 16 == 0) {
#pragma unroll
        for (int w = 0; w + 1 < W; w += 2)
            if (w < a.words) *(ulonglong2*)(row + w) = make_ulonglong2(bits[w], bits[w + 1]);
    } else {
#pragma unroll
        for (int w = 0; w < W; ++w)
            if (w < a.words) row[w] = (int64_t)bits[w];
    }
    for (int w = W; w < a.words; ++w) row[w] = 0;
    if (a.positions) a.positions[lo + i] = start + above - 1;
}

// One CTA per tree.  More than 256 nodes are walked from each to the root.  Parents stand before their children, so that the places on the
// way go down and a node's words are done one after the other, from the last to the first.  The time goes with the sum of the depths, and is that
// of reads that need each other: a chain of 257, 1024, 4096 nodes 24, 234, 3330 us (of 256, by doubling, 4), of 32 768 0.18 s.
__global__ void __launch_bounds__(MASK_THREADS) k_tree_mask(MaskArgs a)
{
    __shared__ int32_t near[MASK_PARENTS];
    __shared__ unsigned long long s_bits[MASK_THREADS / 64][MASK_THREADS];
    const int b = blockIdx.x;
    const int64_t lo = a.offsets[b], hi = a.offsets[b + 1];
    if (lo < 0 || hi < lo || hi > a.tokens) return;
    const int n = (int)(hi - lo), start = a.starts ? a.starts[b] : 0;
    if (n <= 64) return mask_doubling<1>(a, lo, n, start, near, s_bits);
    if (n <= MASK_THREADS) return mask_doubling<MASK_THREADS / 64>(a, lo, n, start, near, s_bits);
    const int32_t* parents = a.parents + lo;
    if (n <= MASK_PARENTS) {
        for (int i = threadIdx.x; i < n; i += MASK_THREADS) near[i] = parents[i];
        __syncthreads();
        parents = near;
    }
    for (int i = threadIdx.x; i < n; i += MASK_THREADS) {
        int64_t* row = a.mask + (lo + i) * a.words;
        int at = i, depth = -1, word = a.words;  // words from `word` on are written
        unsigned long long bits = 0;
        while (at >= 0) {
            const int w = at >> 6;
            if (w < word) {
                if (word < a.words) row[word] = (int64_t)bits;
                for (--word; word > w; --word) row[word] = 0;
                bits = 0;
            }
            if (w < a.words) bits |= 1ull << (at & 63);
            ++depth;
            const int up = parents[at];
            at = up < at ? up : -1;
        }
        if (word < a.words) row[word] = (int64_t)bits;
        for (--word; word >= 0; --word) row[word] = 0;
        if (a.positions) a.positions[lo + i] = start + depth;
    }
}

}  // namespace lda

extern "C" int lda_append_cache(const lda_paged_cache* cache, int64_t tokens, const void* k_dev, int64_t k_token_stride,
                                int64_t k_head_stride, const void* v_dev, int64_t v_token_stride, int64_t v_head_stride,
                                const int32_t* positions_dev, const float* inv_freq_dev, int32_t rotated, int interleaved,
                                const void* q_dev, int64_t q_token_stride, int64_t q_head_stride, int32_t heads, void* q_out_dev,
                                int64_t out_token_stride, int64_t out_head_stride, void* cuda_stream)
{
    using namespace lda;
    AppendArgs a{};
    const int rc = cache_view(cache, tokens, a.cache);
    if (rc != LDA_OK) return rc;
    if (rotated < 0 || rotated % 2 || rotated > cache->dim || (rotated > 0 && (!inv_freq_dev || !aligned(inv_freq_dev, 4)))) return LDA_EINVAL;
    if (heads < 0 || !aligned(positions_dev, 4)) return LDA_EINVAL;
    if (heads > LDA_HEADS_MAX) return LDA_ERANGE;
    if (tokens == 0 || cache->n_seqs == 0) return LDA_OK;
    if (!heads_ok(k_dev, k_token_stride, k_head_stride) || !heads_ok(v_dev, v_token_stride, v_head_stride)) return LDA_EINVAL;
    if (heads > 0 && (!heads_ok(q_dev, q_token_stride, q_head_stride) || !heads_ok(q_out_dev, out_token_stride, out_head_stride))) return LDA_EINVAL;
    if (heads > 0 && q_out_dev == q_dev && (q_token_stride != out_token_stride || q_head_stride != out_head_stride)) return LDA_EINVAL;
    const int64_t most = 1ll << 31;
    if (k_token_stride > most || k_head_stride > most || v_token_stride > most || v_head_stride > most || q_token_stride > most ||
        q_head_stride > most || out_token_stride > most || out_head_stride > most)
        return LDA_ERANGE;
    const int64_t sizes[3] = {cache->pages, cache->page_size, cache->kv_heads};
    if (!strides_apart(sizes, cache->key_strides, cache->dim) || !strides_apart(sizes, cache->value_strides, cache->dim)) return LDA_EINVAL;
    if (heads > 0 && !heads_apart(q_dev, q_token_stride, q_head_stride, q_out_dev, out_token_stride, out_head_stride, tokens, heads, cache->dim)) return LDA_EINVAL;
    a.k = k_dev, a.v = v_dev, a.q = q_dev, a.q_out = q_out_dev;
    a.k_token = k_token_stride, a.k_head = k_head_stride, a.v_token = v_token_stride, a.v_head = v_head_stride;
    a.q_token = q_token_stride, a.q_head = q_head_stride, a.out_token = out_token_stride, a.out_head = out_head_stride;
    a.positions = positions_dev, a.inv_freq = inv_freq_dev, a.heads = heads, a.half = rotated / 2, a.interleaved = interleaved != 0;
    if (cache->dtype == LDA_F16) run_append<__half>(a, (cudaStream_t)cuda_stream);
    else run_append<__nv_bfloat16>(a, (cudaStream_t)cuda_stream);
    return cudaGetLastError() == cudaSuccess ? LDA_OK : LDA_ECUDA;
}

extern "C" int lda_tree_mask(const int32_t* parents_dev, const int64_t* offsets_dev, int64_t n_seqs, int64_t tokens,
                             const int32_t* starts_dev, int32_t words, int64_t* mask_dev, int32_t* positions_dev, void* cuda_stream)
{
    using namespace lda;
    if (n_seqs < 0 || tokens < 0 || words < 1) return LDA_EINVAL;
    if (n_seqs > 0x7ffffffell || tokens > 0x7fffffffll || words > LDA_MASK_MAX_WORDS) return LDA_ERANGE;
    if (n_seqs == 0 || tokens == 0) return LDA_OK;
    if (!parents_dev || !offsets_dev || !mask_dev) return LDA_EINVAL;
    if (!aligned(parents_dev, 4) || !aligned(offsets_dev, 8) || !aligned(starts_dev, 4) || !aligned(mask_dev, 8) || !aligned(positions_dev, 4))
        return LDA_EINVAL;
    const MaskArgs a{parents_dev, offsets_dev, starts_dev, tokens, words, mask_dev, positions_dev};
    k_tree_mask<<<(unsigned)n_seqs, MASK_THREADS, 0, (cudaStream_t)cuda_stream>>>(a);
    return cudaGetLastError() == cudaSuccess ? LDA_OK : LDA_ECUDA;
}
