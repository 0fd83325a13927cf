// What the two kernels of attention over a paged cache share (attend.cu, attend_tc.cu): how the work is shared out, masks, the join.
#pragma once
#include "cache.cuh"
#include "rows.cuh"

namespace lda {

struct AttendArgs {
    CacheView cache;
    const void* q;
    void* out;
    int64_t q_token, q_head, out_token, out_head, mask_stride;
    const int64_t* mask;  // null: a token sees those before it and itself
    int32_t mask_words, heads, group;
    float scale;  // by which a score becomes a power of two's exponent
    int ctas, rows;  // rows of a tile
    float* part;   // [2 ctas][rows][padded dim]: sums of parts of an item
    float2* ml;    // [2 ctas][rows]: their maxima and norms
    int4* desc;    // [ctas]: the item that a CTA begins and others go on with: sequence (-1: none), head, row tile, how many others
};

// --- how the work is shared out -------------------------------------------------------------------------------------------------
// An item is a row tile of a head of a sequence; it has a unit for every tile of keys.  All units stand in one line (by sequence, head, row
// tile, keys), and every CTA takes an equal run of them.  So contexts of any lengths keep all CTAs busy to the end, few long ones too; an item
// that does not lie within one run leaves parts that k_attend_join puts together.
__device__ __forceinline__ int64_t attend_quotient(int64_t n, int64_t d)
{
    // (a division of 64 bits is a call of its own)
    return (n | d) >> 32 ? n / d : (int64_t)((uint32_t)n / (uint32_t)d);
}
struct AttendShare {
    int64_t total, lo, hi;  // units in all, and of this CTA
    int ctas;               // that take part
    __device__ __forceinline__ int64_t begin(int c) const { return attend_quotient(total * c, ctas); }
    // The CTA that has unit u.
    __device__ __forceinline__ int owner(int64_t u) const { return (int)attend_quotient((u + 1) * ctas - 1, total); }
};

struct AttendItem {
    CacheSeq seq;
    int b, keys, row_tiles, tiles, head, row_tile, tile;
    template <int ROWS, int KEYS>
    __device__ __forceinline__ void load(const AttendArgs& a, int b_)
    {
        b = b_;
        seq = a.cache.seq(b);
        keys = (int)min((int64_t)seq.start + seq.n, (int64_t)(a.cache.width * (int)a.cache.page_size.d));
        row_tiles = (int)(((int64_t)seq.n * a.group + ROWS - 1) / ROWS);
        tiles = max(1, (int)(((int64_t)keys + KEYS - 1) / KEYS));  // (rows without keys are written too)
    }
    __device__ __forceinline__ int64_t units(const AttendArgs& a) const { return (int64_t)row_tiles * tiles * a.cache.kv_heads; }
    __device__ __forceinline__ void at(int64_t unit)
    {
        const int64_t item = attend_quotient(unit, tiles);
        tile = (int)(unit - item * tiles);
        head = (int)attend_quotient(item, row_tiles);
        row_tile = (int)(item - (int64_t)head * row_tiles);
    }
    // The next unit of the line; there is one.
    template <int ROWS, int KEYS>
    __device__ __forceinline__ void next(const AttendArgs& a)
    {
        if (++tile < tiles) return;
        tile = 0;
        if (++row_tile < row_tiles) return;
        row_tile = 0;
        if (++head < a.cache.kv_heads) return;
        head = 0;
        do load<ROWS, KEYS>(a, b + 1);
        while (row_tiles == 0 && b + 1 < a.cache.seqs);
    }
};

// Units that a CTA takes at least: what joining a part costs is about what a few tiles cost.
constexpr int LEAST_UNITS = 2;

// This CTA's share, and its first unit's item.  `red`: a number for each warp in shared memory.  False: it has none.
template <int ROWS, int KEYS>
__device__ __forceinline__ bool attend_share(const AttendArgs& a, int cta, AttendShare& s, AttendItem& item, unsigned long long* red)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads >> 5, seqs = a.cache.seqs;
    __shared__ int s_b;
    __shared__ unsigned long long s_before;
    AttendItem own;
    unsigned long long mine = 0;
    const auto look = [&](int b) {
        mine = 0;
        if (b < seqs) {
            own.load<ROWS, KEYS>(a, b);
            mine = own.units(a);
        }
    };
    // units before this thread's sequence and in all of the threads'
    const auto scan = [&](unsigned long long& all) {
        unsigned long long upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        if (lane == 31) red[warp] = upto;
        __syncthreads();
        unsigned long long start = upto - mine;
        all = 0;
        for (int w = 0; w < warps; ++w) {
            if (w < warp) start += red[w];
            all += red[w];
        }
        return start;
    };
    unsigned long long all, start = 0;
    s.total = 0;
    for (int base = 0; base < seqs; base += threads) {
        if (base > 0) __syncthreads();
        look(base + tid);
        start = scan(all);
        s.total += all;
    }
    s.ctas = (int)min((int64_t)a.ctas, max((int64_t)1, s.total / LEAST_UNITS));
    if (s.total == 0 || cta >= s.ctas) return false;
    s.lo = s.begin(cta), s.hi = s.begin(cta + 1);
    // the sequence that has unit lo
    const unsigned long long lo = (unsigned long long)s.lo;
    unsigned long long before = 0;
    for (int base = 0; base < seqs; base += threads) {
        if (seqs > threads) {  // (else the one scan there was says it)
            __syncthreads();
            look(base + tid);
            start = before + scan(all);
            before += all;
        }
        if (mine && start <= lo && lo < start + mine) s_b = base + tid, s_before = start;
    }
    __syncthreads();
    item.load<ROWS, KEYS>(a, s_b);
    item.at(s.lo - (int64_t)s_before);
    return true;
}

// --- masks -----------------------------------------------------------------------------------------------------------------------

// Which of 64 keys (bit j: key 64 tile + j) a new token, number `place` of its sequence, sees.
__device__ __forceinline__ unsigned long long attend_window(const AttendArgs& a, const CacheSeq& seq, int place, int tile)
{
    const int64_t from = (int64_t)tile * 64 - seq.start;  // the new token that the first key belongs to
    if (from <= -64) return ~0ull;
    const auto word = [&](int64_t i) -> unsigned long long {
        if (!a.mask) {
            const int64_t left = place - 64 * i;  // bits 0..left
            return left >= 63 ? ~0ull : left < 0 ? 0ull : (2ull << left) - 1;
        }
        return i < a.mask_words ? (unsigned long long)a.mask[(seq.first + place) * a.mask_stride + i] : 0ull;
    };
    if (from < 0) return word(0) << -from | ((1ull << -from) - 1);
    const int64_t i = from >> 6;
    const int shift = (int)(from & 63);
    return word(i) >> shift | (shift ? word(i + 1) << (64 - shift) : 0ull);
}

// --- values ----------------------------------------------------------------------------------------------------------------------

template <typename T>
__device__ __forceinline__ uint32_t pack_two(float x, float y)
{
    if constexpr (T_is_bf16<T>) {
        const __nv_bfloat162 two = __floats2bfloat162_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&two);
    } else {
        const __half2 two = __floats2half2_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&two);
    }
}

// Exponent that is added to all of a row's probabilities before they are rounded for the second product: fp16 has full precision
// only down to 2^-14, which a row of a hundred thousand keys reaches; up to 2^14 it has as much room above 1.
template <typename T>
constexpr float RAISE = T_is_bf16<T> ? 0.0f : 14.0f;

// Whether one of a group's eight values is infinite or no number; such values become zero.
template <typename T>
__device__ __forceinline__ bool drop_wild(uint4& g)
{
    constexpr uint32_t EXP = T_is_bf16<T> ? 0x7F80u : 0x7C00u;
    uint32_t w[4] = {g.x, g.y, g.z, g.w};
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((w[i] & EXP) == EXP) w[i] &= 0xFFFF0000u, any = true;
        if ((w[i] >> 16 & EXP) == EXP) w[i] &= 0x0000FFFFu, any = true;
    }
    g = make_uint4(w[0], w[1], w[2], w[3]);
    return any;
}

// The other kernel (attend_tc.cu): whether it takes a cache, and its launch (the parts are joined by the caller).
bool attend_tc_takes(const lda_paged_cache& cache);
cudaError_t attend_tc(const AttendArgs& a, const lda_paged_cache& cache, cudaStream_t st);

}  // namespace lda
