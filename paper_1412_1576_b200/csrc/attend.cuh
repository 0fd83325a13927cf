// What the two kernels of attention over a paged cache share (attend.cu, attend_tc.cu): how the work is shared out, masks, the join.
#pragma once
#include "cache.cuh"
#include "rows.cuh"

namespace lda {

struct AttendBegun {
    int64_t row0, first;  // the item's first row, and its sequence's first token
    int head, rows;       // rows: of the tile; 0: there is no such item
    int others, unused;   // how many CTAs go on with it
};

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
    AttendBegun* begun;  // [ctas]: the item that a CTA begins and others go on with
};

// --- how the work is shared out -------------------------------------------------------------------------------------------------
// An item is a row tile of a head of a sequence; it has a unit for every tile of keys (`weight` units where it has 256 rows, as that many
// cost twice as much as 128), and ITEM_EXTRA tiles' worth behind them, without work, for what an item costs besides: queries, and sums out.  All
// units stand in one line (by sequence, head, row tile, keys), and every CTA takes an equal run of them.  So contexts of any lengths keep all CTAs
// busy to the end, few long ones too; an item that does not lie within one run leaves parts that k_attend_join puts together.
// ITEM_EXTRA of 0, 1, 2, 3: 42.5, 38.4, 38.9, 37.8 us for 33 sequences of up to 2050 slots and 13 tokens, 43.3, 39.6, 39.7, 37.5 for 64 of up to 512 and
// one token, 127.9, 128.3, 128.0, 125.3 for 16 of up to 8192 and trees of 64; by the other kernel, pages of 4 and 64 of up to 512, 37.8, 34.9, 32.9, 35.9.
constexpr int ITEM_EXTRA = 2;
__device__ __forceinline__ int64_t attend_quotient(int64_t n, int64_t d)
{
    // (a division of 64 bits is a call of its own)
    return (n | d) >> 32 ? n / d : (int64_t)((uint32_t)n / (uint32_t)d);
}
struct AttendShare {
    int64_t total, lo, hi;  // units in all, and of this CTA
    int ctas, near;         // that take part; how near to an item's end a share's moves there
    __device__ __forceinline__ int64_t begin(int c) const { return attend_quotient(total * c, ctas); }
    // A part of an item costs its CTAs and the join about as much as two tiles: a share's border that is as near to the item's first tile or
    // behind its last is moved there, and else to a tile's begin.  `from`, `left`: units of the item before the border and behind
    // it; returns by how many it moves.
    __device__ __forceinline__ int64_t moved(int64_t from, int64_t left, int weight) const
    {
        return from <= near * weight && from <= left ? -from : left <= (near + ITEM_EXTRA) * weight ? left : -(from & (weight - 1));
    }
    // The last CTA that has units of an item, first .. end - 1, that several have.
    __device__ __forceinline__ int last_of(int64_t first, int64_t end, int weight) const
    {
        int c = (int)attend_quotient(end * ctas - 1, total);
        while (begin(c) > first && begin(c) + moved(begin(c) - first, end - begin(c), weight) >= end) --c;
        return c;
    }
};

struct AttendItem {
    CacheSeq seq;
    int b, keys, row_tiles, tiles, head, row_tile, tile;
    int parts, weight;  // units of a tile of keys for all rows of a head, and for the item's
    template <int ROWS, int KEYS>
    __device__ __forceinline__ void load(const AttendArgs& a, int b_)
    {
        b = b_;
        seq = a.cache.seq(b);
        keys = (int)min((int64_t)seq.start + seq.n, (int64_t)(a.cache.width * (int)a.cache.page_size.d));
        const int64_t rows = (int64_t)seq.n * a.group;
        row_tiles = (int)((rows + ROWS - 1) / ROWS);
        parts = ROWS == 256 ? (int)((rows + 127) / 128) : row_tiles;
        tiles = max(1, (int)(((int64_t)keys + KEYS - 1) / KEYS));  // (rows without keys are written too)
    }
    template <int ROWS>
    __device__ __forceinline__ void weigh()
    {
        weight = ROWS == 256 && 2 * row_tile + 2 <= parts ? 2 : 1;
    }
    __device__ __forceinline__ int64_t units(const AttendArgs& a) const { return (int64_t)parts * (tiles + ITEM_EXTRA) * a.cache.kv_heads; }
    // Of the item, and of what stands behind its last tile.
    __device__ __forceinline__ int64_t own_units() const { return (int64_t)(tiles + ITEM_EXTRA) * weight; }
    __device__ __forceinline__ int extra_units() const { return ITEM_EXTRA * weight; }
    // To the tile that has a unit of the sequence (from `tiles` on: none has); returns how many units of the tile stand before it.
    template <int ROWS>
    __device__ __forceinline__ int at(int64_t unit)
    {
        constexpr int EACH = ROWS == 256 ? 2 : 1;  // units of a tile of a whole item
        const int64_t of_tile = tiles + ITEM_EXTRA, of_head = parts * of_tile;
        head = (int)attend_quotient(unit, of_head);
        const int64_t u = unit - head * of_head;
        row_tile = (int)attend_quotient(u, EACH * of_tile);
        weigh<ROWS>();
        const int off = (int)(u - row_tile * (EACH * of_tile));
        tile = off >> (weight - 1);
        return off & (weight - 1);
    }
    // The next tile of the line; there is one.
    template <int ROWS, int KEYS>
    __device__ __forceinline__ void next(const AttendArgs& a)
    {
        if (++tile < tiles) return;
        tile = 0;
        if (++row_tile >= row_tiles) {
            row_tile = 0;
            if (++head >= a.cache.kv_heads) {
                head = 0;
                do load<ROWS, KEYS>(a, b + 1);
                while (row_tiles == 0 && b + 1 < a.cache.seqs);
            }
        }
        weigh<ROWS>();
    }
};

// This CTA's share, and its first unit's item.  `red`: a number for each warp in shared memory.  False: it has none.
template <int ROWS, int KEYS>
__device__ __forceinline__ bool attend_share(const AttendArgs& a, int cta, AttendShare& s, AttendItem& item, unsigned long long* red)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads >> 5, seqs = a.cache.seqs;
    __shared__ int s_b[2];
    __shared__ unsigned long long s_before[2];
    // (one copy of the code for both rounds: a CTA runs it once, and waits for every line of it to be fetched)
    unsigned long long mine = 0, start = 0, before = 0;
#pragma unroll 1
    for (int round = 0; round < 2; ++round) {
#pragma unroll 1
        for (int base = 0; base < seqs; base += threads) {
            if (round == 0 || seqs > threads) {  // (else the first round's scan says it)
                AttendItem own;
                mine = 0;
                if (base + tid < seqs) {
                    own.load<ROWS, KEYS>(a, base + tid);
                    mine = own.units(a);
                }
                unsigned long long upto = mine;
#pragma unroll 1
                for (int o = 1; o < 32; o <<= 1) {
                    const unsigned long long x = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += x;
                }
                if (base > 0 || round > 0) __syncthreads();
                if (lane == 31) red[warp] = upto;
                __syncthreads();
                start = before + upto - mine;
#pragma unroll 1
                for (int w = 0; w < warps; ++w) {
                    if (w < warp) start += red[w];
                    before += red[w];
                }
            }
            if (round > 0)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const unsigned long long at = (unsigned long long)(i ? s.hi : s.lo);
                    if (mine && start <= at && at < start + mine) s_b[i] = base + tid, s_before[i] = start;
                }
        }
        if (round > 0) break;
        s.total = (int64_t)before;
        s.ctas = (int)min((int64_t)a.ctas, max((int64_t)1, s.total / (ROWS == 256 ? 2 : 1)));
        if (s.total == 0 || cta >= s.ctas) return false;
        s.lo = s.begin(cta), s.hi = s.begin(cta + 1);
        // (two tiles near against one: 25.9 us against 28.0 for 33 sequences of up to 500 slots, five tiles a CTA; 41.6 against 38.8 for up to 2050 slots,
        // 14 tiles a CTA, and 39.1 against 37.8 for two sequences of up to 8192 with trees of 64, as many)
        s.near = s.total > s.ctas ? (s.total >= 2ll * s.ctas && s.total < 8ll * s.ctas ? 2 : 1) : 0;
        before = 0;
    }
    __syncthreads();
    // the borders, moved; the first unit's item stays
#pragma unroll 1
    for (int i = 1; i >= 0; --i) {
        if (i == 1 && s.hi == s.total) continue;
        const int64_t at = i ? s.hi : s.lo;
        item.load<ROWS, KEYS>(a, s_b[i]);
        const int part = item.at<ROWS>(at - (int64_t)s_before[i]);
        if (at == 0) continue;
        const int64_t from = (int64_t)item.tile * item.weight + part, by = s.moved(from, item.own_units() - from, item.weight);
        if (i == 1) s.hi += by;
        else {
            s.lo += by;
            if (by <= 0) item.tile = (int)((from + by) >> (item.weight - 1));
            else if (s.lo < s.total) {
                item.tile = item.tiles - 1;
                item.next<ROWS, KEYS>(a);
            }
        }
    }
    return s.lo < s.hi;
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

// Whether one of a group's eight values is infinite or no number: times zero it is NaN.
template <typename T>
__device__ __forceinline__ bool has_wild(uint4 g)
{
    using T2 = std::conditional_t<T_is_bf16<T>, __nv_bfloat162, __half2>;
    const uint32_t none = 0;
    const auto zero = [&](uint32_t w) {
        const T2 x = __hmul2(*reinterpret_cast<const T2*>(&w), *reinterpret_cast<const T2*>(&none));
        return *reinterpret_cast<const uint32_t*>(&x);
    };
    return ((zero(g.x) | zero(g.y) | zero(g.z) | zero(g.w)) & 0x7FFF7FFFu) != 0;
}
// The group without such values.
template <typename T>
__device__ __noinline__ uint4 without_wild(uint4 g)
{
    constexpr uint32_t EXP = T_is_bf16<T> ? 0x7F80u : 0x7C00u;
    uint32_t w[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((w[i] & EXP) == EXP) w[i] &= 0xFFFF0000u;
        if ((w[i] >> 16 & EXP) == EXP) w[i] &= 0x0000FFFFu;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// The other kernel (attend_tc.cu): whether it takes a cache, and its launch (the parts are joined by the caller).
bool attend_tc_takes(const lda_paged_cache& cache);
cudaError_t attend_tc(const AttendArgs& a, const lda_paged_cache& cache, cudaStream_t st);

}  // namespace lda
