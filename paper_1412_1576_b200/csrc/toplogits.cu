// The largest logits of every row, with their words, and the row's log-sum-exp.
//
// A row's words are ordered by value (NaN first), equal values by the lower word; what is minus infinity is not listed.
#include <algorithm>

#include "lda_device.cuh"
#include "rows.cuh"

namespace lda {

struct TopArgs {
    const void* logits;
    int64_t stride;
    int32_t V, top;
    float scale;     // log2(e) / temperature
    double inv_tau;
    int32_t* ids;
    void* values;
    float* lse;
    int ring;  // bytes of the walk's ring, or of the lists that take its place
};

constexpr int TOP_GROUPS = 4;     // groups of a lane in a chunk (two: 242 us for 229)
constexpr int TOP_DEPTH = 2;      // chunks on their way (three: the same time)
constexpr int TOP_VALUES = 1024;  // groups of pieces whose largest keys give the border, at most
constexpr uint32_t TOP_LOWEST = (KEY_NEG_INF >> 16) + 1;  // first half-key above minus infinity
// Words and pieces that may be left for lists of `top`: about four times what rows in no order leave (95 words for lists of 64 of 131 072).
// Rows in order of their words' frequency and long ties may leave more (534 with a normal part of 0.7 beside the logarithm of the rank, all
// of a row all alike) and then go by top_by_bytes: 4096 such rows of bf16 take 9.6 and 10.0 ms.
__host__ __device__ constexpr int top_room(int top) { return top <= 64 ? 512 : top <= 256 ? 1024 : 2048; }

// What takes the ring's place behind the pass.
struct TopLists {
    unsigned long long* list;  // the words that are left
    int* queue;                // the pieces that are read again
    __device__ __forceinline__ TopLists(void* at, int room)
        : list((unsigned long long*)at), queue((int*)at + 2 * room)
    {
    }
    static __host__ __device__ constexpr int bytes(int room) { return 12 * room; }
};
struct TopCounts {
    int n, queued, need;
    uint32_t prefix;
    int hist[256];
};

__device__ __forceinline__ unsigned long long top_entry(uint32_t key, int v)
{
    return ((unsigned long long)key << 32) | (0xFFFFFFFFu - (uint32_t)v);
}

__device__ __forceinline__ void top_order(unsigned long long& x, unsigned long long& y, bool descending)
{
    const bool swap = (x < y) == descending;
    const unsigned long long t = x;
    x = swap ? y : x;
    y = swap ? t : y;
}

// Sorts list[128 w .. 128 w + 127] for every w, descending, by a warp each, four places to a lane; places from n on become 0.
constexpr int TOP_RUN = 128;
__device__ __forceinline__ void top_sort_runs(unsigned long long* list, int n)
{
    const int lane = threadIdx.x & 31;
    for (int run = threadIdx.x >> 5; run * TOP_RUN < n; run += blockDim.x >> 5) {
        const int place = 4 * lane, at = run * TOP_RUN + place;
        unsigned long long x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = at + e < n ? list[at + e] : 0ull;
        top_order(x[0], x[1], true);
        top_order(x[2], x[3], false);
#pragma unroll 1
        for (int k = 4; k <= TOP_RUN; k *= 2) {
            const bool down = (place & k) == 0;  // descending runs where bit k of the place is 0
#pragma unroll 1
            for (int j = k / 2; j >= 4; j /= 2) {
                const bool keep_large = down == ((place & j) == 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned long long y = __shfl_xor_sync(0xffffffffu, x[e], j / 4);
                    x[e] = (x[e] > y) == keep_large ? x[e] : y;
                }
            }
            top_order(x[0], x[2], down);
            top_order(x[1], x[3], down);
            top_order(x[0], x[1], down);
            top_order(x[2], x[3], down);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) list[at + e] = x[e];
    }
}

// How many entries of a sorted run are above x.
__device__ __forceinline__ int top_above(const unsigned long long* run, unsigned long long x)
{
    int n = 0;
#pragma unroll
    for (int step = TOP_RUN / 2; step > 0; step /= 2)
        if (run[n + step - 1] > x) n += step;
    return n + (run[n] > x);
}

// For rows where the border leaves too many words (long ties): the border value by four passes that count bytes of the keys, then
// what is above it, then the first words at it.  Returns how many words the list has.
template <typename T>
__device__ __noinline__ int top_by_bytes(const T* row, int V, int top, TopCounts& sh, unsigned long long* list)
{
    const int tid = threadIdx.x, threads = blockDim.x, lane = tid & 31;
    uint32_t prefix = 0;
    int need = top;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = tid; i < 256; i += threads) sh.hist[i] = 0;
        __syncthreads();
        for (int v = tid; v - tid < V; v += threads) {
            const uint32_t k = v < V ? order_key(row_value(row[v])) : 0u, byte = (k >> shift) & 255;
            const bool in = v < V && (shift == 24 || (k >> shift >> 8) == (prefix >> shift >> 8));
            // one addition for all lanes with the first lane's byte
            const uint32_t lanes = __ballot_sync(0xffffffffu, in);
            const int first = lanes ? __ffs((int)lanes) - 1 : 0;
            const uint32_t theirs = __shfl_sync(0xffffffffu, byte, first);
            const bool like = in && byte == theirs;
            const uint32_t alike = __ballot_sync(0xffffffffu, like);
            if (like) {
                if (lane == first) atomicAdd(&sh.hist[byte], __popc(alike));
            } else if (in)
                atomicAdd(&sh.hist[byte], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int d = 255, left = need;
            while (d > 0 && sh.hist[d] < left) left -= sh.hist[d--];
            sh.prefix = prefix | ((uint32_t)d << shift);
            sh.need = left;
        }
        __syncthreads();
        prefix = sh.prefix;
        need = sh.need;
    }
    prefix = max(prefix, KEY_NEG_INF);  // (where fewer than `top` words are not masked)
    if (tid == 0) sh.n = 0;
    __syncthreads();
    for (int v = tid; v < V; v += threads) {
        const uint32_t k = order_key(row_value(row[v]));
        if (k > prefix) list[atomicAdd(&sh.n, 1)] = top_entry(k, v);
    }
    __syncthreads();
    // the words at the border in their order: one warp
    if (tid < 32 && prefix > KEY_NEG_INF) {
        int have = sh.n;
        for (int base = 0; base < V && have < top; base += 32) {
            const int v = base + lane;
            const bool at = v < V && order_key(row_value(row[v])) == prefix;
            const uint32_t all = __ballot_sync(0xffffffffu, at);
            const int place = have + __popc(all & ((1u << lane) - 1));
            if (at && place < top) list[place] = top_entry(prefix, v);
            have += __popc(all);
        }
        if (lane == 0) sh.n = min(have, top);
    }
    __syncthreads();
    return sh.n;
}

// What the pass over a row does with a thread's chunk number `turn`: its values into the sum, the largest of every piece (a lane's groups
// of the chunk; FINE: each group) as the upper half of its key, and of every group of pieces (`tops`: this thread's of the first
// groups; it has turns + 1 of them, `threads` places apart).
template <typename T, bool FINE>
__device__ __forceinline__ void top_chunk(const uint4 (&raw)[TOP_GROUPS], uint16_t* keys, uint16_t* tops, int turn, int turns, int threads,
                                          float c, float& m, ExpSum& sum)
{
    constexpr int PIECES = FINE ? TOP_GROUPS : 1;
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
        float x;
        if constexpr (FINE) {
            const uint4 one[1] = {raw[k]};
            x = groups_max<T, 1>(one);
        } else
            x = groups_max<T, TOP_GROUPS>(raw);
        const uint16_t key = (uint16_t)(order_key(x) >> 16);
        keys[32 * k] = key;
        uint16_t* group = tops + (turn * PIECES + k & turns) * threads;
        *group = max(*group, key);
        top = FINE ? max_nan(top, x) : x;
    }
    m = fmaxf(m, top);
    add_groups<T, TOP_GROUPS>(sum, raw, top, c);
}

// Groups of pieces: a power of two of them per thread, so that a fourth at most will reach the border where that is possible.
__host__ __device__ constexpr int top_groups(int threads, int top)
{
    int n = threads < 256 ? 256 : threads;
    while (n < 4 * top && n < TOP_VALUES) n *= 2;
    return n;
}

// The value of a half-key.
__device__ __forceinline__ float half_key_value(uint32_t k) { return key_value(k << 16); }

// A half-key that at least `want` of the groups reach, and not more than `spare` others if there is one; lo: one that at least `want`
// reach, hi: above all that do.  Every warp tries another one at a time, at equal distances between what is too low and what is too
// high: of the values, which finds it in two rounds in rows of ordinary logits, and every other time of the keys, which takes seven
// rounds at most.  (Halving by one warp, 12 rounds: 7 us of the 54 that a CTA spends on 131 072 words of bf16, eight CTAs at a time.)
__device__ __forceinline__ uint32_t top_border(const uint16_t* tops, int groups, int want, int spare, uint32_t lo, uint32_t hi,
                                               int (*counts)[ROW_THREADS / 32])
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const float share = 1.0f / (float)(warps + 1);
    for (int round = 0; lo + 1 < hi; ++round) {
        const float from = half_key_value(lo), range = half_key_value(hi - 1) - from;
        const bool by_value = (round & 1) == 0 && fabsf(range) < INFINITY && fabsf(from) < INFINITY;
        const auto at = [&](int w) {
            const float part = (float)(w + 1) * share;
            const uint32_t k = by_value ? order_key(from + range * part) >> 16 : lo + (uint32_t)((float)(hi - lo) * part);
            return min(max(k, lo + 1), hi - 1);
        };
        const uint32_t mid = at(warp);
        int n = 0;
#pragma unroll 1
        for (int i = lane; i < groups / 8; i += 32) {
            const uint4 eight = reinterpret_cast<const uint4*>(tops)[i];
            const uint32_t two[4] = {eight.x, eight.y, eight.z, eight.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) n += ((two[e] & 0xFFFFu) >= mid) + ((two[e] >> 16) >= mid);
        }
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane == 0) counts[round & 1][warp] = n;
        __syncthreads();
        // lane w looks at warp w's: the highest that enough reach (with their number), the lowest that too few do
        const uint32_t k = at(lane);
        const int c = lane < warps ? counts[round & 1][lane] : 0;
        const uint32_t reached = __reduce_max_sync(0xffffffffu, lane < warps && c >= want ? k << 11 | (uint32_t)c : 0u);
        hi = __reduce_min_sync(0xffffffffu, lane < warps && c < want ? k : hi);
        if (reached) {
            lo = reached >> 11;
            if ((int)(reached & 2047) <= want + spare) break;
        }
    }
    return lo;
}

// Element e of a group of 16-bit values.
template <typename T>
__device__ __forceinline__ float pair_value(uint4 g, int e)
{
    const uint32_t word = e & 4 ? (e & 2 ? g.w : g.z) : (e & 2 ? g.y : g.x), half = e & 1 ? word >> 16 : word & 0xFFFFu;
    if constexpr (T_is_bf16<T>) return __uint_as_float(half << 16);
    return __half2float(__ushort_as_half((unsigned short)half));
}

// Bits of the elements of a group whose half-keys reach the border.  `least`: the border as a value, rounded up (16-bit types, two
// at a time: not below it, or NaN, which is above everything).
template <typename T>
__device__ __forceinline__ uint32_t top_hits(uint4 g, uint32_t border, T least)
{
    const uint32_t word[4] = {g.x, g.y, g.z, g.w};
    uint32_t hits = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 4)
            hits |= (uint32_t)((order_key(__uint_as_float(word[e])) >> 16) >= border) << e;
        else {
            uint32_t m;
            if constexpr (T_is_bf16<T>)
                m = __hgeu2_mask(*reinterpret_cast<const __nv_bfloat162*>(&word[e]), __nv_bfloat162(least, least));
            else
                m = __hgeu2_mask(*reinterpret_cast<const __half2*>(&word[e]), __half2(least, least));
            hits |= ((m & 1) | (m >> 30 & 2)) << 2 * e;
        }
    }
    return hits;
}
template <typename T>
__device__ __forceinline__ T top_least(uint32_t border)
{
    const float x = half_key_value(border);
    if constexpr (sizeof(T) == 4) return x;
    else if constexpr (T_is_bf16<T>) return __float2bfloat16_ru(x);
    else return __float2half_ru(x);
}

// The words that reach the border, into `list` (n counts them, beyond its room too): the pieces that do are read again, a group of
// one to every thread.
template <typename T, bool FINE>
__device__ __forceinline__ void top_collect(const T* row, const RowSplit& split, int V, const uint16_t* keys,
                                            int pieces, uint32_t border, int room, int* queue, int* queued, unsigned long long* list, int* n)
{
    constexpr int R = TOP_GROUPS, PIECES = FINE ? R : 1, SIZE = R / PIECES;  // pieces of a lane's groups, groups of a piece
    const int tid = threadIdx.x, threads = blockDim.x, lane = tid & 31;
    for (int base = 0; base < pieces; base += 32 * threads) {
        // 32 pieces of each thread: eight at a time in four places
        uint32_t hits = 0;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const int i = base + 8 * (h * threads + tid);
            if (i >= pieces) break;
            const uint4 eight = *reinterpret_cast<const uint4*>(keys + i);
            const uint32_t two[4] = {eight.x, eight.y, eight.z, eight.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                hits |= (uint32_t)((two[e] & 0xFFFFu) >= border) << (8 * h + 2 * e);
                hits |= (uint32_t)((two[e] >> 16) >= border) << (8 * h + 2 * e + 1);
            }
        }
        if (!__any_sync(0xffffffffu, hits)) continue;
        const int upto = warp_scan_incl(__popc(hits));
        int at = 0;
        if (lane == 31) at = atomicAdd(queued, upto);
        at = __shfl_sync(0xffffffffu, at, 31) + upto - __popc(hits);
        for (; hits; hits &= hits - 1, ++at) {
            const int bit = __ffs((int)hits) - 1;
            if (at < room) queue[at] = base + 8 * (bit / 8 * threads + tid) + bit % 8;
        }
    }
    __syncthreads();
    const T least = top_least<T>(border);
    const int tasks = *queued * SIZE;
    if (*queued > room) {
        if (tid == 0) atomicAdd(n, room + 1);
        return;
    }
    constexpr int AHEAD = 4;  // groups of a thread that are on their way together
    for (int base = 0; base < tasks; base += AHEAD * threads) {
        uint4 raw[AHEAD];
        int first[AHEAD];
#pragma unroll
        for (int h = 0; h < AHEAD; ++h) {
            const int t = base + h * threads + tid;
            const int i = t < tasks ? queue[t / SIZE] : 0;  // piece i: chunk i / (32 PIECES), its groups 32 k + (i mod 32)
            const int group = FINE ? i % (32 * PIECES) : 32 * (t % SIZE) + i % 32;
            first[h] = t < tasks ? chunk_first<T, R>(split.chunk0 + i / (32 * PIECES), split.pre) + group * PER<T> : V;
            raw[h] = t < tasks ? any_group(row, first[h], V, row_element<T>(-INFINITY)) : uint4{};
        }
#pragma unroll
        for (int h = 0; h < AHEAD; ++h) {
            if (base + h * threads >= tasks) break;
            uint32_t hits = first[h] < V ? top_hits<T>(raw[h], border, least) : 0u;
            if (!__any_sync(0xffffffffu, hits)) continue;
            // (one addition for the warp)
            const int upto = warp_scan_incl(__popc(hits));
            int at = 0;
            if (lane == 31) at = atomicAdd(n, upto);
            at = __shfl_sync(0xffffffffu, at, 31) + upto - __popc(hits);
            if constexpr (sizeof(T) == 4) {
                float x[4];
                unpack<T>(raw[h], x);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (hits >> e & 1) {
                        if (at < room) list[at] = top_entry(order_key(x[e]), first[h] + e);
                        ++at;
                    }
            } else
                for (; hits; hits &= hits - 1, ++at) {
                    const int e = __ffs((int)hits) - 1;
                    if (at < room) list[at] = top_entry(order_key(pair_value<T>(raw[h], e)), first[h] + e);
                }
        }
    }
}

// The row's outputs from its n candidates (room + 1 or more: they did not fit).
template <typename T>
__device__ __forceinline__ void top_finish(const TopArgs& a, int64_t r, const T* row, int room, int n,
                                           unsigned long long* list, TopCounts& sh, ExpSum sum, float m, bool far)
{
    if (n > room) n = top_by_bytes<T>(row, a.V, a.top, sh, list);
    top_sort_runs(list, n);
    __syncthreads();
    // an entry's place: its place in its run, and how many are above it in the others
    const int tid = threadIdx.x, threads = blockDim.x, want = min(n, a.top);
    for (int i = tid; i < n; i += threads) {
        const unsigned long long x = list[i];
        int place = i % TOP_RUN;
        for (int at = 0; at < n; at += TOP_RUN)
            if (at / TOP_RUN != i / TOP_RUN) place += top_above(list + at, x);
        if (place >= want) continue;
        const int v = (int)(0xFFFFFFFFu - (uint32_t)x);
        a.ids[r * a.top + place] = v;
        ((T*)a.values)[r * a.top + place] = row[v];
        if (place == 0) sh.prefix = (uint32_t)(x >> 32);
    }
    for (int i = want + tid; i < a.top; i += threads) {
        a.ids[r * a.top + i] = -1;
        ((T*)a.values)[r * a.top + i] = row_element<T>(-INFINITY);
    }
    if (!a.lse) return;
    __syncthreads();
    if (tid == 0) {
        const uint32_t first = sh.prefix;
        // (log2 of the largest exponential: x c - R, or 0 when far)
        const double largest = far ? 0.0 : (double)m * (double)a.scale - (double)sum.ref;
        a.lse[r] = want == 0 ? -INFINITY
                   : first == KEY_NAN ? NAN
                   : m == INFINITY ? INFINITY
                                   : (float)((double)m * a.inv_tau + ((double)log2f(sum.sum) - largest) * LN2);
    }
}

// Sum of 2^((x - m) c) over a warp's chunks.
template <typename T>
__device__ __noinline__ float top_far_sum(const T* row, const RowSplit& split, int V, float m, float c, int warp, int warps)
{
    constexpr int R = TOP_GROUPS;
    float o = 0.0f;
    for (int chunk = split.chunk0 + warp; chunk < split.chunk1; chunk += warps) {
        uint4 raw[R];
        load_chunk<T, R>(row, chunk_first<T, R>(chunk, split.pre), V, row_element<T>(-INFINITY), raw);
        for (int k = 0; k < R; ++k) {
            float y[PER<T>];
            unpack<T>(raw[k], y);
            for (int i = 0; i < PER<T>; ++i) o += exp2_unit((y[i] - m) * c);
        }
    }
    return warp_reduce_sum(o);
}

// What a CTA knows of its part of the row.
struct TopPart {
    ExpSum sum;
    float max;
    uint32_t share, alone;  // borders
};

// One cluster per row.  The pass leaves the pieces' largest keys.  A border that at least `top` groups of pieces reach
// leaves at least `top` words, and few more (95 for 64 of 131 072); the pieces that reach it are read again (from L2), their words
// sorted, in runs of 128 by a warp each, and merged by rank.
// 4096 rows of 131 072 words of bf16, lists of 64: 214 us, 5.0 TB/s, in a replayed graph of ten calls, as all times here (calls one by
// one on a warm card: 229); no unit is full (of what they can, the multifunction units do
// 59 %, the issue slots 59 %, DRAM 75 %): a row's CTA spends 35 of 53 us on the pass and the rest on its list, eight CTAs at a time.
// 777 rows of 100 003 of fp16, lists of 301: 64 us, 25 of them the pass, 13 the second read of 430 pieces (17 with the border
// compared to a key per element).
// Tried: the lists put together by warps of their own beside the next row's pass (558 us with one such warp, 237 with four: the list
// is more work than they have time for), 256 threads a row (222 us), groups as pieces (259 us; for lists of 301 85 us).
template <typename T, bool FINE>
__global__ void __launch_bounds__(ROW_THREADS, 2) k_top(TopArgs a)
{
    constexpr int R = TOP_GROUPS, PIECES = FINE ? R : 1;
    extern __shared__ __align__(16) uint8_t dynamic[];  // the walk's ring and, later, the lists; the groups' and the pieces' largest keys
    __shared__ TopPart parts[2][ROW_CTAS];
    __shared__ ExpSum ered[ROW_THREADS / 32];
    __shared__ float fred[ROW_THREADS / 32];
    __shared__ int counts[2][ROW_THREADS / 32], valids[ROW_THREADS / 32];
    __shared__ TopCounts sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads / 32, V = a.V;
    const int room = top_room(a.top);
    const TopLists lists(dynamic, room);
    uint16_t* tops = (uint16_t*)(dynamic + a.ring);
    const int groups = top_groups(threads, a.top), turns = groups / threads - 1;
    uint16_t* keys = tops + groups;
    const int64_t r = blockIdx.x / ctas;
    const T* row = (const T*)a.logits + r * a.stride;
    const RowSplit split = RowSplit::of<T, R>(row, V, rank, ctas);
    const int pieces = (split.chunk1 - split.chunk0) * 32 * PIECES;
    ChunkWalk<T, R, TOP_DEPTH> walk;
    walk.start(dynamic, threads, row, split, V);
    if (ctas > 1) cluster_arrive();
    if (tid == 0) sh.n = sh.queued = 0;
    for (int g = tid; g < groups; g += threads) tops[g] = 0;  // (a thread's own)
    int turn = 0;
    ExpSum sum = ExpSum::none();
    float m = -INFINITY;
    walk.each(row, split, V, row_element<T>(-INFINITY), [&](int c, int, uint4(&raw)[R]) {
        top_chunk<T, FINE>(raw, keys + (c - split.chunk0) * 32 * PIECES + lane, tops + tid, turn++, turns, threads, a.scale, m, sum);
    });
    sum.warp_reduce();
    m = warp_reduce_max(m);
    // the groups that are not masked whole: their number, their least and largest key
    uint32_t most = 0, least = 0xFFFFu;
    int valid = 0;
    for (int g = tid; g < groups; g += threads) {  // (its own)
        const uint32_t k = tops[g];
        most = max(most, k);
        if (k >= TOP_LOWEST) least = min(least, k), ++valid;
    }
    most = __reduce_max_sync(0xffffffffu, most);
    least = __reduce_min_sync(0xffffffffu, least);
    valid = __reduce_add_sync(0xffffffffu, valid);
    if (lane == 0) ered[warp] = sum, fred[warp] = m, counts[1][warp] = (int)(most << 16 | least), valids[warp] = valid;
    __syncthreads();
    most = __reduce_max_sync(0xffffffffu, lane < warps ? (uint32_t)counts[1][lane] >> 16 : 0u);
    least = __reduce_min_sync(0xffffffffu, lane < warps ? (uint32_t)counts[1][lane] & 0xFFFFu : 0xFFFFu);
    valid = __reduce_add_sync(0xffffffffu, lane < warps ? valids[lane] : 0);
    // `top` groups of one part are enough, and so are its share of them in every part; what is not masked where there are not that many
    uint32_t alone = 0, share = 0;
#pragma unroll 1
    for (int i = 0; i < (ctas > 1 ? 2 : 1); ++i) {
        const int want = i ? a.top : (a.top + ctas - 1) / ctas, spare = want / 4 + 16 / ctas;
        if (valid < want) alone = TOP_LOWEST;
        else if (valid <= want + spare) alone = least;
        else alone = top_border(tops, groups, want, spare, least, (i ? max(share, least) : most) + 1, counts);
        if (i == 0) share = alone;
        __syncthreads();
    }
    if (warp == 0) {
        sum = lane < warps ? ered[lane] : ExpSum::none();
        sum.warp_reduce();
        m = warp_reduce_max(lane < warps ? fred[lane] : -INFINITY);
    }
    if (ctas > 1) cluster_wait();
    if (tid < ctas) *row_peer(cluster, &parts[0][rank], tid, ctas) = TopPart{sum, m, share, alone};
    row_sync(cluster, ctas);
    uint32_t border = 0, lowest = 0xFFFFFFFFu;
    m = -INFINITY;
    for (int k = 0; k < ctas; ++k) {
        border = max(border, parts[0][k].alone);
        lowest = min(lowest, parts[0][k].share);
        m = fmaxf(m, parts[0][k].max);
    }
    border = max(border, lowest);
    const bool far = exp_far(m, a.scale);
    if (far) {  // (the same in every CTA of the cluster)
        float o = top_far_sum<T>(row, split, V, m, a.scale, warp, warps);
        if (lane == 0) fred[warp] = o;
        __syncthreads();
        if (warp == 0) o = warp_reduce_sum(lane < warps ? fred[lane] : 0.0f);
        if (tid < ctas) *row_peer(cluster, &parts[1][rank], tid, ctas) = TopPart{{0.0f, o}, m, 0, 0};
        row_sync(cluster, ctas);
    }
    top_collect<T, FINE>(row, split, V, keys, pieces, border, room, lists.queue, &sh.queued,
                         row_peer(cluster, lists.list, 0, ctas), row_peer(cluster, &sh.n, 0, ctas));
    row_sync(cluster, ctas);
    if (rank != 0) return;
    sum = parts[far][0].sum;
    for (int k = 1; k < ctas; ++k) sum.add(parts[far][k].sum);
    top_finish<T>(a, r, row, room, sh.n, lists.list, sh, sum, m, far);
}

template <typename T>
static cudaError_t run_top(TopArgs a, int64_t rows, cudaStream_t st)
{
    constexpr int CHUNK = 32 * TOP_GROUPS * PER<T>;
    const int64_t row_bytes = (int64_t)a.V * sizeof(T);
    const int per = a.V / PER<T>, room = top_room(a.top);
    const int chunks = (a.V + PER<T> - 1 + CHUNK - 1) / CHUNK;
    const auto pieces = [&](int ctas, bool fine) { return (chunks + ctas - 1) / ctas * 32 * (fine ? TOP_GROUPS : 1); };
    // 128 bytes a thread at least: one row of 131 072 words of bf16 11.2 us for the 12.6 of 64 bytes, 16 rows 13.4 for 16.2.  Short
    // rows that do not fill the GPU have 256 threads all the same, for the sorting (64 rows of 8 000 words of fp32, the 256 largest:
    // 11.3 us for 14.4 with 128 threads; of 4 000 words: 10.8 for 13.3)
    RowShape shape = row_shape(rows, row_bytes, 1024, 128);
    if (shape.threads == 128 && row_bytes >= 16000 && rows <= 148 * 4) shape.threads = 256;
    const bool fine = per / TOP_GROUPS / shape.ctas < 4 * a.top;
    a.ring = std::max(ChunkWalk<T, TOP_GROUPS, TOP_DEPTH>::bytes(shape, a.V), TopLists::bytes(room));
    const size_t smem = a.ring + 2 * (size_t)(top_groups(shape.threads, a.top) + pieces(shape.ctas, fine));
    return fine ? launch_rows<k_top<T, true>>(a, rows, shape, smem, sizeof(TopCounts) + 1024, st)
                : launch_rows<k_top<T, false>>(a, rows, shape, smem, sizeof(TopCounts) + 1024, st);
}

}  // namespace lda

extern "C" int lda_top_logits(const void* logits_dev, int dtype, int64_t rows, int32_t V, int64_t row_stride, int32_t top,
                              double temperature, int32_t* ids_dev, void* values_dev, float* lse_dev, void* cuda_stream)
{
    using namespace lda;
    int rc = check_rows(logits_dev, dtype, rows, V, row_stride);
    if (rc != LDA_OK) return rc;
    if (top < 1 || !temperature_ok(temperature)) return LDA_EINVAL;
    if (top > LDA_TOP_MAX) return LDA_ERANGE;
    if (rows == 0) return LDA_OK;
    if (!ids_dev || !values_dev) return LDA_EINVAL;
    if (!aligned(ids_dev, 4) || !aligned(values_dev, dtype == LDA_F32 ? 4 : 2) || !aligned(lse_dev, 4)) return LDA_EINVAL;
    TopArgs a{logits_dev, row_stride, V, top, (float)(1.4426950408889634 / temperature), 1.0 / temperature, ids_dev, values_dev,
              lse_dev, 0};
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const cudaError_t e = dtype == LDA_F32 ? run_top<float>(a, rows, st)
                          : dtype == LDA_F16 ? run_top<__half>(a, rows, st)
                                             : run_top<__nv_bfloat16>(a, rows, st);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return LDA_ECUDA;
    }
    return LDA_OK;
}
