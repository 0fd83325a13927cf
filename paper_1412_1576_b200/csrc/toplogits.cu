// The largest logits of every row, with their words, and the row's log-sum-exp.
//
// A row's words are ordered by value (NaN first), equal values by the lower word; what is minus infinity is not listed.
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
};

#ifndef TG
#define TG 4
#endif
#ifndef TB
#define TB 2
#endif
constexpr int TOP_GROUPS = TG;     // groups a lane has in flight
constexpr int TOP_LIST = 2048;      // words that may be left for the longest lists
constexpr int TOP_VALUES = 1024;  // groups of pieces whose largest keys give the border, at most
// Words and pieces that may be left for lists of `top`: about four times what is expected.
__host__ __device__ constexpr int top_room(int top) { return top <= 64 ? 512 : top <= 256 ? 1024 : TOP_LIST; }
constexpr uint32_t TOP_LOWEST = (KEY_NEG_INF >> 16) + 1;  // first half-key above minus infinity

#ifndef TD
#define TD 2
#endif
constexpr int TOP_DEPTH = TD;      // chunks on their way

// What a CTA knows of its part of the row.
struct TopPart {
    ExpSum sum;
    float max;
    uint32_t share, alone;  // borders (half-keys)
};

// Behind the pass over the row its shared memory holds these.
struct TopLists {
    unsigned long long* list;  // the words that are left
    uint16_t* tops;            // (before that, in the same place) the groups' largest keys
    int* queue;                // the pieces that are read again
};

struct TopShared {
    TopPart parts[2][ROW_CTAS];
    ExpSum ered[ROW_THREADS / 32];
    float fred[ROW_THREADS / 32];
    int ired[33];
    int hist[256];
    int n, queued, need;
    uint32_t prefix;
    float max;
};

__host__ __device__ constexpr int top_ring_bytes(int threads, int room)
{
    const int ring = threads * TOP_DEPTH * TOP_GROUPS * 16, lists = room * 12;
    return ring > lists ? ring : lists;
}

__device__ __forceinline__ unsigned long long top_entry(uint32_t key, int v)
{
    return ((unsigned long long)key << 32) | (0xFFFFFFFFu - (uint32_t)v);
}

// Descending sort of list[0..n) by the CTA; list[n..) up to the next power of two is overwritten.
__device__ __forceinline__ void sort_entries(unsigned long long* list, int n)
{
    const int tid = threadIdx.x, threads = blockDim.x;
    int size = 32;
    while (size < n) size *= 2;
    if (size <= threads) {
        // an entry per thread: partners up to 16 places away by shuffles, further ones through shared memory
        unsigned long long x = tid < n ? list[tid] : 0ull;
        for (int k = 2; k <= size; k *= 2)
            for (int j = k / 2; j > 0; j /= 2) {
                unsigned long long y;
                if (j >= 32) {
                    __syncthreads();
                    if (tid < size) list[tid] = x;
                    __syncthreads();
                    y = tid < size ? list[tid ^ j] : 0ull;
                } else {
                    if (tid >= size) continue;  // (whole warps)
                    y = __shfl_xor_sync(0xffffffffu, x, j);
                }
                // descending runs where bit k of the place is 0
                const bool keep_large = ((tid & k) == 0) == ((tid & j) == 0);
                x = (x > y) == keep_large ? x : y;
            }
        __syncthreads();
        if (tid < size) list[tid] = x;
        __syncthreads();
        return;
    }
    for (int i = n + tid; i < size; i += threads) list[i] = 0;
    __syncthreads();
    for (int k = 2; k <= size; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            for (int i = tid; i < size / 2; i += threads) {
                const int lo = 2 * i - (i & (j - 1)), hi = lo + j;
                const unsigned long long x = list[lo], y = list[hi];
                if ((x < y) == ((lo & k) == 0)) list[lo] = y, list[hi] = x;
            }
            __syncthreads();
        }
}

// For rows where the border leaves too many words (long ties): the border value by four passes that count bytes of the keys, then
// what is above it, then the first words at it.  One CTA, the whole row; returns how many words the list has.
template <typename T>
__device__ __noinline__ int top_by_bytes(const T* row, int V, int top, TopShared& sh, unsigned long long* list)
{
    const int tid = threadIdx.x, threads = blockDim.x;
    uint32_t prefix = 0;
    int need = top;
    for (int shift = 24; shift >= 0; shift -= 8) {
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
                if ((tid & 31) == first) atomicAdd(&sh.hist[byte], __popc(alike));
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
        __syncthreads();
    }
    if (prefix <= KEY_NEG_INF) prefix = KEY_NEG_INF;  // (fewer than `top` words are not masked)
    if (tid == 0) sh.n = 0;
    __syncthreads();
    for (int v = tid; v < V; v += threads) {
        const uint32_t k = order_key(row_value(row[v]));
        if (k > prefix) list[atomicAdd(&sh.n, 1)] = top_entry(k, v);
    }
    __syncthreads();
    int have = sh.n;
    __syncthreads();
    for (int base = 0; base < V && have < top && prefix > KEY_NEG_INF; base += threads) {
        const int v = base + tid;
        const int at = v < V && order_key(row_value(row[v])) == prefix;
        int total;
        const int before = block_scan_excl(at, sh.ired, total);
        if (at && have + before < top) list[have + before] = top_entry(prefix, v);
        have += total;
        __syncthreads();
    }
    return min(have, top);
}

// One cluster per row.  The pass that adds up the exponentials leaves the largest value of every piece (a lane's groups of a chunk;
// FINE: each group) as the upper half of its key.  A border that at least `top` of them reach leaves at least `top` words, and few
// more: the pieces that reach it are read again (from L2), their words at or above it are sorted.
template <typename T, bool FINE>
__global__ void __launch_bounds__(ROW_THREADS, TB) k_top(TopArgs a)
{
    constexpr int R = TOP_GROUPS, PIECES = FINE ? R : 1, SIZE = R / PIECES;  // pieces of a lane's groups, groups of a piece
    extern __shared__ __align__(16) uint8_t dynamic[];  // the walk's ring and, later, the lists; the pieces' keys
    const int room = top_room(a.top);
    const TopLists lists{(unsigned long long*)dynamic, (uint16_t*)dynamic, (int*)(dynamic + 8 * room)};
    uint16_t* keys = (uint16_t*)(dynamic + top_ring_bytes(blockDim.x, room));
    __shared__ TopShared sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, WARPS = threads / 32, V = a.V;
    const int64_t r = blockIdx.x / ctas;
    const T* row = (const T*)a.logits + r * a.stride;
    const RowSplit split = RowSplit::of<T, R>(row, V, rank, ctas);
    const int pieces = (split.chunk1 - split.chunk0) * 32 * PIECES;
    ChunkWalk<T, R, TOP_DEPTH> walk;
    walk.start(dynamic, row, split, V);
    if (ctas > 1) cluster_arrive();
    if (tid == 0) sh.n = sh.queued = 0;
    ExpSum sum = ExpSum::none();
    float m = -INFINITY;
    walk.each(row, split, V, row_element<T>(-INFINITY), [&](int c, uint4(&raw)[R]) {
        const int at = (c - split.chunk0) * 32 * PIECES + lane;
        float top;
        if (FINE) {
            top = -INFINITY;
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const uint4 one[1] = {raw[k]};
                const float x = groups_max<T, 1>(one);
                keys[at + 32 * k] = (uint16_t)(order_key(x) >> 16);
                top = max_nan(top, x);
            }
        } else {
            top = groups_max<T, R>(raw);
            keys[at] = (uint16_t)(order_key(top) >> 16);
        }
        m = fmaxf(m, top);
        add_groups<T, R>(sum, raw, top, a.scale);
    });
    sum.warp_reduce();
    m = warp_reduce_max(m);
    if (lane == 0) sh.ered[warp] = sum, sh.fred[warp] = m;
    __syncthreads();
    // the pieces' keys in `values` groups, the largest of each; every fourth at most will reach the border
    int values = 256;
    while (values < 4 * a.top && values < TOP_VALUES) values *= 2;
    for (int g = tid; g < values; g += threads) {
        uint32_t top = 0;
        for (int i = g; i < pieces; i += values) top = max(top, (uint32_t)keys[i]);
        lists.tops[g] = (uint16_t)top;
    }
    __syncthreads();
    uint32_t share = 0, alone = 0;
    if (warp == 0) {
        sum = lane < WARPS ? sh.ered[lane] : ExpSum::none();
        sum.warp_reduce();
        m = warp_reduce_max(lane < WARPS ? sh.fred[lane] : -INFINITY);
        const int per = values / 32;
        uint32_t tops[TOP_VALUES / 32], best = 0;
#pragma unroll
        for (int k = 0; k < TOP_VALUES / 32; ++k) {
            tops[k] = k < per ? lists.tops[k * 32 + lane] : 0u;
            best = max(best, tops[k]);
        }
        best = __reduce_max_sync(0xffffffffu, best);
        // The largest half-key that at least `want` of the groups reach, or one that not many more do: steps of doubling width down
        // from `hi` (that fewer reach), then halving; minus infinity's successor if there are not that many.
        auto border_of = [&](int want, uint32_t hi) {
            uint32_t lo = TOP_LOWEST, step = 64;
            while (lo + 1 < hi) {
                const bool down = lo == TOP_LOWEST && hi > lo + step;
                const uint32_t mid = down ? hi - step : (lo + hi) / 2;
                step = down ? step * 2 : step;
                int n = 0;
#pragma unroll
                for (int k = 0; k < TOP_VALUES / 32; k += 8)
                    if (k < per)
#pragma unroll
                        for (int e = 0; e < 8; ++e) n += tops[k + e] >= mid;
                n = __reduce_add_sync(0xffffffffu, n);
                if (n >= want) {
                    lo = mid;
                    if (n <= want + want / 4 + 16 / ctas) break;
                } else
                    hi = mid;
            }
            return lo;
        };
        // `top` groups of one part are enough, and so are its share of them in every part
        share = border_of((a.top + ctas - 1) / ctas, best + 1);
        alone = ctas > 1 ? border_of(a.top, share + 1) : share;
    }
    if (ctas > 1) cluster_wait();
    if (tid < ctas) *cluster.map_shared_rank(&sh.parts[0][rank], tid) = TopPart{sum, m, share, alone};
    row_sync(cluster, ctas);
    uint32_t border = 0, least = 0xFFFFFFFFu;
    m = -INFINITY;
    for (int k = 0; k < ctas; ++k) {
        border = max(border, sh.parts[0][k].alone);
        least = min(least, sh.parts[0][k].share);
        m = fmaxf(m, sh.parts[0][k].max);
    }
    border = max(border, least);
    const bool far = exp_far(m, a.scale);
    if (far) {  // (the same in every CTA of the cluster)
        float o = 0.0f;
        for (int c = split.chunk0 + warp; c < split.chunk1; c += WARPS) {
            uint4 raw[R];
            load_chunk<T, R>(row, chunk_first<T, R>(c, split.pre), V, row_element<T>(-INFINITY), raw);
            for (int k = 0; k < R; ++k) {
                float y[PER<T>];
                unpack<T>(raw[k], y);
                for (int i = 0; i < PER<T>; ++i) o += exp2_unit((y[i] - m) * a.scale);
            }
        }
        o = warp_reduce_sum(o);
        if (lane == 0) sh.fred[warp] = o;
        __syncthreads();
        if (warp == 0) o = warp_reduce_sum(lane < WARPS ? sh.fred[lane] : 0.0f);
        if (tid < ctas) *cluster.map_shared_rank(&sh.parts[1][rank], tid) = TopPart{{0.0f, o}, m, 0, 0};
        row_sync(cluster, ctas);
    }
    // the pieces that reach the border, then a group of one to every thread
    int* n_all = cluster.map_shared_rank(&sh.n, 0);
    unsigned long long* list = cluster.map_shared_rank(lists.list, 0);
    for (int i = 8 * tid; i < pieces; i += 8 * threads) {
        const uint4 eight = *reinterpret_cast<const uint4*>(keys + i);
        const uint32_t two[4] = {eight.x, eight.y, eight.z, eight.w};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (((two[e / 2] >> (e % 2 * 16)) & 0xFFFFu) >= border) {
                const int at = atomicAdd(&sh.queued, 1);
                if (at < room) lists.queue[at] = i + e;
            }
    }
    __syncthreads();
    const int queued = sh.queued;
    if (queued > room) {
        if (tid == 0) atomicAdd(n_all, room + 1);
    } else
        for (int base = 0; base < queued * SIZE; base += 2 * threads) {
            // (two groups at a time: the second is on its way while the first is looked at)
            uint4 raw[2];
            int first[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int t = base + h * threads + tid;
                const bool any = t < queued * SIZE;
                const int i = any ? lists.queue[t / SIZE] : 0;  // piece i: chunk i / (32 PIECES), its groups 32 k + (i mod 32)
                const int chunk = split.chunk0 + i / (32 * PIECES);
                const int group = FINE ? i % (32 * PIECES) : 32 * (t % SIZE) + i % 32;
                first[h] = any ? chunk_first<T, R>(chunk, split.pre) + group * PER<T> : V;
                raw[h] = any_group(row, first[h], V, row_element<T>(-INFINITY));
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float x[PER<T>];
                unpack<T>(raw[h], x);
#pragma unroll
                for (int e = 0; e < PER<T>; ++e) {
                    const uint32_t k = order_key(x[e]);
                    const bool hit = (k >> 16) >= border;
                    const uint32_t hits = __ballot_sync(0xffffffffu, hit);
                    if (hits == 0) continue;
                    int at = 0;
                    if (lane == 0) at = ctas == 1 ? atomicAdd(&sh.n, __popc(hits)) : atomicAdd(n_all, __popc(hits));
                    at = __shfl_sync(0xffffffffu, at, 0) + __popc(hits & ((1u << lane) - 1));
                    if (hit && at < room) list[at] = top_entry(k, first[h] + e);
                }
            }
        }
    row_sync(cluster, ctas);
    if (rank != 0) return;
    int n = sh.n;
    if (n > room) {
        __syncthreads();
        n = top_by_bytes<T>(row, V, a.top, sh, lists.list);
        __syncthreads();
    }
    sort_entries(lists.list, n);
    const int want = min(n, a.top);
    for (int i = tid; i < a.top; i += threads) {
        const int64_t at = r * a.top + i;
        const int v = i < want ? (int)(0xFFFFFFFFu - (uint32_t)lists.list[i]) : -1;
        a.ids[at] = v;
        ((T*)a.values)[at] = v >= 0 ? row[v] : row_element<T>(-INFINITY);
    }
    if (a.lse && tid == 0) {
        sum = sh.parts[far][0].sum;
        for (int k = 1; k < ctas; ++k) sum.add(sh.parts[far][k].sum);
        const uint32_t first = want > 0 ? (uint32_t)(lists.list[0] >> 32) : 0;
        // (log2 of the largest exponential: x c, or 0 when far)
        const double most2 = far ? 0.0 : (double)m * (double)a.scale - (double)sum.ref;
        a.lse[r] = want == 0 ? -INFINITY
                   : first == KEY_NAN ? NAN
                   : m == INFINITY ? INFINITY
                                   : (float)((double)m * a.inv_tau + ((double)log2f(sum.sum) - most2) * LN2);
    }
}

template <typename T>
static cudaError_t run_top(const TopArgs& a, int64_t rows, cudaStream_t st)
{
    constexpr int CHUNK = 32 * TOP_GROUPS * PER<T>;
    RowShape shape = row_shape(rows, (int64_t)a.V * sizeof(T), 1024, 64);
    const int per = a.V / PER<T>;
    const bool fine = per / TOP_GROUPS / shape.ctas < 4 * a.top;
    const int chunks = (a.V + PER<T> - 1 + CHUNK - 1) / CHUNK;
    const size_t smem = top_ring_bytes(shape.threads, top_room(a.top)) + (size_t)((chunks + shape.ctas - 1) / shape.ctas) * 32 * (fine ? TOP_GROUPS : 1) * 2;
    return launch_rows(fine ? k_top<T, true> : k_top<T, false>, a, rows, shape, smem, sizeof(TopShared), st);
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
    TopArgs a{logits_dev, row_stride, V, top, (float)(1.4426950408889634 / temperature), 1.0 / temperature, ids_dev, values_dev,
              lse_dev};
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
