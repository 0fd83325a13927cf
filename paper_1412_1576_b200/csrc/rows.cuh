// Shared pieces of the operators on rows of logits or probabilities (toplogits.cu, distill.cu, verify.cu, logprobs.cu): element types,
// 2^x, keys that order values, a row split over CTAs and walked over, sums of exponentials, launches.
#pragma once
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

#include "../../include/lda_b200.h"

namespace lda {

namespace cg = cooperative_groups;

// The two halves of a cluster's barrier: shared memory of the others may be written once `wait` has returned (they all run then).
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

constexpr double LN2 = 0.69314718055994531;

__device__ __forceinline__ float row_value(float x) { return x; }
__device__ __forceinline__ float row_value(__half x) { return __half2float(x); }
__device__ __forceinline__ float row_value(__nv_bfloat16 x) { return __bfloat162float(x); }
// Element i of an array whose type (LDA_F32, ...) is an argument.
__device__ __forceinline__ float any_value(const void* p, int dtype, int64_t i)
{
    if (dtype == LDA_F32) return ((const float*)p)[i];
    return dtype == LDA_F16 ? row_value(((const __half*)p)[i]) : row_value(((const __nv_bfloat16*)p)[i]);
}
template <typename T>
constexpr bool T_is_bf16 = false;
template <>
constexpr bool T_is_bf16<__nv_bfloat16> = true;
template <typename T>
__device__ __forceinline__ T row_element(float x);
template <>
__device__ __forceinline__ float row_element<float>(float x) { return x; }
template <>
__device__ __forceinline__ __half row_element<__half>(float x) { return __float2half_rn(x); }
template <>
__device__ __forceinline__ __nv_bfloat16 row_element<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// 2^x by the multifunction unit (at most 2^-22 off, relative; results below 2^-126 are zero).
__device__ __forceinline__ float exp2_unit(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Whole numbers in the order of the values: NaN of either sign above +infinity, both zeros alike.
constexpr uint32_t KEY_NAN = 0xFFFFFFFFu, KEY_NEG_INF = 0x007FFFFFu;
__device__ __forceinline__ uint32_t order_key(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return x != x ? KEY_NAN : b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t key) { return __uint_as_float(key >> 31 ? key ^ 0x80000000u : ~key); }

__device__ __forceinline__ float warp_reduce_max(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// --- a row in 16-byte groups, split over the CTAs of a cluster -------------------------------------------------------------------
// Rows start at any element, groups at addresses that are multiples of 16: group g of a row holds its elements
// g PER - pre .. g PER - pre + PER - 1, where `pre` elements of the first group lie before the row (not read, like those behind its
// end).  A warp takes 32 R consecutive groups at a time (a chunk; lane l the groups l, 32 + l, ...), and the CTAs of a cluster take
// runs of consecutive chunks.
template <typename T>
constexpr int PER = 16 / (int)sizeof(T);

struct RowSplit {
    int pre, chunk0, chunk1;  // this CTA's chunks
    template <typename T, int R>
    static __device__ __forceinline__ RowSplit of(const T* row, int V, int rank, int ctas)
    {
        RowSplit s;
        s.pre = (int)((uintptr_t)row % 16 / sizeof(T));
        const int chunks = (int)(((unsigned)(s.pre + V) + 32 * R * PER<T> - 1) / (32 * R * PER<T>));
        const int shift = __ffs(ctas) - 1;  // (a power of two)
        s.chunk0 = chunks * rank >> shift;
        s.chunk1 = chunks * (rank + 1) >> shift;
        return s;
    }
};

// A chunk's first element, and whether all of it lies inside the row.
template <typename T, int R>
__device__ __forceinline__ int chunk_first(int chunk, int pre) { return chunk * (32 * R * PER<T>) - pre; }
template <typename T, int R>
__device__ __forceinline__ bool chunk_inside(int first, int V) { return first >= 0 && first + 32 * R * PER<T> <= V; }

// A group at the row's edge: element by element, `fill` outside the row.
template <typename T>
__device__ __forceinline__ uint4 edge_group(const T* row, int first, int V, T fill)
{
    union {
        uint4 raw;
        T e[PER<T>];
    } g;
#pragma unroll
    for (int i = 0; i < PER<T>; ++i) g.e[i] = first + i >= 0 && first + i < V ? row[first + i] : fill;
    return g.raw;
}

template <typename T>
__device__ __forceinline__ bool group_inside(int first, int V) { return first >= 0 && first + PER<T> <= V; }
template <typename T>
__device__ __forceinline__ uint4 any_group(const T* row, int first, int V, T fill)
{
    return group_inside<T>(first, V) ? __ldcg(reinterpret_cast<const uint4*>(row + first)) : edge_group(row, first, V, fill);
}

// The lane's groups of a chunk.  (Loads that pass L1 by: what is read twice is read from L2 the second time.)
template <typename T, int R>
__device__ __forceinline__ void load_chunk(const T* row, int first, int V, T fill, uint4 (&raw)[R])
{
    const int lane = threadIdx.x & 31;
    if (chunk_inside<T, R>(first, V)) {
        const uint4* p = reinterpret_cast<const uint4*>(row + first) + lane;
#pragma unroll
        for (int r = 0; r < R; ++r) raw[r] = __ldcg(p + 32 * r);
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r) raw[r] = any_group(row, first + (32 * r + lane) * PER<T>, V, fill);
    }
}

// How the rows share the GPU's threads: a row has a CTA, or a cluster of 2, 4 or 8 of them, so that all rows together come to not
// quite `per_sm` threads per multiprocessor, but a row has at least 128 threads and a thread at least `least` bytes.
struct RowShape {
    int ctas, threads;  // threads of a CTA: 128, 256 or 512
};
constexpr int ROW_THREADS = 512, ROW_CTAS = 8;  // at most
inline RowShape row_shape(int64_t rows, int64_t row_bytes, int64_t per_sm, int64_t least)
{
    int64_t most = 148 * per_sm / rows;
    if (most > row_bytes / least) most = row_bytes / least;
    int n = 128;
    while (n < ROW_CTAS * ROW_THREADS && 2 * n <= most) n *= 2;
    const int threads = n < 256 ? 128 : n <= 256 * ROW_CTAS ? 256 : ROW_THREADS;
    return RowShape{n / threads, threads};
}

// A warp's walk over its chunks of a part (every warps-th from its own number on).  A lane copies its groups of the next DEPTH chunks
// into places of its own in shared memory (`ring`: R 16 bytes per thread for each of them), so that what is on its way costs no registers and
// nothing has to be waited for but the lane's own copies.
template <typename T, int R, int DEPTH>
struct ChunkWalk {
    static constexpr int BYTES = DEPTH * R * 16;  // of the ring, per thread
    // Bytes of a ring for no more chunks than a warp has to walk over.
    static int bytes(const RowShape& shape, int V)
    {
        const int chunks = (V + PER<T> - 1 + 32 * R * PER<T> - 1) / (32 * R * PER<T>), warps = shape.ctas * shape.threads / 32;
        const int slots = (chunks + shape.ctas - 1) / shape.ctas * shape.ctas;  // (CTAs' parts differ by a chunk)
        const int each = (slots + warps - 1) / warps;
        return shape.threads * R * 16 * (each < DEPTH ? each : DEPTH);
    }
    uint4* ring;
    int threads, warps;  // that walk together
    // Chunk c (if the part has it) into the ring's slot; one group of copies, empty or not.
    __device__ __forceinline__ void fetch(const T* row, const RowSplit& split, int V, int c, int slot)
    {
        if (c < split.chunk1) {
            const int first = chunk_first<T, R>(c, split.pre);
            const int mine = first + (int)(threadIdx.x & 31) * PER<T>;
            const T* from = row + mine;
            const uint32_t to = (uint32_t)__cvta_generic_to_shared(place(slot, 0));
            const bool inside = chunk_inside<T, R>(first, V);
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (inside || group_inside<T>(mine + 32 * PER<T> * r, V))
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + r * (uint32_t)threads * 16),
                                 "l"(from + 32 * PER<T> * r)
                                 : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    template <int LEFT>
    static __device__ __forceinline__ void wait()
    {
        asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
    }
    // Group r of a slot's chunk (the warp's groups of one r are consecutive).
    __device__ __forceinline__ uint4* place(int slot, int r) const { return ring + (slot * R + r) * threads; }
    __device__ __forceinline__ void start(void* shared, int threads_, const T* row, const RowSplit& split, int V)
    {
        ring = (uint4*)shared + threadIdx.x;
        threads = threads_;
        warps = threads / 32;
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) fetch(row, split, V, split.chunk0 + (int)(threadIdx.x >> 5) + d * warps, d);
    }
    // What a slot holds of a chunk; `fill` stands outside the row.
    __device__ __forceinline__ void take(const T* row, const RowSplit& split, int V, T fill, int chunk, int slot, uint4 (&raw)[R])
    {
        const int first = chunk_first<T, R>(chunk, split.pre);
        if (chunk_inside<T, R>(first, V)) {
#pragma unroll
            for (int r = 0; r < R; ++r) raw[r] = *place(slot, r);
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int v = first + (32 * r + (int)(threadIdx.x & 31)) * PER<T>;
                raw[r] = group_inside<T>(v, V) ? *place(slot, r) : edge_group(row, v, V, fill);
            }
        }
    }
    // f(chunk, slot, groups) for each chunk of a part of any length.
    template <typename F>
    __device__ __forceinline__ void each(const T* row, const RowSplit& split, int V, T fill, F f)
    {
        int slot = 0;
        for (int chunk = split.chunk0 + (int)(threadIdx.x >> 5); chunk < split.chunk1; chunk += warps) {
            wait<DEPTH - 1>();
            uint4 raw[R];
            take(row, split, V, fill, chunk, slot, raw);
            f(chunk, slot, raw);
            // (the place is free: its groups have been worked on)
            fetch(row, split, V, chunk + DEPTH * warps, slot);
            slot = slot + 1 == DEPTH ? 0 : slot + 1;
        }
        wait<0>();
    }
    // The same once more behind `each`, last chunk first: the ring still holds the last DEPTH of them.
    template <typename F>
    __device__ __forceinline__ void back(const T* row, const RowSplit& split, int V, T fill, F f)
    {
        const int first = split.chunk0 + (int)(threadIdx.x >> 5);
        const int n = (split.chunk1 - first + warps - 1) / warps;  // chunks of this warp (none if not above 0)
        int slot = n > 0 ? (n - 1) % DEPTH : 0;
        for (int chunk = first + (n - 1) * warps; chunk >= first; chunk -= warps) {
            wait<DEPTH - 1>();
            uint4 raw[R];
            take(row, split, V, fill, chunk, slot, raw);
            f(chunk, slot, raw);
            fetch(row, split, V, chunk - DEPTH * warps >= first ? chunk - DEPTH * warps : split.chunk1, slot);
            slot = slot == 0 ? DEPTH - 1 : slot - 1;
        }
        wait<0>();
    }
};

// A group's values.
template <typename T>
__device__ __forceinline__ void unpack(uint4 g, float (&x)[PER<T>])
{
    if constexpr (sizeof(T) == 4) {
        x[0] = __uint_as_float(g.x), x[1] = __uint_as_float(g.y), x[2] = __uint_as_float(g.z), x[3] = __uint_as_float(g.w);
    } else {
        const uint32_t w[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (T_is_bf16<T>) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            } else {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
                x[2 * i] = f.x, x[2 * i + 1] = f.y;
            }
        }
    }
}

// --- sums of exponentials in one pass ---------------------------------------------------------------------------------------------
// 2^(x c - R) is added up with R the largest x c met so far, rounded down.  With R whole, moving a sum from one R to another
// is exact, and x c - R is rounded once (a fused multiply-add).  |R| <= 2^22 keeps R c's rounding out; rows whose maximum lies
// beyond that (the type's lowest value as a mask, say) are added up again as 2^((x - maximum) c): `far`.
// In 32 bits: a chunk's terms are added in a tree and a thread has few chunks, which leaves chains of some tens of additions, off
// by 2^-24 each at most.
constexpr float REF_MOST = 4194304.0f;
__device__ __forceinline__ float exp_ref(float max, float c)
{
    // (rounded down by adding 1.5 2^23, whose neighbours are 1 away: floorf is the multifunction unit's, which is the busiest)
    const float x = fminf(fmaxf(max * c, -REF_MOST), REF_MOST);
    return __fadd_rd(x, 12582912.0f) - 12582912.0f;
}
__device__ __forceinline__ bool exp_far(float max, float c) { return max != -INFINITY && !(fabsf(max * c) < REF_MOST); }

// 2^d for a whole number d <= 0.
__device__ __forceinline__ float exp2_whole(float d) { return d < -126.0f ? 0.0f : __int_as_float((127 + (int)d) << 23); }

struct ExpSum {
    float ref, sum;
    static __device__ __forceinline__ ExpSum none() { return ExpSum{-REF_MOST, 0.0f}; }
    __device__ __forceinline__ void raise(float to)
    {
        if (to > ref) {
            sum *= exp2_whole(ref - to);
            ref = to;
        }
    }
    __device__ __forceinline__ void add(ExpSum o)
    {
        raise(o.ref);
        sum += o.sum * exp2_whole(o.ref - ref);
    }
    // Of the warp; every lane has it.
    __device__ __forceinline__ void warp_reduce()
    {
#pragma unroll 1  // (small code: what runs once is fetched once, and small calls are bound by that)
        for (int o = 16; o > 0; o >>= 1) add(ExpSum{__shfl_xor_sync(0xffffffffu, ref, o), __shfl_xor_sync(0xffffffffu, sum, o)});
    }
};

// The larger of two values, NaN if one of them is.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// Largest value of N groups (NaN if there is one).
template <typename T, int N>
__device__ __forceinline__ float groups_max(const uint4 (&raw)[N])
{
    if constexpr (sizeof(T) == 4) {
        float m = -INFINITY;
#pragma unroll
        for (int r = 0; r < N; ++r) {
            float x[4];
            unpack<T>(raw[r], x);
            m = max_nan(m, max_nan(max_nan(x[0], x[1]), max_nan(x[2], x[3])));
        }
        return m;
    } else {
        // two at a time
        using T2 = std::conditional_t<T_is_bf16<T>, __nv_bfloat162, __half2>;
        auto two = [](uint32_t w) { return *reinterpret_cast<T2*>(&w); };
        T2 m = two(raw[0].x);
#pragma unroll
        for (int r = 0; r < N; ++r)
            m = __hmax2_nan(m, __hmax2_nan(__hmax2_nan(two(raw[r].x), two(raw[r].y)), __hmax2_nan(two(raw[r].z), two(raw[r].w))));
        return max_nan(row_value(m.x), row_value(m.y));
    }
}

// Two products and sums, products or sums in one instruction.
__device__ __forceinline__ float2 fma_two(float2 a, float2 b, float2 c)
{
    unsigned long long y;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(y)
        : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)),
          "l"(*reinterpret_cast<unsigned long long*>(&c)));
    return *reinterpret_cast<float2*>(&y);
}
__device__ __forceinline__ float2 mul_two(float2 a, float2 b)
{
    unsigned long long y;
    asm("mul.rn.f32x2 %0, %1, %2;"
        : "=l"(y)
        : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)));
    return *reinterpret_cast<float2*>(&y);
}
__device__ __forceinline__ float2 add_two(float2 a, float2 b)
{
    unsigned long long y;
    asm("add.rn.f32x2 %0, %1, %2;"
        : "=l"(y)
        : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)));
    return *reinterpret_cast<float2*>(&y);
}

// Adds N groups to a sum.  `max`: not below any of their values.
template <typename T, int N>
__device__ __forceinline__ void add_groups(ExpSum& s, const uint4 (&raw)[N], float max, float c)
{
    s.raise(exp_ref(max, c));
    const float2 cc = make_float2(c, c), ref = make_float2(-s.ref, -s.ref);
    float2 part[N];
#pragma unroll
    for (int r = 0; r < N; ++r) {
        float x[PER<T>];
        unpack<T>(raw[r], x);
        float2 e[PER<T> / 2];
#pragma unroll
        for (int i = 0; i < PER<T> / 2; ++i) {
            const float2 y = fma_two(make_float2(x[2 * i], x[2 * i + 1]), cc, ref);
            e[i] = make_float2(exp2_unit(y.x), exp2_unit(y.y));
        }
#pragma unroll
        for (int w = PER<T> / 4; w > 0; w /= 2)
#pragma unroll
            for (int i = 0; i < w; ++i) e[i] = add_two(e[i], e[i + w]);
        part[r] = e[0];
    }
#pragma unroll
    for (int r = 1; r < N; ++r) part[0] = add_two(part[0], part[r]);
    s.sum += part[0].x + part[0].y;
}

// Sums of exponentials and of how far they lie below the largest, for log probabilities and entropies.  The words at the largest value met
// so far (`max`, the same in all lanes of a warp) are counted and stay out of the sums: beside their ones the rest of a row that is nearly
// sure, which is all that its entropy and its likely word's log probability consist of, would lose its digits.  What is left is
//   sum = sum 2^(x c - R),   spread = sum 2^(x c - R) (x c - R)     over the words below it, R as in ExpSum
struct SpreadSum {
    float max, ref, sum, spread;
    int most;
    static __device__ __forceinline__ SpreadSum none() { return SpreadSum{-INFINITY, -REF_MOST, 0.0f, 0.0f, 0}; }
    __device__ __forceinline__ void raise(float to)
    {
        if (to > ref) {
            const float by = ref - to, f = exp2_whole(by);
            spread = __fmaf_rn(by, sum, spread) * f;
            sum *= f;
            ref = to;
        }
    }
    // A larger value (or NaN) has been met: the counted words go into the sums.
    __device__ __forceinline__ void top(float to, float c)
    {
        if (to == max || max != max) return;  // (NaN stays)
        raise(exp_ref(to, c));
        if (most && max > -INFINITY) {
            const float y = __fmaf_rn(max, c, -ref), e = exp2_unit(y) * (float)most;
            sum += e;
            spread = __fmaf_rn(e, y > -200.0f ? y : -200.0f, spread);
        }
        most = 0;
        max = to;
    }
    // Adds N groups of each lane of a warp, of which `lane_max` is the largest value (NaN if there is one).
    template <typename T, int N>
    __device__ __forceinline__ void add(const uint4 (&raw)[N], float lane_max, float c)
    {
        const float to = key_value(__reduce_max_sync(0xffffffffu, order_key(lane_max)));
        const bool has = !(to < max);
        if (has) top(to, c);
        if (has) add_groups<T, N, true>(raw, c);
        else add_groups<T, N, false>(raw, c);
    }
    // The same with what the exponent is relative to given: 2^((x - max) c) (rows far from zero, `exp_far`).
    template <typename T, int N, bool HAS, bool FAR = false>
    __device__ __forceinline__ void add_groups(const uint4 (&raw)[N], float c)
    {
        const float2 cc = make_float2(c, c), from = FAR ? make_float2(-max, -max) : make_float2(-ref, -ref);
        float2 part[N], far_off[N];
#pragma unroll
        for (int r = 0; r < N; ++r) {
            float x[PER<T>];
            unpack<T>(raw[r], x);
            float2 e[PER<T> / 2];
            far_off[r] = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < PER<T> / 2; ++i) {
                const float2 two = make_float2(x[2 * i], x[2 * i + 1]);
                float2 y = FAR ? mul_two(add_two(two, from), cc) : fma_two(two, cc, from);
                // (a masked word's minus infinity times its zero)
                y.x = max_nan(y.x, -200.0f), y.y = max_nan(y.y, -200.0f);
                e[i] = make_float2(exp2_unit(y.x), exp2_unit(y.y));
                if (HAS) {
                    if (two.x == max) e[i].x = 0.0f, ++most;
                    if (two.y == max) e[i].y = 0.0f, ++most;
                }
                far_off[r] = fma_two(e[i], y, far_off[r]);
            }
#pragma unroll
            for (int w = PER<T> / 4; w > 0; w /= 2)
#pragma unroll
                for (int i = 0; i < w; ++i) e[i] = add_two(e[i], e[i + w]);
            part[r] = e[0];
        }
#pragma unroll
        for (int r = 1; r < N; ++r) part[0] = add_two(part[0], part[r]), far_off[0] = add_two(far_off[0], far_off[r]);
        sum += part[0].x + part[0].y;
        spread += far_off[0].x + far_off[0].y;
    }
    // Of the lanes of a warp, whose largest values and R are the same; every lane has it.
    __device__ __forceinline__ void lanes()
    {
#pragma unroll 1
        for (int o = 16; o > 0; o >>= 1) {
            sum += __shfl_xor_sync(0xffffffffu, sum, o);
            spread += __shfl_xor_sync(0xffffffffu, spread, o);
        }
        most = (int)__reduce_add_sync(0xffffffffu, (unsigned)most);
    }
    // Those of other words (not of rows far from zero).
    __device__ __forceinline__ void join(SpreadSum o, float c)
    {
        const float m = max_nan(max, o.max);
        top(m, c);
        o.top(m, c);
        raise(exp_ref(m, c));
        o.raise(ref);
        sum += o.sum, spread += o.spread, most += o.most;
    }
    // Of the lanes of a warp; every lane has it.
    __device__ __forceinline__ void warp_reduce(float c)
    {
        top(key_value(__reduce_max_sync(0xffffffffu, order_key(max))), c);
        raise(exp_ref(max, c));
        lanes();
    }
};

// What the sums say of a row (by one thread): in natural units, relative to the largest value.
struct SpreadRow {
    float max;
    double log_z, mean;  // logarithm of the sum of exponentials; mean of (max - x) / tau
    static __device__ __forceinline__ SpreadRow of(const SpreadSum& s, bool far, float c)
    {
        const double phi = far ? 0.0 : (double)__fmaf_rn(s.max, c, -s.ref), to = exp2(-phi);
        const double rest = (double)s.sum * to, z = rest + s.most;
        SpreadRow r;
        r.max = s.max;
        if (s.max == -INFINITY) {  // masked whole
            r.log_z = r.mean = 0;
            return r;
        }
        r.log_z = s.max < INFINITY ? log1p(rest + (s.most - 1)) : NAN;  // (NaN too, and infinity, of which nothing is left)
        const double mean = (phi * s.sum - s.spread) * to * LN2 / z;
        r.mean = !(s.max < INFINITY) ? NAN : mean < 0 ? 0.0 : mean;
        return r;
    }
    __device__ __forceinline__ double entropy() const { return log_z + mean; }
    // Of a word with logit x.
    __device__ __forceinline__ double logprob(float x, double inv_tau) const
    {
        return max == -INFINITY ? -INFINITY : ((double)x - (double)max) * inv_tau - log_z;
    }
};

// A group of values, each rounded once.
template <typename T>
__device__ __forceinline__ uint4 pack(const float (&x)[PER<T>])
{
    if constexpr (sizeof(T) == 4)
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (T_is_bf16<T>) {
                const __nv_bfloat162 two = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&two);
            } else {
                const __half2 two = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&two);
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// `p`, a variable in shared memory, in the CTA `rank` of the cluster.
template <typename P>
__device__ __forceinline__ P* row_peer(cg::cluster_group& cluster, P* p, int rank, int ctas)
{
    return ctas > 1 ? cluster.map_shared_rank(p, rank) : p;
}

// Barrier of all threads that share a row.
__device__ __forceinline__ void row_sync(cg::cluster_group& cluster, int ctas)
{
    if (ctas > 1) cluster.sync();
    else __syncthreads();
}

// Launches a cluster of CTAs for every row; `smem`: dynamic shared memory, `fixed`: what the kernel has besides, about.  The
// allowance for more than 48 KB is asked for once per kernel and device, as large as it can be (a call costs a microsecond).
template <auto Kernel, typename Args>
inline cudaError_t launch_rows(const Args& args, int64_t rows, RowShape shape, size_t smem, size_t fixed, cudaStream_t st)
{
    cudaLaunchConfig_t c{};
    c.gridDim = dim3((unsigned)(rows * shape.ctas));
    c.blockDim = dim3((unsigned)shape.threads);
    c.dynamicSmemBytes = smem;
    c.stream = st;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = (unsigned)shape.ctas;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    c.attrs = &at;
    c.numAttrs = shape.ctas > 1 ? 1 : 0;
    if (smem + fixed > 46 * 1024) {
        static std::atomic<bool> allowed[64];
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (dev >= 64 || !allowed[dev].load(std::memory_order_acquire)) {
            cudaFuncAttributes f;
            e = cudaFuncGetAttributes(&f, Kernel);
            if (e == cudaSuccess)
                e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - (int)f.sharedSizeBytes);
            if (e != cudaSuccess) return e;
            if (dev < 64) allowed[dev].store(true, std::memory_order_release);
        }
    }
    return cudaLaunchKernelEx(&c, Kernel, args);
}

// Sizes that every one of the operators refuses.
inline int check_rows(const void* p, int dtype, int64_t rows, int32_t V, int64_t stride)
{
    if (dtype != LDA_F32 && dtype != LDA_F16 && dtype != LDA_BF16) return LDA_EINVAL;
    if (rows < 0 || V <= 0 || stride < 0) return LDA_EINVAL;
    if (rows > 0x7fffffffll || V > LDA_ROW_MAX_V) return LDA_ERANGE;
    // an element's number stays inside 63 bits
    if (stride > (1ll << 31)) return LDA_ERANGE;
    if (rows > 0 && (!p || (uintptr_t)p % (dtype == LDA_F32 ? 4 : 2))) return LDA_EINVAL;
    return LDA_OK;
}

// Whether an address is a multiple of n (NULL is).
inline bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

// Temperatures at which 1 / tau and log2(e) / tau are ordinary single-precision values.
inline bool temperature_ok(double tau) { return tau >= 1e-6 && tau <= 1e6; }

}  // namespace lda
