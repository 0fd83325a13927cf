// Distillation from a teacher's top logits: loss of a row and its gradient with respect to the student's logits.
//
// Row: student's logits x_0..x_{V-1}, a list of words with the teacher's logits t_j, temperature tau.  q = softmax(x / tau);
// p_j = softmax of t_j / tau over the list, or, with the teacher's log-sum-exp L over its whole row, p_j = exp(t_j / tau - L) and
// one bucket more for the words that the list leaves out: P = max(0, 1 - sum p_j) against Q = sum of q over them.
//   loss  = tau^2 ( sum_j p_j (log p_j - log q_j) + P (log P - log Q) )
//   dloss / dx_v = tau (W q_v - sum of the p_j at v)   for a word of the list, W = sum p_j + P
//                = tau q_v (W - P / Q)                 for any other
// Q is summed over the unlisted words themselves: 1 - sum q_j would lose what matters where the list holds nearly all mass.
#include <algorithm>

#include "lda_device.cuh"
#include "rows.cuh"

namespace lda {

struct DistillArgs {
    const void* logits;
    int64_t stride;
    int32_t V, top;
    const int32_t* ids;
    const void* values;
    int values_dtype;
    int64_t list_stride;
    const float* teacher_lse;  // null: softmax over the list
    const float* weights;      // of the rows' losses in the gradient; null: all 1
    float* loss;               // may be null with a gradient
    void* grad;                // null: loss alone
    int64_t grad_stride;
    float scale;               // log2(e) / tau
    double tau, inv_tau;
    int ring;                  // bytes of the walk's ring (loss alone)
};

constexpr int DISTILL_GROUPS = 4;  // groups of a lane in a chunk
// Chunks on their way.  With a gradient two: 274 us for 258 (more rows at a time, which L2 holds less well); the loss alone
// with three: 150 us for 147.
__host__ __device__ constexpr int distill_depth(bool grad) { return grad ? 3 : 4; }

// What a CTA knows of its part of the row: exponentials of the words outside the list and of those on it, each word once (without a
// tail: of all words, and none), and the largest value of the former.
struct DistillPart {
    ExpSum out;
    float in, max;
};

// What the exponentials of one side, outside or on the list, are relative to: 2^(x c - ref), or 2^((x - max) c) where `far`.  Each side
// has its own, by its largest value: neither loses what it has to the other's distance, or to the row's from zero.
struct DistillScale {
    float ref, max;
    bool far;
    static __device__ __forceinline__ DistillScale of(float max, float c) { return DistillScale{exp_ref(max, c), max, exp_far(max, c)}; }
    __device__ __forceinline__ float exponent(float x, float c) const { return far ? (x - max) * c : __fmaf_rn(x, c, -ref); }
    // Where its exponents start; minus infinity for a side without mass.
    __device__ __forceinline__ double origin(float sum, float c) const
    {
        return sum == 0.0f ? -INFINITY : far ? (double)max * (double)c : (double)ref;
    }
};

// The list in shared memory, and a map with a bit for each word of the CTA's part.
struct DistillList {
    int* ids;                // -1: padding
    float *p, *t, *x;        // the teacher's exponentials (with a tail: probabilities) and logits, the student's logits
    uint32_t* bits;
    static __host__ __device__ constexpr int bytes(int top, int bits_bytes) { return (16 * top + bits_bytes + 15) / 16 * 16; }
    __device__ __forceinline__ DistillList(void* at, int top)
        : ids((int*)at), p((float*)at + top), t((float*)at + 2 * top), x((float*)at + 3 * top), bits((uint32_t*)at + 4 * top)
    {
    }
    // Whether place j stands for its word, which the list may hold twice: the first does.
    __device__ __forceinline__ bool leads(int j, bool twice) const
    {
        bool first = true;
        if (twice)
            for (int o = 0; o < j; ++o) first = first && ids[o] != ids[j];
        return first;
    }
};

// A CTA's part of a row: its words v0..v1-1; the map's first bit is word bit0.
template <typename T>
struct DistillSpan {
    RowSplit split;
    int bit0, v0, v1;
    __device__ __forceinline__ DistillSpan(const T* row, int V, int rank, int ctas)
    {
        split = RowSplit::of<T, DISTILL_GROUPS>(row, V, rank, ctas);
        bit0 = chunk_first<T, DISTILL_GROUPS>(split.chunk0, split.pre);
        v0 = max(0, bit0);
        v1 = max(v0, min(V, chunk_first<T, DISTILL_GROUPS>(split.chunk1, split.pre)));
    }
};

// Bytes of the map for parts of `chunks` chunks.
template <typename T>
__host__ __device__ constexpr int distill_bits(int chunks) { return chunks * (32 * DISTILL_GROUPS * PER<T> / 8); }

// Logarithm of a teacher's exponential e^(t / tau - shift), and the exponential in 64 bits from what expf makes of it in 32, at most two
// units of the last place off: the rounding of its argument, much larger for small probabilities, is taken out.
struct DistillTeacher {
    double inv_tau, shift;  // shift: the teacher's log-sum-exp, or the largest of the list
    __device__ __forceinline__ double log_of(float t) const { return (double)t * inv_tau - shift; }
    // (e above 0 or NaN: where the logarithm is beyond single precision, what its rounding takes away is no number)
    static __device__ __forceinline__ double exact(float e, double log_e) { return (double)e * (1.0 + (log_e - (double)(float)log_e)); }
};

// The teacher's exponentials (by one warp); returns their sum.
__device__ __forceinline__ double distill_teacher(const DistillArgs& a, const DistillList& list, const DistillTeacher& teacher)
{
    double z = 0;
    for (int j = threadIdx.x & 31; j < a.top; j += 32) {
        const float t = list.t[j];
        const double l = teacher.log_of(t);
        const float e = list.ids[j] < 0 || t == -INFINITY ? 0.0f : expf((float)l);
        list.p[j] = e;
        if (e != 0.0f) z += DistillTeacher::exact(e, l);
    }
    return warp_reduce_sum(z);
}

// Largest of the teacher's logits of the list (by one warp).
__device__ __forceinline__ float distill_teacher_max(const DistillArgs& a, const DistillList& list)
{
    float m = -INFINITY;
    for (int j = threadIdx.x & 31; j < a.top; j += 32)
        if (list.ids[j] >= 0) m = fmaxf(m, list.t[j]);
    return warp_reduce_max(m);
}

// Largest of the student's logits of the list (by one warp).
__device__ __forceinline__ float distill_list_max(const DistillArgs& a, const DistillList& list)
{
    float m = -INFINITY;
    for (int j = threadIdx.x & 31; j < a.top; j += 32)
        if (list.ids[j] >= 0) m = fmaxf(m, list.x[j]);
    return key_value(__reduce_max_sync(0xffffffffu, order_key(m)));
}

// Sum of the exponentials of the list's words in v0..v1-1, each once (by one warp).
__device__ __forceinline__ float distill_listed(const DistillArgs& a, const DistillList& list, int v0, int v1, bool twice, const DistillScale& scale)
{
    float in = 0.0f;
    for (int j = threadIdx.x & 31; j < a.top; j += 32)
        if (list.ids[j] >= v0 && list.ids[j] < v1 && list.leads(j, twice)) in += exp2_unit(scale.exponent(list.x[j], a.scale));
    return warp_reduce_sum(in);
}

// Bits of a group's elements in the map.
template <typename T>
__device__ __forceinline__ uint32_t group_bits(const uint32_t* bits, int group)
{
    const uint32_t byte = ((const uint8_t*)bits)[group * PER<T> / 8];
    return PER<T> == 8 ? byte : (byte >> (group * PER<T> % 8)) & ((1u << PER<T>) - 1);
}

// Minus infinity in the list's places of a lane's groups; `group`: the first one's number in the part.
template <typename T>
__device__ __forceinline__ void distill_mask(uint4 (&raw)[DISTILL_GROUPS], const uint32_t* bits, int group)
{
#pragma unroll
    for (int k = 0; k < DISTILL_GROUPS; ++k) {
        const uint32_t marked = group_bits<T>(bits, group + 32 * k);
        if (marked) {
            union {
                uint4 raw;
                T e[PER<T>];
            } u;
            u.raw = raw[k];
#pragma unroll
            for (int i = 0; i < PER<T>; ++i)
                if (marked >> i & 1) u.e[i] = row_element<T>(-INFINITY);
            raw[k] = u.raw;
        }
    }
}

// Sum of 2^((x - m) c) over a warp's chunks of the part, the list's words left out (TAIL).
template <typename T, bool TAIL>
__device__ __noinline__ float distill_far_sum(const T* row, const RowSplit& split, int V, float m, float c, const uint32_t* bits, int warps)
{
    constexpr int R = DISTILL_GROUPS;
    const int lane = threadIdx.x & 31;
    float o = 0.0f;
    for (int chunk = split.chunk0 + (int)(threadIdx.x >> 5); chunk < split.chunk1; chunk += warps) {
        uint4 raw[R];
        load_chunk<T, R>(row, chunk_first<T, R>(chunk, split.pre), V, row_element<T>(-INFINITY), raw);
        if (TAIL) distill_mask<T>(raw, bits, (chunk - split.chunk0) * 32 * R + lane);
        for (int k = 0; k < R; ++k) {
            float y[PER<T>];
            unpack<T>(raw[k], y);
            for (int i = 0; i < PER<T>; ++i) o += exp2_unit((y[i] - m) * c);
        }
    }
    return warp_reduce_sum(o);
}

// The row's sums from its parts.
struct DistillRow {
    DistillScale out_scale, in_scale;  // (without a tail the list's words are among the others: on their scale)
    float out, in;
    float sum_p, p_rest;  // the teacher's probabilities: on the list, outside
    template <bool TAIL>
    static __device__ __forceinline__ DistillRow of(const DistillPart (*parts)[ROW_CTAS], int ctas, DistillScale out_scale, float in_max, float c,
                                                    float sum_p, float p_rest)
    {
        DistillRow w;
        ExpSum out = parts[out_scale.far][0].out;
        w.in = parts[0][0].in;
        for (int k = 1; k < ctas; ++k) {
            out.add(parts[out_scale.far][k].out);
            w.in += parts[0][k].in;
        }
        w.out = out.sum;
        w.out_scale = out_scale;
        w.out_scale.ref = out.ref;
        w.in_scale = TAIL ? DistillScale::of(in_max, c) : w.out_scale;
        w.sum_p = sum_p;
        w.p_rest = TAIL && w.out != 0.0f ? p_rest : 0.0f;
        return w;
    }
    // The row's loss, by one warp, in 64 bits: it is a small difference of large logarithms where the student is near the teacher
    // (in single precision 1e-4 of a loss of 0.03, at 2 units of the last place of a logarithm of 17), and a listed word at the
    // type's lowest value has a finite log q.  z: the sum of the teacher's exponentials.
    template <bool TAIL>
    __device__ __forceinline__ float loss(const DistillArgs& a, const DistillList& list, const DistillTeacher& teacher, double z) const
    {
        const double c = a.scale, from_out = out_scale.origin(out, a.scale), from_in = in_scale.origin(in, a.scale);
        const double from = fmax(fmax(from_out, from_in), -1e300), apart = from_out - from_in;
        const double total = apart < 0 ? (double)in + (double)out * exp2(apart) : apart < INFINITY ? (double)out + (double)in * exp2(-apart) : (double)out;
        const double log_total = total == 0 ? 0.0 : log(total);  // (without mass log q is minus infinity)
        double l = 0;
        for (int j = threadIdx.x & 31; j < a.top; j += 32) {
            const float e = list.p[j];
            if (!(e > 0.0f || e != e)) continue;
            const double log_p = teacher.log_of(list.t[j]);
            l += DistillTeacher::exact(e, log_p) * (log_p - (((double)list.x[j] * c - from) * LN2 - log_total));
        }
        l = warp_reduce_sum(l);
        if (!TAIL) l = z == 0 ? 0.0 : l / z - log(z);
        // (log Q in logarithms: Q itself may be less than any number of 64 bits)
        else if (p_rest != 0.0f) l += (1 - z) * (log((1 - z) / (double)out) + log_total - (from_out - from) * LN2);
        return (float)(l * a.tau * a.tau);
    }
};

// The gradient: e times `others` for a word outside the list, w (e listed - p) for one of the list, e by its side's scale.  So the
// bucket's part, -w P times their share of it, is as large where the words outside have next to nothing of the student's mass.
struct DistillFactors {
    float others, listed, w;
    template <bool TAIL>
    static __device__ __forceinline__ DistillFactors of(const DistillRow& row, float weight, double tau, float c)
    {
        DistillFactors f;
        f.w = (float)((double)weight * tau);
        // each side's scale to the larger one (without a tail there is one)
        const float apart = TAIL ? (float)(row.out_scale.origin(row.out, c) - row.in_scale.origin(row.in, c)) : INFINITY;
        const float out_to = apart < 0 ? exp2f(apart) : 1.0f, in_to = apart > 0 ? exp2f(-apart) : 1.0f;
        const float s_out = row.out * out_to, s_in = row.in * in_to, total = s_out + s_in, p_rest = row.p_rest;
        const float each = total == 0.0f ? 0.0f : (row.sum_p + p_rest) / total;
        f.listed = each * (TAIL ? in_to : out_to);
        // W out_to / total - P / out, without the part that is in both (in single precision: the sums, 2^-22 off each, are no better)
        f.others = f.w * (p_rest != 0.0f ? (row.sum_p * s_out - p_rest * s_in) / (total * row.out) : each * out_to);
        if (weight == 0.0f) f.others = 0.0f;
        return f;
    }
};

// The gradient of a lane's groups of a chunk as if no word were listed; `stage`: the lane's places of the walk's ring.
template <typename T, typename Walk>
__device__ __forceinline__ void distill_put(T* grad, int first, int V, uint4 (&raw)[DISTILL_GROUPS], const DistillFactors& f,
                                            const DistillScale& scale, float c, bool zero, bool abreast, const Walk& walk, int slot)
{
    constexpr int R = DISTILL_GROUPS;
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 0; k < R; ++k) {
        float y[PER<T>];
        unpack<T>(raw[k], y);
        if (!scale.far) {
#pragma unroll
            for (int i = 0; i < PER<T>; i += 2) {
                const float2 e = fma_two(make_float2(y[i], y[i + 1]), make_float2(c, c), make_float2(-scale.ref, -scale.ref));
                const float2 g = mul_two(make_float2(exp2_unit(e.x), exp2_unit(e.y)), make_float2(f.others, f.others));
                y[i] = g.x, y[i + 1] = g.y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < PER<T>; ++i) y[i] = exp2_unit((y[i] - scale.max) * c) * f.others;
        }
        raw[k] = zero ? make_uint4(0, 0, 0, 0) : pack<T>(y);
    }
    if (abreast && chunk_inside<T, R>(first, V)) {
        uint4* to = reinterpret_cast<uint4*>(grad + first) + lane;
#pragma unroll
        for (int k = 0; k < R; ++k) __stcs(to + 32 * k, raw[k]);
    } else {
        // the row's edges, and rows that lie otherwise to 16 bytes than the logits': through the ring, by elements
#pragma unroll
        for (int k = 0; k < R; ++k) *walk.place(slot, k) = raw[k];
        __syncwarp();
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const T* from = (const T*)(walk.place(slot, k) - lane);
#pragma unroll
            for (int i = lane; i < 32 * PER<T>; i += 32) {
                const int v = first + 32 * PER<T> * k + i;
                if (v >= 0 && v < V) grad[v] = from[i];
            }
        }
        __syncwarp();
    }
}

// The list's words over that, by threads tid, tid + threads, ...; all: what the teacher's exponentials are divided by.
template <typename T>
__device__ __forceinline__ void distill_put_list(T* grad, const DistillArgs& a, const DistillList& list, int v0, int v1, bool twice,
                                                 const DistillFactors& f, const DistillScale& scale, float all, int tid, int threads)
{
    for (int j = tid; j < a.top; j += threads) {
        const int id = list.ids[j];
        if (id < v0 || id >= v1 || !list.leads(j, twice)) continue;
        float p = list.p[j];
        if (twice)
            for (int o = j + 1; o < a.top; ++o)
                if (list.ids[o] == id) p += list.p[o];
        grad[id] = row_element<T>(f.w * (exp2_unit(scale.exponent(list.x[j], a.scale)) * f.listed - p / all));
    }
}

// One cluster per row; every CTA has the whole list and a part of the row.  The words of the list are marked in a bit map of that
// part, so that one pass adds up the exponentials of the others; those of the list come from its own places.  The CTAs exchange
// their sums; each works out the gradient of its part from a second read, which L2 answers, and puts the list's words over it.
// 2048 rows of 141 000 words of bf16, lists of 64, loss and gradient: 254 us, 4.5 TB/s of the logits' one read and the gradient's
// write (DRAM sees 10 % more), in a replayed graph of ten calls, as all times here (calls one by one on a warm card: 277).  Both
// exponentials per word keep the multifunction units 53 % busy, the issue slots are 54 % full: what bounds it is latency.  A CTA (half a
// row) spends 14 of 24 us on the two passes, the rest on the list, the exchange and the sums, three CTAs at a time.
// The loss alone, 4096 rows of 100 000 of fp16, lists of 128: 148 us, 5.5 TB/s (calls: 168).
// The loss worked out behind the second pass by all warps, from exponentials of 64 bits: 259 us, and 13 % more for 16 rows.
// Tried: a cluster that goes from row to row with the row held in shared memory and the list worked on by a warp of its own (759 us:
// 2 KB of a row to a thread do not pay for an exchange), rows in clusters of eight held in shared memory (414 us).
template <typename T, bool TAIL, bool GRAD>
__global__ void __launch_bounds__(ROW_THREADS, 2) k_distill(DistillArgs a)
{
    constexpr int R = DISTILL_GROUPS;
    constexpr bool BITS = TAIL || GRAD;
    using Walk = ChunkWalk<T, R, distill_depth(GRAD)>;
    extern __shared__ __align__(16) uint8_t dynamic[];  // the walk's ring, the list
    const DistillList list(dynamic + (GRAD ? (int)blockDim.x * Walk::BYTES : a.ring), a.top);
    __shared__ ExpSum ered[ROW_THREADS / 32];
    __shared__ float fred[ROW_THREADS / 32];
    __shared__ DistillPart parts[2][ROW_CTAS];
    __shared__ double s_z;
    __shared__ float s_max_t, s_list_max;
    __shared__ int s_any, s_twice;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads / 32, V = a.V;
    const int64_t r = blockIdx.x / ctas;
    const T* row = (const T*)a.logits + r * a.stride;
    T* grad = GRAD ? (T*)a.grad + r * a.grad_stride : nullptr;
    const T none = row_element<T>(-INFINITY);
    const float weight = GRAD && a.weights ? a.weights[r] : 1.0f;
    const float teacher_lse = TAIL ? a.teacher_lse[r] : 0.0f;
    const DistillSpan<T> span(row, V, rank, ctas);
    const RowSplit& split = span.split;
    const int v0 = span.v0, v1 = span.v1;
    // The list's reads go ahead of the row's, which would hold them up for as long as it takes to fill the rings of all CTAs.  (The
    // student's logits of the list stay in registers until behind the pass: nothing waits for them.)
    constexpr int OWN = LDA_TOP_MAX / 128;  // places of the list per thread
    int id[OWN];
    float t[OWN];
    T own[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const int j = tid + i * threads;
        const int64_t at = r * a.list_stride + j;
        id[i] = j < a.top ? a.ids[at] : -1;
        t[i] = j < a.top ? any_value(a.values, a.values_dtype, at) : 0.0f;
    }
    Walk walk;
    walk.start(dynamic, threads, row, split, V);
    if (tid == 0) s_any = s_twice = 0;
    if (BITS)
        for (int i = tid; i < distill_bits<T>(split.chunk1 - split.chunk0) / 16; i += threads)
            ((uint4*)list.bits)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const int j = tid + i * threads;
        if (j >= a.top) break;
        const bool ok = id[i] >= 0 && id[i] < V;
        if (!ok) id[i] = -1;
        list.t[j] = t[i];
        list.ids[j] = id[i];
        if (ok) {
            s_any = 1;
            if (BITS && id[i] >= v0 && id[i] < v1) {
                const int bit = id[i] - span.bit0;
                if (atomicOr(&list.bits[bit >> 5], 1u << (bit & 31)) >> (bit & 31) & 1) s_twice = 1;
            }
            own[i] = row[id[i]];
        }
    }
    __syncthreads();
    const bool twice = s_twice;
    if (!s_any || (GRAD && weight == 0.0f && !a.loss)) {  // (the same in every CTA of the cluster)
        if (a.loss && rank == 0 && tid == 0) a.loss[r] = 0.0f;
        Walk::template wait<0>();
        if (GRAD)
            for (int v = v0 + tid; v < v1; v += threads) grad[v] = row_element<T>(0.0f);
        return;
    }
    if (ctas > 1) cluster_arrive();
    if (warp == 0) {
        const float max_t = TAIL ? 0.0f : distill_teacher_max(a, list);
        const double z = distill_teacher(a, list, DistillTeacher{a.inv_tau, TAIL ? (double)teacher_lse : (double)max_t * a.inv_tau});
        if (lane == 0) s_z = z, s_max_t = max_t;
    }
    ExpSum out = ExpSum::none();
    float m = -INFINITY;
    walk.each(row, split, V, none, [&](int chunk, int, uint4(&raw)[R]) {
        if (TAIL) distill_mask<T>(raw, list.bits, (chunk - split.chunk0) * 32 * R + lane);
        const float top = groups_max<T, R>(raw);
        m = fmaxf(m, top);  // (a NaN goes into the sums)
        add_groups<T, R>(out, raw, top, a.scale);
    });
    out.warp_reduce();
    m = warp_reduce_max(m);
    if (lane == 0) ered[warp] = out, fred[warp] = m;
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const int j = tid + i * threads;
        if (j < a.top) list.x[j] = id[i] >= 0 ? row_value(own[i]) : 0.0f;
    }
    __syncthreads();
    float in = 0.0f;
    if (warp == 0) {
        if (TAIL) {
            const float most = distill_list_max(a, list);
            in = distill_listed(a, list, v0, v1, twice, DistillScale::of(most, a.scale));
            if (lane == 0) s_list_max = most;
        }
        out = lane < warps ? ered[lane] : ExpSum::none();
        out.warp_reduce();
        m = warp_reduce_max(lane < warps ? fred[lane] : -INFINITY);
    }
    if (ctas > 1) cluster_wait();
    if (tid < ctas) *row_peer(cluster, &parts[0][rank], tid, ctas) = DistillPart{out, in, m};
    row_sync(cluster, ctas);
    m = parts[0][0].max;
    for (int k = 1; k < ctas; ++k) m = fmaxf(m, parts[0][k].max);
    const bool far = exp_far(m, a.scale);
    if (far) {  // (the same in every CTA of the cluster)
        float o = distill_far_sum<T, TAIL>(row, split, V, m, a.scale, list.bits, warps);
        if (lane == 0) fred[warp] = o;
        __syncthreads();
        if (warp == 0) o = warp_reduce_sum(lane < warps ? fred[lane] : 0.0f);
        if (tid < ctas) *row_peer(cluster, &parts[1][rank], tid, ctas) = DistillPart{{0.0f, o}, 0.0f, m};
        row_sync(cluster, ctas);
    }
    if (!GRAD && (warp != 0 || rank != 0)) return;
    const double z = s_z;  // (a list of nothing but minus infinity has no mass)
    const float sum_p = TAIL || z == 0 || z != z ? (float)z : 1.0f, p_rest = !TAIL ? 0.0f : z != z ? (float)z : (float)fmax(0.0, 1 - z);
    const DistillRow whole = DistillRow::of<TAIL>(parts, ctas, DistillScale{0.0f, m, far}, s_list_max, a.scale, sum_p, p_rest);
    if (a.loss && rank == 0 && warp == 0) {
        const float l = whole.loss<TAIL>(a, list, DistillTeacher{a.inv_tau, TAIL ? (double)teacher_lse : (double)s_max_t * a.inv_tau}, z);
        if (lane == 0) a.loss[r] = l;
    }
    if (!GRAD) return;
    const DistillFactors f = DistillFactors::of<TAIL>(whole, weight, a.tau, a.scale);
    const bool abreast = (uintptr_t)grad % 16 == (uintptr_t)row % 16;
    walk.back(row, split, V, none, [&](int chunk, int slot, uint4(&raw)[R]) {
        distill_put<T>(grad, chunk_first<T, R>(chunk, split.pre), V, raw, f, whole.out_scale, a.scale, weight == 0.0f, abreast, walk, slot);
    });
    if (weight == 0.0f) return;
    __syncthreads();
    distill_put_list<T>(grad, a, list, v0, v1, twice, f, whole.in_scale, TAIL || z == 0 ? 1.0f : (float)z, tid, threads);
}

template <typename T>
static cudaError_t run_distill(DistillArgs a, int64_t rows, cudaStream_t st)
{
    constexpr int CHUNK = 32 * DISTILL_GROUPS * PER<T>;
    const int64_t row_bytes = (int64_t)a.V * sizeof(T);
    const bool tail = a.teacher_lse, grad = a.grad;
    // what is read twice has to stay in L2 in between: rows of about 60 MB under way together (40 MB, more CTAs to a row: 302 us for
    // the 258 of then; 90 MB: 280)
    const int64_t most = grad ? std::min<int64_t>(rows, std::max<int64_t>(1, (60ll << 20) / row_bytes)) : rows;
    const RowShape shape = row_shape(most, row_bytes, 1024, 128);
    // a bit for every word of a CTA's part
    const int chunks = (a.V + PER<T> - 1 + CHUNK - 1) / CHUNK;
    // the loss alone has a ring no larger than it needs (64 rows of 131 072 words of bf16: 11.5 us for 16.3); with a gradient the list's
    // places come out cheaper from a ring of one size (the 254 above: for 260)
    a.ring = grad ? shape.threads * ChunkWalk<T, DISTILL_GROUPS, distill_depth(true)>::BYTES
                  : ChunkWalk<T, DISTILL_GROUPS, distill_depth(false)>::bytes(shape, a.V);
    const size_t smem = a.ring +
                        DistillList::bytes(a.top, tail || grad ? distill_bits<T>((chunks + shape.ctas - 1) / shape.ctas) : 0);
    constexpr size_t fixed = 2 * 1024;
    if (tail)
        return grad ? launch_rows<k_distill<T, true, true>>(a, rows, shape, smem, fixed, st)
                    : launch_rows<k_distill<T, true, false>>(a, rows, shape, smem, fixed, st);
    return grad ? launch_rows<k_distill<T, false, true>>(a, rows, shape, smem, fixed, st)
                : launch_rows<k_distill<T, false, false>>(a, rows, shape, smem, fixed, st);
}

static int distill(const DistillArgs& a, int dtype, int64_t rows, void* stream)
{
    const int values_dtype = a.values_dtype;
    int rc = check_rows(a.logits, dtype, rows, a.V, a.stride);
    if (rc != LDA_OK) return rc;
    if (values_dtype != LDA_F32 && values_dtype != LDA_F16 && values_dtype != LDA_BF16) return LDA_EINVAL;
    if (a.top < 1 || a.list_stride < 0 || !temperature_ok(a.tau)) return LDA_EINVAL;
    if (a.top > LDA_TOP_MAX || a.list_stride > (1ll << 31)) return LDA_ERANGE;
    if (rows == 0) return LDA_OK;
    if (!a.ids || !a.values || !aligned(a.ids, 4) || !aligned(a.values, values_dtype == LDA_F32 ? 4 : 2)) return LDA_EINVAL;
    if (!aligned(a.teacher_lse, 4) || !aligned(a.weights, 4) || !aligned(a.loss, 4)) return LDA_EINVAL;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = dtype == LDA_F32 ? run_distill<float>(a, rows, st)
                          : dtype == LDA_F16 ? run_distill<__half>(a, rows, st)
                                             : run_distill<__nv_bfloat16>(a, rows, st);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return LDA_ECUDA;
    }
    return LDA_OK;
}

}  // namespace lda

extern "C" int lda_distill_loss(const void* logits_dev, int dtype, int64_t rows, int32_t V, int64_t row_stride,
                                const int32_t* ids_dev, const void* values_dev, int values_dtype, int32_t top, int64_t list_stride,
                                const float* teacher_lse_dev, double temperature, float* loss_dev, void* cuda_stream)
{
    using namespace lda;
    if (rows > 0 && !loss_dev) return LDA_EINVAL;
    const DistillArgs a{logits_dev, row_stride, V, top, ids_dev, values_dev, values_dtype, list_stride, teacher_lse_dev, nullptr, loss_dev,
                        nullptr, 0, (float)(1.4426950408889634 / temperature), temperature, 1.0 / temperature, 0};
    return distill(a, dtype, rows, cuda_stream);
}

extern "C" int lda_distill_grad(const void* logits_dev, int dtype, int64_t rows, int32_t V, int64_t row_stride,
                                const int32_t* ids_dev, const void* values_dev, int values_dtype, int32_t top, int64_t list_stride,
                                const float* teacher_lse_dev, double temperature, const float* weights_dev, float* loss_dev,
                                void* grad_dev, int64_t grad_stride, void* cuda_stream)
{
    using namespace lda;
    int rc = check_rows(grad_dev, dtype, rows, V, grad_stride);
    if (rc != LDA_OK) return rc;
    if (rows > 1 && grad_stride < V) return LDA_EINVAL;
    // the gradient may take the logits' place, row for row, and may not overlap them otherwise
    if (grad_dev == logits_dev && rows > 1 && grad_stride != row_stride) return LDA_EINVAL;
    const DistillArgs a{logits_dev, row_stride, V, top, ids_dev, values_dev, values_dtype, list_stride, teacher_lse_dev, weights_dev, loss_dev,
                        grad_dev, grad_stride, (float)(1.4426950408889634 / temperature), temperature, 1.0 / temperature, 0};
    return distill(a, dtype, rows, cuda_stream);
}
