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
};

#ifndef DG
#define DG 4
#endif
#ifndef DB
#define DB 2
#endif
#ifndef DD
#define DD 3
#endif
constexpr int DISTILL_GROUPS = DG;  // groups of a lane in a chunk
constexpr int DISTILL_DEPTH = DD;   // chunks on their way

// What a CTA knows of its part of the row.
struct DistillPart {
    ExpSum out, in;  // over the words outside the list and on it, each word once (without a tail: all words, nothing)
    float max;
};

// What the gradient needs of the whole row: 2^(x c - ref) times `others` for a word outside the list; weight tau W / sum of
// exponentials and weight tau for those of the list.
struct DistillRow {
    float ref, others, listed, w, list_ref;
};

// Bits of a group's elements in a map with a bit for each element.
template <typename T>
__device__ __forceinline__ uint32_t group_bits(const uint32_t* bits, int group)
{
    const uint32_t byte = ((const uint8_t*)bits)[group * PER<T> / 8];
    return PER<T> == 8 ? byte : (byte >> (group * PER<T> % 8)) & ((1u << PER<T>) - 1);
}

// One cluster per row; every CTA has the whole list and a part of the row.  The words of the list are marked in a bit map of that
// part, so that one pass adds up the exponentials of the others; those of the list come from its own places.  The CTAs exchange
// their sums, and each works out the gradient of its part: the same factor times the exponential for all words, then the list's
// words over it.  KEEP: the ring holds all of the CTA's part from the first pass on; else it is read again, from L2.
template <typename T, bool TAIL, bool GRAD, bool KEEP>
__global__ void __launch_bounds__(ROW_THREADS, DB) k_distill(DistillArgs a)
{
    constexpr int R = DISTILL_GROUPS, CHUNK = 32 * R * PER<T>;
    constexpr bool BITS = TAIL || GRAD;
    using Walk = ChunkWalk<T, R, DISTILL_DEPTH>;
    extern __shared__ __align__(16) uint8_t dynamic[];  // the walk's ring, the list, the map of its words
    int* ids = (int*)(dynamic + blockDim.x * Walk::BYTES);
    float *p = (float*)(ids + a.top), *log_p = p + a.top, *x = log_p + a.top;
    uint32_t* bits = (uint32_t*)(x + a.top);
    __shared__ ExpSum ered[ROW_THREADS / 32];
    __shared__ float fred[ROW_THREADS / 32];
    __shared__ DistillPart parts[2][ROW_CTAS];
    __shared__ DistillRow whole;
    __shared__ int s_any, s_twice;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, WARPS = threads / 32, V = a.V;
    const int64_t r = blockIdx.x / ctas;
    const T* row = (const T*)a.logits + r * a.stride;
    T* grad = GRAD ? (T*)a.grad + r * a.grad_stride : nullptr;
    const T none = row_element<T>(-INFINITY);
    const float weight = GRAD && a.weights ? a.weights[r] : 1.0f;
    const float teacher_lse = TAIL ? a.teacher_lse[r] : 0.0f;
    const RowSplit split = RowSplit::of<T, R>(row, V, rank, ctas);
    // this CTA's words, and the word of the map's first bit
    const int bit0 = chunk_first<T, R>(split.chunk0, split.pre);
    const int v0 = max(0, bit0), v1 = max(v0, min(V, chunk_first<T, R>(split.chunk1, split.pre)));
    Walk walk;
    walk.start(dynamic, row, split, V);
    if (tid == 0) s_any = s_twice = 0;
    if (BITS)
        for (int i = tid; i < (split.chunk1 - split.chunk0) * (CHUNK / 128); i += threads) ((uint4*)bits)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    for (int j = tid; j < a.top; j += threads) {
        const int64_t at = r * a.list_stride + j;
        const int id = a.ids[at];
        const bool ok = id >= 0 && id < V;
        p[j] = any_value(a.values, a.values_dtype, at);
        ids[j] = ok ? id : -1;
        if (ok) {
            s_any = 1;
            if (BITS && id >= v0 && id < v1) {
                const int bit = id - bit0;
                if (atomicOr(&bits[bit >> 5], 1u << (bit & 31)) >> (bit & 31) & 1) s_twice = 1;
            }
            x[j] = row_value(row[id]);
        }
    }
    __syncthreads();
    if (!s_any || (GRAD && weight == 0.0f && !a.loss)) {  // (the same in every CTA of the cluster)
        if (a.loss && rank == 0 && tid == 0) a.loss[r] = 0.0f;
        walk.drop();
        if (GRAD) {
            const bool aligned = (uintptr_t)grad % 16 == (uintptr_t)row % 16;
            for (int v = v0 + tid * PER<T>; v < v1 + PER<T>; v += threads * PER<T>) {
                const int first = (v + split.pre) / PER<T> * PER<T> - split.pre;  // the group that v is in
                if (aligned && first >= v0 && first + PER<T> <= v1)
                    *reinterpret_cast<uint4*>(grad + first) = make_uint4(0, 0, 0, 0);
                else
                    for (int i = max(first, v0); i < min(first + PER<T>, v1); ++i) grad[i] = row_element<T>(0.0f);
            }
        }
        return;
    }
    if (ctas > 1) cluster_arrive();
    // which place of the list stands for a word that it holds twice: the first
    auto leads = [&](int j) {
        bool first = true;
        if (s_twice)
            for (int o = 0; o < j; ++o) first = first && ids[o] != ids[j];
        return first;
    };
    // the teacher's probabilities and the student's words on the list (warp 0)
    float sum_p = 0.0f;
    ExpSum in = ExpSum::none();
    if (warp == 0) {
        float max_t = -INFINITY, z = 0.0f;
        if (!TAIL) {
            for (int j = lane; j < a.top; j += 32)
                if (ids[j] >= 0) max_t = fmaxf(max_t, p[j]);
            max_t = warp_reduce_max(max_t);
        }
        for (int j = lane; j < a.top; j += 32) {
            const float t = p[j];
            float l = (float)(TAIL ? (double)t * a.inv_tau - (double)teacher_lse : ((double)t - (double)max_t) * a.inv_tau);
            if (ids[j] < 0 || t == -INFINITY) l = -INFINITY;
            const float e = l == -INFINITY ? 0.0f : expf(l);
            log_p[j] = l;
            p[j] = e;
            z += e;
            if (TAIL && ids[j] >= v0 && ids[j] < v1 && leads(j)) {
                in.raise(exp_ref(x[j], a.scale));
                in.sum += exp2_unit(__fmaf_rn(x[j], a.scale, -in.ref));
            }
        }
        z = warp_reduce_sum(z);
        if (TAIL) {
            sum_p = z;
            in.warp_reduce();
        } else if (z > 0.0f || z != z) {  // (a list of nothing but minus infinity has no mass)
            const float log_z = logf(z);
            for (int j = lane; j < a.top; j += 32) {
                p[j] = p[j] / z;
                log_p[j] -= log_z;
            }
            sum_p = z == z ? 1.0f : z;
        }
    }
    // the student's words outside the list
    ExpSum out = ExpSum::none();
    float m = -INFINITY;
    // minus infinity in the list's places
    auto mask = [&](int c, uint4(&raw)[R]) {
        if (!TAIL) return;
        const int g = (c - split.chunk0) * 32 * R + lane;
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const uint32_t marked = group_bits<T>(bits, g + 32 * k);
            if (marked) {
                union {
                    uint4 raw;
                    T e[PER<T>];
                } u;
                u.raw = raw[k];
#pragma unroll
                for (int i = 0; i < PER<T>; ++i)
                    if (marked >> i & 1) u.e[i] = none;
                raw[k] = u.raw;
            }
        }
    };
    walk.each(row, split, V, none, [&](int c, uint4(&raw)[R]) {
        const float top = groups_max<T, R>(raw);
        mask(c, raw);
        m = fmaxf(m, top);  // (a NaN goes into the sums)
        add_groups<T, R>(out, raw, top, a.scale);
    });
    if (GRAD && !KEEP) walk.start(dynamic, row, split, V);  // the second read is under way while the sums are put together
    out.warp_reduce();
    m = warp_reduce_max(m);
    if (lane == 0) ered[warp] = out, fred[warp] = m;
    __syncthreads();
    if (warp == 0) {
        out = lane < WARPS ? ered[lane] : ExpSum::none();
        out.warp_reduce();
        m = warp_reduce_max(lane < WARPS ? fred[lane] : -INFINITY);
    }
    if (ctas > 1) cluster_wait();
    if (tid < ctas) *cluster.map_shared_rank(&parts[0][rank], tid) = DistillPart{out, in, m};
    row_sync(cluster, ctas);
    m = parts[0][0].max;
    for (int k = 1; k < ctas; ++k) m = fmaxf(m, parts[0][k].max);
    const bool far = exp_far(m, a.scale);
    if (far) {  // (the same in every CTA of the cluster)
        float o = 0.0f, l = 0.0f;
        for (int c = split.chunk0 + warp; c < split.chunk1; c += WARPS) {
            uint4 raw[R];
            load_chunk<T, R>(row, chunk_first<T, R>(c, split.pre), V, none, raw);
            mask(c, raw);
            for (int k = 0; k < R; ++k) {
                float y[PER<T>];
                unpack<T>(raw[k], y);
                for (int i = 0; i < PER<T>; ++i) o += exp2_unit((y[i] - m) * a.scale);
            }
        }
        if (TAIL && warp == 0)
            for (int j = lane; j < a.top; j += 32)
                if (ids[j] >= v0 && ids[j] < v1 && leads(j)) l += exp2_unit((x[j] - m) * a.scale);
        o = warp_reduce_sum(o);
        l = warp_reduce_sum(l);
        if (lane == 0) fred[warp] = o;
        __syncthreads();
        if (warp == 0) o = warp_reduce_sum(lane < WARPS ? fred[lane] : 0.0f);
        if (tid < ctas) *cluster.map_shared_rank(&parts[1][rank], tid) = DistillPart{{0.0f, o}, {0.0f, l}, m};
        row_sync(cluster, ctas);
    }
    auto exponent = [&](float y, float ref) { return far ? (y - m) * a.scale : __fmaf_rn(y, a.scale, -ref); };
    if (warp == 0) {
        out = parts[far][0].out, in = parts[far][0].in;
        for (int k = 1; k < ctas; ++k) {
            out.add(parts[far][k].out);
            in.add(parts[far][k].in);
        }
        const float ref = fmaxf(out.ref, in.ref), gap = out.ref - ref;
        const float s_out = out.sum * exp2_whole(gap), total = s_out + in.sum * exp2_whole(in.ref - ref);
        const bool rest = TAIL && out.sum != 0.0f;
        const float p_rest = rest ? (sum_p != sum_p ? sum_p : fmaxf(0.0f, 1.0f - sum_p)) : 0.0f;
        const float log2_total = total == 0.0f ? 0.0f : log2f(total);  // (without mass log q is minus infinity)
        if (a.loss && rank == 0) {
            // (in 64 bits: a listed word at the type's lowest value has a finite log q)
            double l = 0;
            for (int j = lane; j < a.top; j += 32)
                if (p[j] > 0.0f || p[j] != p[j]) {
                    const double y = far ? ((double)x[j] - (double)m) * (double)a.scale : (double)x[j] * (double)a.scale - (double)ref;
                    l += (double)p[j] * ((double)log_p[j] - (y - (double)log2_total) * LN2);
                }
            l = warp_reduce_sum(l);
            if (p_rest != 0.0f) l += (double)(p_rest * (logf(p_rest) - (gap + log2f(out.sum) - log2_total) * (float)LN2));
            if (lane == 0) a.loss[r] = (float)(l * a.tau * a.tau);
        }
        if (GRAD && lane == 0) {
            const float w = (float)((double)weight * a.tau), mass = sum_p + p_rest;
            const float q = total == 0.0f ? 0.0f : mass / total;
            whole.list_ref = whole.ref = ref;
            whole.w = w;
            whole.listed = q;
            whole.others = w * (p_rest != 0.0f ? q - p_rest / s_out : q);
            if (gap < -100.0f) {
                // less than 2^-80 of the student's mass is outside the list: it counts for the bucket alone, on a scale of its own
                whole.ref = out.ref;
                whole.others = p_rest != 0.0f ? -w * p_rest / out.sum : 0.0f;
            }
        }
    }
    if (!GRAD) return;
    __syncthreads();
    const float ref = whole.ref, others = whole.others;
    const bool abreast = (uintptr_t)grad % 16 == (uintptr_t)row % 16;
    const auto put = [&](int c, uint4(&raw)[R]) {
        const int first = chunk_first<T, R>(c, split.pre);
        const bool inside = chunk_inside<T, R>(first, V);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            float y[PER<T>];
            unpack<T>(raw[k], y);
            if (!far) {
#pragma unroll
                for (int i = 0; i < PER<T>; ++i) y[i] = exp2_unit(__fmaf_rn(y[i], a.scale, -ref)) * others;
            } else {
#pragma unroll
                for (int i = 0; i < PER<T>; ++i) y[i] = exp2_unit((y[i] - m) * a.scale) * others;
            }
            raw[k] = weight == 0.0f ? make_uint4(0, 0, 0, 0) : pack<T>(y);
        }
        if (abreast && inside) {
            uint4* to = reinterpret_cast<uint4*>(grad + first) + lane;
#pragma unroll
            for (int k = 0; k < R; ++k) __stcs(to + 32 * k, raw[k]);
        } else {
            // the row's edges, and rows that lie otherwise to 16 bytes than the logits': through the ring, by elements
#pragma unroll
            for (int k = 0; k < R; ++k) *walk.place(k) = raw[k];
            __syncwarp();
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const T* from = (const T*)(walk.place(k) - lane);
#pragma unroll
                for (int i = lane; i < 32 * PER<T>; i += 32) {
                    const int v = first + 32 * PER<T> * k + i;
                    if (v >= 0 && v < V) grad[v] = from[i];
                }
            }
            __syncwarp();
        }
    };
    if (KEEP) walk.again(row, split, V, none, put);
    else walk.each(row, split, V, none, put);
    if (weight == 0.0f) return;
    __syncthreads();  // the list's words over the rest
    for (int j = tid; j < a.top; j += threads) {
        if (ids[j] < v0 || ids[j] >= v1 || !leads(j)) continue;
        float pj = p[j];
        if (s_twice)
            for (int o = j + 1; o < a.top; ++o)
                if (ids[o] == ids[j]) pj += p[o];
        grad[ids[j]] = row_element<T>(whole.w * (exp2_unit(exponent(x[j], whole.list_ref)) * whole.listed - pj));
    }
}

template <typename T>
static cudaError_t run_distill(const DistillArgs& a, int64_t rows, cudaStream_t st)
{
    constexpr int CHUNK = 32 * DISTILL_GROUPS * PER<T>;
    const int64_t row_bytes = (int64_t)a.V * sizeof(T);
    const bool tail = a.teacher_lse, grad = a.grad;
    using Walk = ChunkWalk<T, DISTILL_GROUPS, DISTILL_DEPTH>;
    RowShape shape = row_shape(rows, row_bytes, 1024, 64);
    bool keep = false;
    if (grad) {
        // as many threads as it takes to hold the row; else what is read twice has to stay in L2 in between: all rows under way
        // together at most 40 MB
        RowShape large = shape;
        while (!Walk::holds(large, a.V) && large.ctas * large.threads < ROW_CTAS * ROW_THREADS) {
            if (large.threads < 256 || large.ctas == ROW_CTAS) large.threads *= 2;
            else large.ctas *= 2;
        }
        keep = Walk::holds(large, a.V);
        shape = keep ? large : row_shape(std::min<int64_t>(rows, std::max<int64_t>(1, (40ll << 20) / row_bytes)), row_bytes, 1024, 64);
    }
    // a bit for every word of a CTA's part
    const int chunks = (a.V + PER<T> - 1 + CHUNK - 1) / CHUNK;
    const size_t smem = shape.threads * Walk::BYTES + 16 * a.top +
                        (tail || grad ? (size_t)((chunks + shape.ctas - 1) / shape.ctas) * (CHUNK / 8) : 0);
    const auto kernel = !grad ? (tail ? k_distill<T, true, false, false> : k_distill<T, false, false, false>)
                        : keep ? (tail ? k_distill<T, true, true, true> : k_distill<T, false, true, true>)
                               : (tail ? k_distill<T, true, true, false> : k_distill<T, false, true, false>);
    return launch_rows(kernel, a, rows, shape, smem, 2 * 1024, st);
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
    if (!a.ids || !a.values || (uintptr_t)a.values % (values_dtype == LDA_F32 ? 4 : 2)) return LDA_EINVAL;
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
                        nullptr, 0, (float)(1.4426950408889634 / temperature), temperature, 1.0 / temperature};
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
                        grad_dev, grad_stride, (float)(1.4426950408889634 / temperature), temperature, 1.0 / temperature};
    return distill(a, dtype, rows, cuda_stream);
}
