// Distillation from a teacher's top logits: loss of a row and its gradient with respect to the student's logits.
//
// Row: student's logits x_0..x_{V-1}, a list of words with the teacher's logits t_j, temperature tau.  q = softmax(x / tau);
// p_j = softmax of t_j / tau over the list, or, with the teacher's log-sum-exp L over its whole row, p_j = exp(t_j / tau - L) and
// one bucket more for the words that the list leaves out: P = max(0, 1 - sum p_j) against Q = sum of q over them.
//   loss  = tau^2 ( sum_j p_j (log p_j - log q_j) + P (log P - log Q) )
//   dloss / dx_v = tau (W q_v - sum of the p_j at v)   for a word of the list, W = sum p_j + P
//                = tau q_v (W - P / Q)                 for any other
// Q is summed over the unlisted words themselves: 1 - sum q_j would lose what matters where the list holds nearly all mass.
#include "lda_device.cuh"
#include "rows.cuh"

namespace lda {

struct DistillArgs {
    const void* logits;
    int64_t stride;
    int32_t V, top;
    const int32_t* ids;
    const void* values;
    int64_t list_stride;
    const float* teacher_lse;  // null: softmax over the list
    const float* weights;      // of the rows' losses in the gradient; null: all 1
    float* loss;               // may be null with a gradient
    void* grad;                // null: loss alone
    int64_t grad_stride;
    float scale;               // log2(e) / tau
    double tau, inv_tau;
};

constexpr int DISTILL_THREADS = 256;

// One CTA per row.  Dynamic shared memory: one bit per word of the vocabulary.
template <typename T, typename TV>
__global__ void __launch_bounds__(DISTILL_THREADS) k_distill(DistillArgs a)
{
    extern __shared__ uint32_t listed[];
    __shared__ int ids[LDA_TOP_MAX];
    __shared__ float p[LDA_TOP_MAX], x[LDA_TOP_MAX];
    __shared__ double dred[33];
    __shared__ float fred[32];
    __shared__ int s_any, s_twice;
    const int tid = threadIdx.x, V = a.V;
    const int64_t r = blockIdx.x;
    const T* row = (const T*)a.logits + r * a.stride;
    T* grad = a.grad ? (T*)a.grad + r * a.grad_stride : nullptr;
    const float weight = a.weights && grad ? a.weights[r] : 1.0f;
    const int words = (V + 31) / 32;
    for (int i = tid; i < words; i += DISTILL_THREADS) listed[i] = 0;
    if (tid == 0) s_any = s_twice = 0;
    __syncthreads();
    for (int j = tid; j < a.top; j += DISTILL_THREADS) {
        const int id = a.ids[r * a.list_stride + j];
        const bool ok = id >= 0 && id < V;
        ids[j] = ok ? id : -1;
        if (ok) {
            s_any = 1;
            if (atomicOr(&listed[id >> 5], 1u << (id & 31)) >> (id & 31) & 1) s_twice = 1;
            x[j] = row_value(row[id]);
        }
    }
    __syncthreads();
    if (!s_any || (weight == 0.0f && !a.loss)) {
        if (a.loss && tid == 0) a.loss[r] = 0.0f;
        if (grad)
            for (int v = tid; v < V; v += DISTILL_THREADS) grad[v] = row_element<T>(0.0f);
        return;
    }
    // the teacher's side
    const TV* values = (const TV*)a.values + r * a.list_stride;
    double t_ref = 0.0, base;  // log p = (t - t_ref) / tau - base
    if (a.teacher_lse) base = (double)a.teacher_lse[r];
    else {
        float tm = -INFINITY;
        for (int j = tid; j < a.top; j += DISTILL_THREADS)
            if (ids[j] >= 0) tm = fmaxf(tm, row_value(values[j]));
        tm = block_reduce_max(tm, fred);
        double z = 0;
        for (int j = tid; j < a.top; j += DISTILL_THREADS)
            if (ids[j] >= 0) z += (double)expf((float)(((double)row_value(values[j]) - (double)tm) * a.inv_tau));
        z = block_reduce_sum(z, dred);
        t_ref = tm == -INFINITY ? 0.0 : (double)tm;
        base = tm == -INFINITY ? INFINITY : log(z);  // nothing but minus infinity: no mass
    }
    double sum_p = 0;
    for (int j = tid; j < a.top; j += DISTILL_THREADS) {
        float e = 0.0f;
        if (ids[j] >= 0) {
            const float t = row_value(values[j]);
            e = t == -INFINITY ? 0.0f : expf((float)(((double)t - t_ref) * a.inv_tau - base));
        }
        p[j] = e;
        sum_p += (double)e;
    }
    sum_p = block_reduce_sum(sum_p, dred);
    // the student's side
    float m = -INFINITY;
    for (int v = tid; v < V; v += DISTILL_THREADS) m = fmaxf(m, row_value(row[v]));
    m = block_reduce_max(m, fred);
    const float ref = m == -INFINITY ? 0.0f : m;
    float in = 0.0f, out = 0.0f;
    for (int v = tid; v < V; v += DISTILL_THREADS) {
        const float e = exp2_unit((row_value(row[v]) - ref) * a.scale);
        if (listed[v >> 5] >> (v & 31) & 1) in += e;
        else out += e;
    }
    in = block_reduce_sum(in, fred);
    out = block_reduce_sum(out, fred);
    const double total = (double)in + (double)out;
    const double log_total = total == 0 ? 0.0 : log(total);  // (a row without mass: log q is minus infinity everywhere)
    const double p_rest = a.teacher_lse && out != 0.0f ? fmax(0.0, 1.0 - sum_p) + (sum_p != sum_p ? sum_p : 0.0) : 0.0;
    const double q_rest = total > 0 || total != total ? (double)out / total : 0.0;
    if (a.loss) {
        double l = 0;
        for (int j = tid; j < a.top; j += DISTILL_THREADS)
            if (p[j] > 0.0f || p[j] != p[j])
                l += (double)p[j] * ((((double)row_value(values[j]) - t_ref) * a.inv_tau - base) -
                                     (((double)x[j] - (double)ref) * a.inv_tau - log_total));
        l = block_reduce_sum(l, dred);
        if (p_rest != 0.0) l += p_rest * log(p_rest / q_rest);
        if (tid == 0) a.loss[r] = (float)(l * a.tau * a.tau);
    }
    if (!grad) return;
    const double mass = sum_p + p_rest;
    const double inv = total == 0 ? 0.0 : 1.0 / total;
    const double w = (double)weight * a.tau;
    const float others = weight == 0.0f ? 0.0f : (float)(w * inv * (p_rest != 0.0 ? mass - p_rest / q_rest : mass));
    __syncthreads();
    for (int v = tid; v < V; v += DISTILL_THREADS)
        if (!(listed[v >> 5] >> (v & 31) & 1))
            grad[v] = row_element<T>(weight == 0.0f ? 0.0f : exp2_unit((row_value(row[v]) - ref) * a.scale) * others);
    for (int j = tid; j < a.top; j += DISTILL_THREADS) {
        if (ids[j] < 0) continue;
        double pj = (double)p[j];
        bool first = true;
        if (s_twice)
            for (int o = 0; o < a.top; ++o)
                if (o != j && ids[o] == ids[j]) {
                    first = first && o > j;
                    pj += (double)p[o];
                }
        const float e = exp2_unit((x[j] - ref) * a.scale);
        if (first) grad[ids[j]] = row_element<T>(weight == 0.0f ? 0.0f : (float)(w * ((double)e * inv * mass - pj)));
    }
}

template <typename T, typename TV>
static cudaError_t run_distill(const DistillArgs& a, int64_t rows, cudaStream_t st)
{
    const size_t smem = (size_t)(a.V + 31) / 32 * 4;
    if (smem > 32 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(k_distill<T, TV>, cudaFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
        if (e != cudaSuccess) return e;
    }
    k_distill<T, TV><<<(unsigned)rows, DISTILL_THREADS, smem, st>>>(a);
    return cudaGetLastError();
}

template <typename T>
static cudaError_t run_distill(const DistillArgs& a, int values_dtype, int64_t rows, cudaStream_t st)
{
    return values_dtype == LDA_F32 ? run_distill<T, float>(a, rows, st)
           : values_dtype == LDA_F16 ? run_distill<T, __half>(a, rows, st)
                                     : run_distill<T, __nv_bfloat16>(a, rows, st);
}

static int distill(const DistillArgs& a, int dtype, int values_dtype, int64_t rows, void* stream)
{
    int rc = check_rows(a.logits, dtype, rows, a.V, a.stride);
    if (rc != LDA_OK) return rc;
    if (values_dtype != LDA_F32 && values_dtype != LDA_F16 && values_dtype != LDA_BF16) return LDA_EINVAL;
    if (a.top < 1 || a.list_stride < 0 || !temperature_ok(a.tau)) return LDA_EINVAL;
    if (a.top > LDA_TOP_MAX || a.list_stride > (1ll << 31)) return LDA_ERANGE;
    if (rows == 0) return LDA_OK;
    if (!a.ids || !a.values || (uintptr_t)a.values % (values_dtype == LDA_F32 ? 4 : 2)) return LDA_EINVAL;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = dtype == LDA_F32 ? run_distill<float>(a, values_dtype, rows, st)
                          : dtype == LDA_F16 ? run_distill<__half>(a, values_dtype, rows, st)
                                             : run_distill<__nv_bfloat16>(a, values_dtype, rows, st);
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
    const DistillArgs a{logits_dev, row_stride, V, top, ids_dev, values_dev, list_stride, teacher_lse_dev, nullptr, loss_dev,
                        nullptr, 0, (float)(1.4426950408889634 / temperature), temperature, 1.0 / temperature};
    return distill(a, dtype, values_dtype, rows, cuda_stream);
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
    const DistillArgs a{logits_dev, row_stride, V, top, ids_dev, values_dev, list_stride, teacher_lse_dev, weights_dev, loss_dev,
                        grad_dev, grad_stride, (float)(1.4426950408889634 / temperature), temperature, 1.0 / temperature};
    return distill(a, dtype, values_dtype, rows, cuda_stream);
}
