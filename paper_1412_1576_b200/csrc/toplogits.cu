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

constexpr int TOP_THREADS = 256;

// One CTA per row: the border value by four passes that count bytes of the keys, then what is above it, then the first words at it.
template <typename T>
__global__ void __launch_bounds__(TOP_THREADS) k_top(TopArgs a)
{
    __shared__ float fred[32];
    __shared__ int ired[33];
    __shared__ int hist[256];
    __shared__ unsigned long long list[LDA_TOP_MAX];
    __shared__ uint32_t s_prefix;
    __shared__ int s_need, s_n;
    const int tid = threadIdx.x, V = a.V;
    const T* row = (const T*)a.logits + (int64_t)blockIdx.x * a.stride;
    float m = -INFINITY;
    int n_valid = 0;
    for (int v = tid; v < V; v += TOP_THREADS) {
        const float x = row_value(row[v]);
        m = fmaxf(m, x);
        n_valid += x != -INFINITY;
    }
    m = block_reduce_max(m, fred);
    n_valid = block_reduce_sum(n_valid, ired);
    float s = 0.0f;
    for (int v = tid; v < V; v += TOP_THREADS) s += exp2_unit((row_value(row[v]) - m) * a.scale);
    s = block_reduce_sum(s, fred);
    const int want = min(a.top, n_valid);
    // the largest key that at least `want` words reach
    uint32_t prefix = 0;
    int need = want;
    for (int shift = 24; shift >= 0 && want > 0; shift -= 8) {
        for (int i = tid; i < 256; i += TOP_THREADS) hist[i] = 0;
        __syncthreads();
        for (int v = tid; v < V; v += TOP_THREADS) {
            const uint32_t k = order_key(row_value(row[v]));
            if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int d = 255, left = need;
            while (d > 0 && hist[d] < left) left -= hist[d--];
            s_prefix = prefix | ((uint32_t)d << shift);
            s_need = left;
        }
        __syncthreads();
        prefix = s_prefix;
        need = s_need;
        __syncthreads();
    }
    if (tid == 0) s_n = 0;
    __syncthreads();
    if (want > 0) {
        for (int v = tid; v < V; v += TOP_THREADS) {
            const uint32_t k = order_key(row_value(row[v]));
            if (k > prefix) list[atomicAdd(&s_n, 1)] = ((unsigned long long)k << 32) | (0xFFFFFFFFu - (uint32_t)v);
        }
        __syncthreads();
        int have = s_n;
        for (int base = 0; base < V && have < want; base += TOP_THREADS) {
            const int v = base + tid;
            const int at = v < V && order_key(row_value(row[v])) == prefix;
            int total;
            const int before = block_scan_excl(at, ired, total);
            if (at && have + before < want)
                list[have + before] = ((unsigned long long)prefix << 32) | (0xFFFFFFFFu - (uint32_t)v);
            have += total;
            __syncthreads();
        }
    }
    int size = 1;
    while (size < want) size *= 2;
    for (int i = want + tid; i < size; i += TOP_THREADS) list[i] = 0;
    __syncthreads();
    for (int k = 2; k <= size; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            for (int i = tid; i < size; i += TOP_THREADS) {
                const int o = i ^ j;
                if (o > i) {
                    const unsigned long long x = list[i], y = list[o];
                    if ((x < y) == ((i & k) == 0)) list[i] = y, list[o] = x;
                }
            }
            __syncthreads();
        }
    for (int i = tid; i < a.top; i += TOP_THREADS) {
        const int64_t at = (int64_t)blockIdx.x * a.top + i;
        const int v = i < want ? (int)(0xFFFFFFFFu - (uint32_t)list[i]) : -1;
        a.ids[at] = v;
        ((T*)a.values)[at] = v >= 0 ? row[v] : row_element<T>(-INFINITY);
    }
    if (a.lse && tid == 0) {
        const uint32_t first = want > 0 ? (uint32_t)(list[0] >> 32) : 0;
        a.lse[blockIdx.x] = want == 0 ? -INFINITY
                            : first == KEY_NAN ? NAN
                            : m == INFINITY ? INFINITY
                                            : (float)((double)m * a.inv_tau + (double)logf(s));
    }
}

template <typename T>
static cudaError_t run_top(const TopArgs& a, int64_t rows, cudaStream_t st)
{
    k_top<T><<<(unsigned)rows, TOP_THREADS, 0, st>>>(a);
    return cudaGetLastError();
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
