// Log probabilities of given tokens and entropies of their rows, and the gradient of both.
//
// Row: logits x_0..x_{V-1}, token t, temperature tau, m the largest logit.  With q = softmax(x / tau):
//   Z = sum exp((x - m) / tau),  mean = sum q (m - x) / tau
//   log q_t = (x_t - m) / tau - log Z,   entropy = log Z + mean        (all terms of one sign: nothing cancels)
//   d log q_t / dx_v = ((v = t) - q_v) / tau,   d entropy / dx_v = -q_v (mean - (m - x_v) / tau) / tau
// With a list of the largest words too: toplogits.cu.
#include <algorithm>

#include "lda_device.cuh"
#include "rows.cuh"
#include "toplogits.cuh"

namespace lda {

struct LogprobArgs {
    const void* logits;
    int64_t stride;
    int32_t V;
    const int32_t* tokens;
    float scale;  // log2(e) / tau
    double inv_tau;
    float *logprobs, *entropy, *stats;
};

constexpr int LOGPROB_GROUPS = 4, LOGPROB_DEPTH = 4;  // groups of a lane in a chunk, chunks on their way

// One cluster per row: one pass, then the CTAs' sums.  2048 rows of 141 000 words of bf16: 101 us, 5.7 TB/s; 777 rows of 100 003 of fp16: 38 us (six rows
// on some multiprocessors, five on others: 740 rows take 34).  Multifunction units 58 %, issue slots 55 % full.
// Tried: 256 threads a row (101 and 40 us), rings of three and two chunks (99 to 100), rows of the second kind in clusters of two or four (40, 46).
template <typename T>
__global__ void __launch_bounds__(ROW_THREADS, 2) k_logprobs(LogprobArgs a)
{
    constexpr int R = LOGPROB_GROUPS;
    extern __shared__ __align__(16) uint8_t dynamic[];  // the walk's ring
    __shared__ SpreadSum red[ROW_THREADS / 32], parts[2][ROW_CTAS];
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads / 32, V = a.V;
    const int64_t r = blockIdx.x / ctas;
    const T* row = (const T*)a.logits + r * a.stride;
    const T none = row_element<T>(-INFINITY);
    const RowSplit split = RowSplit::of<T, R>(row, V, rank, ctas);
    int token = -1;
    float x = 0.0f;
    if (rank == 0 && tid == 0) {  // (read ahead of the row, needed behind it)
        token = a.tokens[r];
        if (token < 0 || token >= V) token = -1;
    }
    ChunkWalk<T, R, LOGPROB_DEPTH> walk;
    walk.start(dynamic, threads, row, split, V);
    if (ctas > 1) cluster_arrive();
    if (token >= 0) x = row_value(row[token]);
    SpreadSum sum = SpreadSum::none();
    walk.each(row, split, V, none, [&](int, int, uint4(&raw)[R]) { sum.add<T, R>(raw, groups_max<T, R>(raw), a.scale); });
    sum.lanes();
    if (lane == 0) red[warp] = sum;
    __syncthreads();
    if (warp == 0) {
        sum = lane < warps ? red[lane] : SpreadSum::none();
        sum.warp_reduce(a.scale);
    }
    if (ctas > 1) cluster_wait();
    if (tid < ctas) *row_peer(cluster, &parts[0][rank], tid, ctas) = sum;
    row_sync(cluster, ctas);
    float m = -INFINITY;
    for (int k = 0; k < ctas; ++k) m = max_nan(m, parts[0][k].max);
    const bool far = exp_far(m, a.scale);
    if (far) {  // (the same in every CTA of the cluster)
        sum = SpreadSum::none();
        sum.max = m;
        for (int chunk = split.chunk0 + warp; chunk < split.chunk1; chunk += warps) {
            uint4 raw[R];
            load_chunk<T, R>(row, chunk_first<T, R>(chunk, split.pre), V, none, raw);
            sum.add_groups<T, R, true, true>(raw, a.scale);
        }
        sum.lanes();
        if (lane == 0) red[warp] = sum;
        __syncthreads();
        if (warp == 0) {
            sum = lane < warps ? red[lane] : SpreadSum::none();
            sum.max = m;
            sum.lanes();
        }
        if (tid < ctas) *row_peer(cluster, &parts[1][rank], tid, ctas) = sum;
        row_sync(cluster, ctas);
    }
    if (rank != 0 || warp != 0) return;
    sum = lane < ctas ? parts[far][lane] : SpreadSum::none();
    if (far) sum.max = m, sum.lanes();
    else sum.warp_reduce(a.scale);
    if (lane != 0) return;
    const SpreadRow of = SpreadRow::of(sum, far, a.scale);
    a.logprobs[r] = token < 0 ? 0.0f : (float)of.logprob(x, a.inv_tau);
    a.entropy[r] = (float)of.entropy();
    if (a.stats) a.stats[3 * r] = of.max, a.stats[3 * r + 1] = (float)of.log_z, a.stats[3 * r + 2] = (float)of.mean;
}

template <typename T>
static cudaError_t run_logprobs(const LogprobArgs& a, int64_t rows, cudaStream_t st)
{
    const RowShape shape = row_shape(rows, (int64_t)a.V * sizeof(T), 1024, 128);
    const size_t smem = ChunkWalk<T, LOGPROB_GROUPS, LOGPROB_DEPTH>::bytes(shape, a.V);
    return launch_rows<k_logprobs<T>>(a, rows, shape, smem, 1024, st);
}

// --- gradient ----------------------------------------------------------------------------------------------------------------

struct LogprobGradArgs {
    const void* logits;
    int64_t stride;
    int32_t V;
    const int32_t* tokens;
    const float *stats, *logprob_weights, *entropy_weights;  // weights may be null: none
    float scale;
    double inv_tau;
    void* grad;
    int64_t grad_stride;
    int32_t parts;  // CTAs of a row
};

constexpr int LOGPROB_GRAD_THREADS = 256, LOGPROB_GRAD_CHUNKS = 4;  // chunks of a warp

// A CTA has a run of a row's chunks; a warp loads a chunk of 16-byte groups and writes its gradient.  The last rows come first: of what
// the forward pass has read last, L2 still holds some (both together 300 -> 296 us).  2048 rows of 141 000 words of bf16: 188 us, 6.15 TB/s.
template <typename T>
__global__ void __launch_bounds__(LOGPROB_GRAD_THREADS) k_logprobs_grad(LogprobGradArgs a)
{
    constexpr int R = LOGPROB_GROUPS, WARPS = LOGPROB_GRAD_THREADS / 32;
    __shared__ uint4 stage[WARPS][R * 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, V = a.V;
    const int64_t block = gridDim.x - 1 - blockIdx.x, r = block / a.parts;
    const int part = (int)(block - r * a.parts);
    const T* row = (const T*)a.logits + r * a.stride;
    T* grad = (T*)a.grad + r * a.grad_stride;
    const int pre = (int)((uintptr_t)row % 16 / sizeof(T));
    const int token = a.tokens[r];
    const float w = a.logprob_weights && token >= 0 && token < V ? a.logprob_weights[r] : 0.0f;
    const float h = a.entropy_weights ? a.entropy_weights[r] : 0.0f;
    const float m = a.stats[3 * r], log_z = a.stats[3 * r + 1], mean = a.stats[3 * r + 2];
    const bool zero = (w == 0.0f && h == 0.0f) || m == -INFINITY, abreast = (uintptr_t)grad % 16 == (uintptr_t)row % 16;
    const bool far = exp_far(m, a.scale);
    const float ref = exp_ref(m, a.scale), phi = __fmaf_rn(m, a.scale, -ref);
    // of 2^((x - m) c): the factor of its own, and of it times (x - m) c
    const double each = -exp(-(double)log_z) * a.inv_tau;
    const float by = (float)(each * ((double)w + (double)h * mean)), by_y = (float)(each * h * LN2);
#pragma unroll 1
    for (int i = 0; i < LOGPROB_GRAD_CHUNKS; ++i) {
        const int first = chunk_first<T, R>((part * LOGPROB_GRAD_CHUNKS + i) * WARPS + warp, pre);
        if (first >= V) break;
        uint4 raw[R];
        if (!zero) load_chunk<T, R>(row, first, V, row_element<T>(-INFINITY), raw);
        else
#pragma unroll
            for (int k = 0; k < R; ++k) raw[k] = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            float x[PER<T>];
            unpack<T>(raw[k], x);
            const int at = token - (first + (32 * k + lane) * PER<T>);
            float own = 0.0f;  // the token's logit
            const bool here = at >= 0 && at < PER<T>;
            if (here)
#pragma unroll
                for (int e = 0; e < PER<T>; ++e)
                    if (e == at) own = x[e];
#pragma unroll
            for (int e = 0; e < PER<T>; e += 2) {
                float2 y = make_float2(x[e], x[e + 1]);
                if (!far) {
                    y = fma_two(y, make_float2(a.scale, a.scale), make_float2(-ref, -ref));
                    y.x = fmaxf(y.x, -200.0f) - phi, y.y = fmaxf(y.y, -200.0f) - phi;  // (0 at the largest)
                } else
                    y.x = fmaxf((y.x - m) * a.scale, -200.0f), y.y = fmaxf((y.y - m) * a.scale, -200.0f);
                const float2 f = fma_two(y, make_float2(by_y, by_y), make_float2(by, by));
                const float2 g = mul_two(make_float2(exp2_unit(y.x), exp2_unit(y.y)), f);
                x[e] = g.x, x[e + 1] = g.y;
            }
            if (here) {
                // (1 - q of a likely token from its logarithm)
                const double below = ((double)own - (double)m) * a.inv_tau, l = below - log_z, q = exp(l);
                const float g = (float)((-expm1(l) * w - (q == 0 ? 0.0 : q * (below + mean) * h)) * a.inv_tau);
#pragma unroll
                for (int e = 0; e < PER<T>; ++e)
                    if (e == at) x[e] = g;
            }
            raw[k] = zero ? make_uint4(0, 0, 0, 0) : pack<T>(x);
        }
        if (abreast && chunk_inside<T, R>(first, V)) {
            uint4* to = reinterpret_cast<uint4*>(grad + first) + lane;
#pragma unroll
            for (int k = 0; k < R; ++k) __stcs(to + 32 * k, raw[k]);
        } else {
            // the row's edges, and rows that lie otherwise to 16 bytes than the logits': by elements
#pragma unroll
            for (int k = 0; k < R; ++k) stage[warp][32 * k + lane] = raw[k];
            __syncwarp();
            const T* from = (const T*)stage[warp];
            for (int e = lane; e < 32 * R * PER<T>; e += 32)
                if (first + e >= 0 && first + e < V) grad[first + e] = from[e];
            __syncwarp();
        }
    }
}

template <typename T>
static cudaError_t run_logprobs_grad(LogprobGradArgs a, int64_t rows, cudaStream_t st)
{
    constexpr int64_t PART = (int64_t)LOGPROB_GRAD_CHUNKS * (LOGPROB_GRAD_THREADS / 32) * 32 * LOGPROB_GROUPS * PER<T>;
    a.parts = (int32_t)((a.V + PER<T> - 1 + PART - 1) / PART);
    if (rows * a.parts > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    k_logprobs_grad<T><<<(unsigned)(rows * a.parts), LOGPROB_GRAD_THREADS, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace lda

extern "C" int lda_token_logprobs(const void* logits_dev, int dtype, int64_t rows, int32_t V, int64_t row_stride, const int32_t* tokens_dev,
                                  int32_t top, double temperature, float* logprobs_dev, float* entropy_dev, float* stats_dev,
                                  int32_t* ids_dev, float* alternatives_dev, void* cuda_stream)
{
    using namespace lda;
    const int rc = check_rows(logits_dev, dtype, rows, V, row_stride);
    if (rc != LDA_OK) return rc;
    if (top < 0 || !temperature_ok(temperature)) return LDA_EINVAL;
    if (top > LDA_TOP_MAX) return LDA_ERANGE;
    if (rows == 0) return LDA_OK;
    if (!tokens_dev || !logprobs_dev || !entropy_dev || (top > 0 && (!ids_dev || !alternatives_dev))) return LDA_EINVAL;
    if (!aligned(tokens_dev, 4) || !aligned(logprobs_dev, 4) || !aligned(entropy_dev, 4) || !aligned(stats_dev, 4)) return LDA_EINVAL;
    if (top > 0 && (!aligned(ids_dev, 4) || !aligned(alternatives_dev, 4))) return LDA_EINVAL;
    const float scale = (float)(1.4426950408889634 / temperature);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e;
    if (top > 0) {
        const TopArgs a{logits_dev, row_stride, V, top, scale, 1.0 / temperature, ids_dev, nullptr, nullptr, 0,
                        tokens_dev, logprobs_dev, entropy_dev, stats_dev, alternatives_dev};
        e = top_logprobs(a, dtype, rows, st);
    } else {
        const LogprobArgs a{logits_dev, row_stride, V, tokens_dev, scale, 1.0 / temperature, logprobs_dev, entropy_dev, stats_dev};
        e = dtype == LDA_F32 ? run_logprobs<float>(a, rows, st) : dtype == LDA_F16 ? run_logprobs<__half>(a, rows, st) : run_logprobs<__nv_bfloat16>(a, rows, st);
    }
    if (e != cudaSuccess) {
        cudaGetLastError();
        return LDA_ECUDA;
    }
    return LDA_OK;
}

extern "C" int lda_token_logprobs_grad(const void* logits_dev, int dtype, int64_t rows, int32_t V, int64_t row_stride, const int32_t* tokens_dev,
                                       const float* stats_dev, const float* logprob_weights_dev, const float* entropy_weights_dev,
                                       double temperature, void* grad_dev, int64_t grad_stride, void* cuda_stream)
{
    using namespace lda;
    int rc = check_rows(logits_dev, dtype, rows, V, row_stride);
    if (rc == LDA_OK) rc = check_rows(grad_dev, dtype, rows, V, grad_stride);
    if (rc != LDA_OK) return rc;
    if (!temperature_ok(temperature) || (rows > 1 && grad_stride < V)) return LDA_EINVAL;
    // the gradient may take the logits' place, row for row
    if (grad_dev == logits_dev && rows > 1 && grad_stride != row_stride) return LDA_EINVAL;
    if (rows == 0) return LDA_OK;
    if (!tokens_dev || !stats_dev || !aligned(tokens_dev, 4) || !aligned(stats_dev, 4)) return LDA_EINVAL;
    if (!aligned(logprob_weights_dev, 4) || !aligned(entropy_weights_dev, 4)) return LDA_EINVAL;
    const LogprobGradArgs a{logits_dev, row_stride, V, tokens_dev, stats_dev, logprob_weights_dev, entropy_weights_dev,
                            (float)(1.4426950408889634 / temperature), 1.0 / temperature, grad_dev, grad_stride, 0};
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const cudaError_t e = dtype == LDA_F32 ? run_logprobs_grad<float>(a, rows, st)
                          : dtype == LDA_F16 ? run_logprobs_grad<__half>(a, rows, st)
                                             : run_logprobs_grad<__nv_bfloat16>(a, rows, st);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return LDA_ECUDA;
    }
    return LDA_OK;
}
