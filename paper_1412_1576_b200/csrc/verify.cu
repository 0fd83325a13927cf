// Verification of drafted tokens against the target's probabilities, from given random numbers.
//
// A sequence of n drafts x_1..x_n has rows p_0..p_n of the target (p_i: before draft i+1) and rows q_0..q_{n-1} of the drafter.
// Draft i is accepted iff u_i q(x_i) < p(x_i): the Metropolis-Hastings test of an independence proposal with the ratio's
// denominator on the left, as the sweep's own accept pass has it.  Behind the leading accepted drafts one token is drawn, from the
// masses max(p - q, 0) where a draft was refused and from p behind the last draft; accepted and drawn tokens together follow p.
// Decisions are exact: the test compares products of 24 by 24 bits in doubles, and the draw is the inverse CDF over masses that
// are whole multiples of 2^-42, added up as integers, so that no order of summation and no split of the row changes a token.
#include "lda_device.cuh"
#include "rows.cuh"

namespace lda {

struct VerifyArgs {
    const int64_t* offsets;
    const int32_t* drafts;
    const void* target;
    const void* probs;  // null: the drafter has put its whole mass on the draft
    const float *accept_u, *draw_u;
    int32_t *tokens, *accepted;
    int64_t n_drafts, target_stride, probs_stride;
    int32_t V;
};

constexpr int VERIFY_THREADS = 256;

// A probability as a multiple of 2^-42: NaN and what is below zero as 0, what is above one as 1.
__device__ __forceinline__ unsigned long long prob_mass(float r)
{
    return __float2ull_rz(fminf(fmaxf(r, 0.0f), 1.0f) * 4398046511104.0f);
}

template <typename T, bool PROBS>
__global__ void __launch_bounds__(VERIFY_THREADS) k_verify(VerifyArgs a)
{
    __shared__ unsigned long long red[33];
    __shared__ int s_first, s_token;
    const int64_t b = blockIdx.x, lo = a.offsets[b], hi = a.offsets[b + 1];
    if (lo < 0 || hi < lo || hi > a.n_drafts) {
        if (threadIdx.x == 0) a.accepted[b] = -1;
        return;
    }
    const int64_t n = hi - lo;
    const T* target = (const T*)a.target;
    const T* probs = (const T*)a.probs;
    int64_t taken = 0;
    if (threadIdx.x == 0) s_token = -1;
    for (int64_t base = 0; base < n; base += VERIFY_THREADS) {
        __syncthreads();
        if (threadIdx.x == 0) s_first = VERIFY_THREADS;
        __syncthreads();
        const int64_t i = lo + base + threadIdx.x;
        if (i < hi) {
            const int32_t x = a.drafts[i];
            bool ok = false;
            if (x >= 0 && x < a.V) {
                const double p = row_value(target[(i + b) * a.target_stride + x]);
                const double q = PROBS ? (double)row_value(probs[i * a.probs_stride + x]) : 1.0;
                ok = (double)a.accept_u[i] * q < p;
            }
            if (!ok) atomicMin(&s_first, (int)threadIdx.x);
        }
        __syncthreads();
        if (s_first < VERIFY_THREADS) {
            taken += s_first;
            break;
        }
        taken += min((int64_t)VERIFY_THREADS, n - base);
    }
    const bool refused = taken < n;
    const T* prow = target + (lo + taken + b) * a.target_stride;
    const T* qrow = PROBS && refused ? probs + (lo + taken) * a.probs_stride : nullptr;
    const int32_t gone = !PROBS && refused ? a.drafts[lo + taken] : -1;
    const int per = (a.V + VERIFY_THREADS - 1) / VERIFY_THREADS;
    const int v0 = min(a.V, (int)threadIdx.x * per), v1 = min(a.V, v0 + per);
    const float u = a.draw_u[b];
    const unsigned long long U = u > 0.0f ? (u < 1.0f ? __float2ull_rz(u * 4294967296.0f) : 0xFFFFFFFFull) : 0ull;
    for (int plain = 0; plain < 2; ++plain) {
        auto mass = [&](int v) {
            float r = row_value(prow[v]);
            if (!plain) r = qrow ? r - row_value(qrow[v]) : v == gone ? 0.0f : r;
            return prob_mass(r);
        };
        unsigned long long sum = 0, total;
        for (int v = v0; v < v1; ++v) sum += mass(v);
        const unsigned long long before = block_scan_excl(sum, red, total);
        if (total == 0) continue;
        const unsigned long long want = __umul64hi(total, U << 32);
        if (sum > 0 && before <= want && want < before + sum) {
            unsigned long long run = before;
            int v = v0;
            for (; v < v1; ++v) {
                run += mass(v);
                if (run > want) break;
            }
            s_token = v;
        }
        break;
    }
    __syncthreads();
    for (int64_t i = threadIdx.x; i <= n; i += VERIFY_THREADS)
        a.tokens[lo + b + i] = i < taken ? a.drafts[lo + i] : i == taken ? s_token : -1;
    if (threadIdx.x == 0) a.accepted[b] = (int32_t)taken;
}

template <typename T>
static cudaError_t run_verify(const VerifyArgs& a, int64_t n_seqs, cudaStream_t st)
{
    if (a.probs) k_verify<T, true><<<(unsigned)n_seqs, VERIFY_THREADS, 0, st>>>(a);
    else k_verify<T, false><<<(unsigned)n_seqs, VERIFY_THREADS, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace lda

extern "C" int lda_verify_drafts(const int64_t* draft_offsets_dev, int64_t n_seqs, const int32_t* drafts_dev, int64_t n_drafts,
                                 const void* target_dev, int64_t target_stride, const void* draft_probs_dev, int64_t probs_stride,
                                 int dtype, int32_t V, const float* accept_u_dev, const float* draw_u_dev, int32_t* tokens_dev,
                                 int32_t* accepted_dev, void* cuda_stream)
{
    using namespace lda;
    if (n_seqs < 0 || n_drafts < 0) return LDA_EINVAL;
    if (n_seqs > 0x7fffffffll || n_drafts > 0x7fffffffll) return LDA_ERANGE;
    int rc = check_rows(target_dev, dtype, n_seqs, V, target_stride);
    if (rc == LDA_OK && draft_probs_dev) rc = check_rows(draft_probs_dev, dtype, n_drafts, V, probs_stride);
    if (rc != LDA_OK) return rc;
    if (n_seqs == 0) return n_drafts == 0 ? LDA_OK : LDA_EINVAL;
    if (!draft_offsets_dev || !draw_u_dev || !tokens_dev || !accepted_dev) return LDA_EINVAL;
    if (n_drafts > 0 && (!drafts_dev || !accept_u_dev)) return LDA_EINVAL;
    VerifyArgs a{draft_offsets_dev, drafts_dev, target_dev, draft_probs_dev, accept_u_dev, draw_u_dev, tokens_dev,
                 accepted_dev, n_drafts, target_stride, probs_stride, V};
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const cudaError_t e = dtype == LDA_F32 ? run_verify<float>(a, n_seqs, st)
                          : dtype == LDA_F16 ? run_verify<__half>(a, n_seqs, st)
                                             : run_verify<__nv_bfloat16>(a, n_seqs, st);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return LDA_ECUDA;
    }
    return LDA_OK;
}
