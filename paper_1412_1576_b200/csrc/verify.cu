// Verification of drafted tokens against the target's probabilities, from given random numbers.
//
// A sequence of n drafts x_1..x_n has rows p_0..p_n of the target (p_i: before draft i+1) and rows q_0..q_{n-1} of the drafter.
// Draft i is accepted iff u_i q(x_i) < p(x_i): the Metropolis-Hastings test of an independence proposal with the ratio's
// denominator on the left, as the sweep's own accept pass has it.  Behind the leading accepted drafts one token is drawn, from the
// masses max(p - q, 0) where a draft was refused and from p behind the last draft; accepted and drawn tokens together follow p, as finely
// as the uniforms do: a float32 uniform has 2^24 values as generators give it, so that of 10^6 words of equal mass some answer to 16 of them and some to 17.
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

constexpr int VERIFY_GROUPS = 4;  // groups of each row a lane has in flight
constexpr int VERIFY_CHUNKS = LDA_ROW_MAX_V / (32 * VERIFY_GROUPS * PER<float>) + 1;

// Masses: floor(2^42 x) for x in [0, 1], as 19 upper and 23 lower bits.  The bits are pushed to the end of a float by an addition of
// 2^23 that rounds down; what that leaves over is exact and goes the same way.
constexpr uint32_t MASS_ONE = 0x4B000000u;  // 2^23
struct MassSum {
    uint32_t upper, lower;
    __device__ __forceinline__ void add(float x)  // x in [0, 1]
    {
        const float hi = __fmaf_rz(x, 524288.0f, 8388608.0f);
        const float rest = __fmaf_rn(x, 524288.0f, 8388608.0f - hi);
        const float lo = __fmaf_rz(rest, 8388608.0f, 8388608.0f);
        upper += __float_as_uint(hi) - MASS_ONE;
        lower += __float_as_uint(lo) - MASS_ONE;
    }
    __device__ __forceinline__ unsigned long long value() const { return ((unsigned long long)upper << 23) + lower; }
};

// The PER values of a row from element `first` on, whose address is `off` bytes behind a multiple of 16 (off > 0, the same for all
// groups of a chunk walk): the two aligned pieces that hold them, pushed together.  Zeros outside the row.
template <typename T>
__device__ __forceinline__ uint4 shifted_group(const T* row, int first, int V, int off)
{
    const int back = off / (int)sizeof(T);  // elements of the first piece that are not wanted
    if (first - back < 0 || first - back + 2 * PER<T> > V) return edge_group(row, first, V, row_element<T>(0.0f));
    const uint4* p = reinterpret_cast<const uint4*>(row + first - back);
    const uint4 a = p[0], b = p[1];  // (b is the next lane's a: from L1)
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (off & 8)
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    if (off & 4)
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    if (sizeof(T) == 2 && (off & 2))
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// One cluster per sequence.  Every CTA finds the first draft that is refused by itself (the sequences are short), then each adds
// up the masses of its part of the row, a sum per chunk; the CTA in whose part the drawn mass falls looks for the chunk and
// reads that again to find the word.
// Bound by the read of one row of the target and, behind a refusal, one of the drafter: 256 sequences of up to five drafts over
// 141 000 words of bf16 (108 MB) take 29 us, of which the pass is 16 us at 6.6 TB/s; before it stand three reads that need each other
// (offsets, drafts, probabilities: 3 us), behind it the cluster's exchange and the search (6 us).  All sequences are on the GPU at
// once (row_shape: 256 threads in two CTAs each here); with twice the threads, in two turns, 34 us.  Eight groups of each row in
// flight 36 us, two 31.  Where a drafter's row starts at another offset from 16 bytes than the target's, its groups are put
// together from two aligned pieces: 42 us (word by word: 104).
template <typename T, bool PROBS>
__global__ void __launch_bounds__(ROW_THREADS, 2) k_verify(VerifyArgs a)
{
    constexpr int R = VERIFY_GROUPS, CHUNK = 32 * R * PER<T>;
    __shared__ unsigned long long sums[VERIFY_CHUNKS], red[33], parts[2][ROW_CTAS], s_want;
    __shared__ int s_taken, s_chunk, s_token;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x;
    const int64_t b = blockIdx.x / ctas, lo = a.offsets[b], hi = a.offsets[b + 1];
    if (lo < 0 || hi < lo || hi > a.n_drafts) {  // (the same in every CTA of the cluster)
        if (rank == 0 && tid == 0) a.accepted[b] = -1;
        return;
    }
    const int n = (int)(hi - lo);
    const float u = a.draw_u[b];
    const T* target = (const T*)a.target;
    const T* probs = (const T*)a.probs;
    if (ctas > 1) cluster_arrive();
    if (warp == 0) {
        int taken = n;
        for (int base = 0; base < n; base += 32) {
            const int64_t i = lo + base + lane;
            bool ok = true;
            if (i < hi) {
                const int32_t x = a.drafts[i];
                ok = false;
                if (x >= 0 && x < a.V) {
                    const double p = row_value(target[(i + b) * a.target_stride + x]);
                    const double q = PROBS ? (double)row_value(probs[i * a.probs_stride + x]) : 1.0;
                    ok = (double)a.accept_u[i] * q < p;
                }
            }
            const uint32_t refusals = __ballot_sync(0xffffffffu, !ok);
            if (refusals) {
                taken = base + __ffs((int)refusals) - 1;
                break;
            }
        }
        if (lane == 0) s_taken = taken;
    }
    __syncthreads();
    const int taken = s_taken;
    const bool refused = taken < n;
    const T* prow = target + (lo + taken + b) * a.target_stride;
    const T* qrow = PROBS && refused ? probs + (lo + taken) * a.probs_stride : nullptr;
    const int V = a.V;
    int32_t gone = !PROBS && refused ? a.drafts[lo + taken] : -1;  // the word that the draft takes out of p
    if (gone < 0 || gone >= V) gone = -1;
    const RowSplit split = RowSplit::of<T, R>(prow, V, rank, ctas);
    // how far the drafter's groups are behind multiples of 16 bytes, where the target's are at one
    const int off = PROBS && qrow ? (int)(((uintptr_t)qrow - (uintptr_t)prow) & 15) : 0;
    if (ctas > 1) cluster_wait();
    int token = -1;
    bool here = true;  // whether this CTA writes the token
    for (int plain = 0; plain < 2; ++plain) {
        const T* q = plain ? nullptr : qrow;
        const int32_t out = plain ? -1 : gone;
        auto part = [&](int v) {
            const float p = row_value(prow[v]);
            return q ? __saturatef(p - row_value(q[v])) : v == out ? 0.0f : __saturatef(p);
        };
        for (int c = split.chunk0 + warp; c < split.chunk1; c += threads / 32) {
            const int first = chunk_first<T, R>(c, split.pre);
            MassSum sum{0, 0};  // of 32 words at most: below 2^25 and 2^28
            uint4 rp[R], rq[R];
            load_chunk<T, R>(prow, first, V, row_element<T>(0.0f), rp);
            if (q) {
                if (off == 0) load_chunk<T, R>(q, first, V, row_element<T>(0.0f), rq);
                else
#pragma unroll
                    for (int r = 0; r < R; ++r) rq[r] = shifted_group(q, first + (32 * r + lane) * PER<T>, V, off);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float xp[PER<T>], xq[PER<T>];
                unpack<T>(rp[r], xp);
                if (q) {
                    unpack<T>(rq[r], xq);
#pragma unroll
                    for (int i = 0; i < PER<T>; ++i) sum.add(__saturatef(xp[i] - xq[i]));
                } else {
                    const int at = out - (first + (32 * r + lane) * PER<T>);
#pragma unroll
                    for (int i = 0; i < PER<T>; ++i) sum.add(i == at ? 0.0f : __saturatef(xp[i]));
                }
            }
            // (the lower halves in two parts, so that 32 lanes' sums stay inside 32 bits)
            const uint32_t upper = __reduce_add_sync(0xffffffffu, sum.upper);
            const uint32_t low = __reduce_add_sync(0xffffffffu, sum.lower & 0xFFFFu), high = __reduce_add_sync(0xffffffffu, sum.lower >> 16);
            if (lane == 0) sums[c - split.chunk0] = ((unsigned long long)upper << 23) + ((unsigned long long)high << 16) + low;
        }
        __syncthreads();
        const int chunks = split.chunk1 - split.chunk0;
        unsigned long long own = 0;
        for (int c = tid; c < chunks; c += threads) own += sums[c];
        own = block_reduce_sum(own, red);
        if (tid < ctas) *row_peer(cluster, &parts[plain][rank], tid, ctas) = own;
        row_sync(cluster, ctas);
        unsigned long long total = 0, before = 0;
        for (int k = 0; k < ctas; ++k) {
            if (k < rank) before += parts[plain][k];
            total += parts[plain][k];
        }
        if (total == 0) {
            here = rank == 0;
            continue;
        }
        const unsigned long long U = u > 0.0f ? (u < 1.0f ? __float2ull_rz(u * 4294967296.0f) : 0xFFFFFFFFull) : 0ull;
        const unsigned long long want = __umul64hi(total, U << 32);
        here = before <= want && want < before + own;
        if (!here) break;
        for (int c = 0; c < chunks; c += threads) {
            unsigned long long all;
            const unsigned long long sum = c + tid < chunks ? sums[c + tid] : 0ull;
            const unsigned long long start = before + block_scan_excl(sum, red, all);
            if (start <= want && want < start + sum) {
                s_chunk = c + tid;
                s_want = want - start;
            }
            before += all;
        }
        __syncthreads();
        // a thread takes consecutive words, all read before the first is looked at
        const int each = CHUNK / threads;  // 8 at most
        const int first = chunk_first<T, R>(split.chunk0 + s_chunk, split.pre) + tid * each;
        const unsigned long long looked_for = s_want;
        float x[8];
        MassSum mine{0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < each && first + i >= 0 && first + i < V ? part(first + i) : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) mine.add(x[i]);
        unsigned long long all, upto = block_scan_excl(mine.value(), red, all);
        if (upto <= looked_for && looked_for < upto + mine.value()) {
            int passed = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                MassSum one{0, 0};
                one.add(x[i]);
                upto += one.value();
                passed += upto <= looked_for;
            }
            s_token = first + passed;
        }
        __syncthreads();
        token = s_token;
        break;
    }
    if (!here) return;
    for (int i = tid; i <= n; i += threads) a.tokens[lo + b + i] = i < taken ? a.drafts[lo + i] : i == taken ? token : -1;
    if (tid == 0) a.accepted[b] = taken;
}

template <typename T>
static cudaError_t run_verify(const VerifyArgs& a, int64_t n_seqs, cudaStream_t st)
{
    // 128 bytes a thread where the sequences fill the GPU (256 of 32 000 words of bf16: 10.9 us for the 12.7 of 32 bytes); few
    // short rows are done sooner by more CTAs (one of 32 000 words: 7.4 us for 9.2), of 256 threads at most (16 of 131 072 words by
    // eight CTAs of 256: 8.1 us for the 9.2 of eight of 512)
    const int64_t row_bytes = (int64_t)a.V * sizeof(T);
    RowShape shape = row_shape(n_seqs, row_bytes, 1024, 128);
    const RowShape wide = row_shape(n_seqs, row_bytes, 256, 32);
    if (wide.threads <= 256 && wide.ctas * wide.threads > shape.ctas * shape.threads) shape = wide;
    return a.probs ? launch_rows<k_verify<T, true>>(a, n_seqs, shape, 0, 17 * 1024, st)
                   : launch_rows<k_verify<T, false>>(a, n_seqs, shape, 0, 17 * 1024, st);
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
    if (!aligned(draft_offsets_dev, 8) || !aligned(drafts_dev, 4) || !aligned(accept_u_dev, 4) || !aligned(draw_u_dev, 4) ||
        !aligned(tokens_dev, 4) || !aligned(accepted_dev, 4))
        return LDA_EINVAL;
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
