// Attention of new tokens (one per sequence, or a tree of drafted ones) over a paged cache of keys and values.
//
//   out_i = sum_j softmax_j(scale q_i k_j) v_j     over the context and over the new tokens that the mask names
//
// One pass over the keys with the running maximum and sum of the softmax.  The rows that share a head of the cache (the new tokens of a
// sequence times the query heads of a group) are taken together, so that a key is read once for all of them.
#include "attend.cuh"

namespace lda {

constexpr int KEYS = 64;  // of a tile

// --- matrix products -------------------------------------------------------------------------------------------------------------

template <typename T>
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (T_is_bf16<T>)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void load_matrices_turned(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
template <int DIM, int ROWS>
struct AttendShape {
    static constexpr int THREADS = 128;
    static constexpr int ROW_BYTES = DIM * 2, TILE_BYTES = KEYS * ROW_BYTES;  // of keys; of values as many
    static constexpr int STAGES = DIM == 64 ? 4 : 3;
    static constexpr int CTAS = DIM == 64 ? 3 : DIM == 128 ? 2 : 1;  // of a multiprocessor
    static constexpr int ROW_GROUPS = ROWS / 16, KEY_GROUPS = 4 / ROW_GROUPS;
    static constexpr int CHUNK = 32, PITCH = CHUNK + 4;  // columns that are joined at a time
    static constexpr bool Q_SHARED = DIM > 128;
    static constexpr int SHARED = STAGES * 2 * TILE_BYTES + 64 * PITCH * 4 + (Q_SHARED ? ROWS * ROW_BYTES : 0);
};

// The kernel for caches that the tensor cores' own memory does not suit: heads of more than 128 values, pages that are no multiple of 8 slots.
// A CTA of four warps walks over its units; a warp has 16 rows and, with fewer than four groups of rows, a share of every tile's keys.
// Tiles of keys and values come by asynchronous copies of 16 bytes into a ring of stages (a warp brings 16 keys of each; pages may lie
// anywhere), two or three tiles ahead, across the ends of items; what lies behind the last key is filled with zeros.
// 64 sequences of up to 8192 slots in pages of 4, one token each, 32 query heads on 8 of 128 values: 316 us, 4.3 TB/s (in pages of 16 277, for the
// 212 to 230 of the other kernel); with heads of 256 872 us, 3.1 TB/s.  Bound by latency: eight warps of a multiprocessor, four with heads of 256, go
// through copies, products and exponentials one after the other (issue slots 36 and 22 % full).
template <typename T, int DIM, int ROWS>
__global__ void __launch_bounds__(128) k_attend(const __grid_constant__ AttendArgs a)
{
    using S = AttendShape<DIM, ROWS>;
    constexpr int NK = KEYS / S::KEY_GROUPS / 8, ND = DIM / 8, CH = DIM / 8;  // blocks of 8 keys of a warp, of 8 columns; groups of a row
    extern __shared__ __align__(128) uint8_t dynamic[];
    __shared__ unsigned long long red[4], wild[S::STAGES];
    __shared__ __align__(8) uint16_t valid[S::STAGES][4];
    __shared__ float s_m[4][16], s_l[4][16];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rg = warp % S::ROW_GROUPS, kg = warp / S::ROW_GROUPS;
    const CacheView& c = a.cache;
    const uint32_t stages = (uint32_t)__cvta_generic_to_shared(dynamic);
    float* region = (float*)(dynamic + S::STAGES * 2 * S::TILE_BYTES);
    const uint32_t q_shared = stages + S::STAGES * 2 * S::TILE_BYTES + 64 * S::PITCH * 4;
    AttendShare share;
    AttendItem item, ahead;
    AttendBegun begun{};
    if (!attend_share<ROWS, KEYS>(a, blockIdx.x, share, item, red)) {
        if (tid == 0) a.begun[blockIdx.x] = begun;
        return;
    }

    // --- copies: a lane of the lower half knows the page of one of the warp's 16 keys, of the unit after the one that is copied next
    ahead = item;
    int64_t to_copy = share.lo;
    int page = -1, place = 0, copy_head = 0;
    const auto look = [&] {  // at the pages of unit `to_copy`, which `ahead` stands at
        page = -1, place = 0, copy_head = ahead.head;
        if (to_copy >= share.hi) return;
        const int key = ahead.tile * KEYS + 16 * warp + (lane & 15);
        if (key < ahead.keys) page = c.page(ahead.b, (uint32_t)key, place);
    };
    const auto copy = [&](int stage) {
        if (to_copy < share.hi) {
            const uint32_t there = __ballot_sync(0xffffffffu, page >= 0);
            if (lane == 0) valid[stage][warp] = (uint16_t)there;
            if (tid == 0) wild[stage] = 0;
            const T* keys = (const T*)c.keys + copy_head * c.k_head;
            const T* values = (const T*)c.values + copy_head * c.v_head;
            const uint32_t to = stages + stage * 2 * S::TILE_BYTES;
            const int ch = lane % CH;
#pragma unroll
            for (int i = 0; i < 16 * CH / 32; ++i) {
                const int row = i * 32 / CH + lane / CH;
                const int64_t p = __shfl_sync(0xffffffffu, page, row);
                const int s = __shfl_sync(0xffffffffu, place, row);
                const bool ok = p >= 0 && ch * 8 < c.dim;
                const int size = ok ? 16 : 0;
                const T* k = ok ? keys + p * c.k_page + s * c.k_slot + ch * 8 : (const T*)a.q;
                const T* v = ok ? values + p * c.v_page + s * c.v_slot + ch * 8 : (const T*)a.q;  // (not read)
                const uint32_t at = to + (16 * warp + row) * S::ROW_BYTES + ((ch ^ (row & 7)) << 4);
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(k), "r"(size) : "memory");
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at + S::TILE_BYTES), "l"(v), "r"(size) : "memory");
            }
            to_copy += ahead.tile + 1 == ahead.tiles ? 1 + ahead.extra_units() : 1;
            if (to_copy < share.hi) ahead.next<ROWS, KEYS>(a);
            look();
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    look();
#pragma unroll 1
    for (int s = 0; s < S::STAGES - 1; ++s) copy(s);

    // --- a warp's state: scores' maxima (times scale) and norms of its rows lane / 4 and lane / 4 + 8, and their outputs
    float m[2], l[2], o[ND][4];
    uint32_t qf[S::Q_SHARED ? 1 : DIM / 16][4];
    int place_of[2];  // the rows' tokens, -1: no row
    const auto begin_item = [&] {
#pragma unroll
        for (int i = 0; i < 2; ++i) m[i] = -INFINITY, l[i] = 0.0f;
#pragma unroll
        for (int n = 0; n < ND; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.0f;
        const T* row[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t r = (int64_t)item.row_tile * ROWS + rg * 16 + lane / 4 + 8 * i;
            const bool there = r < (int64_t)item.seq.n * a.group;
            const int token = there ? (int)(r / a.group) : 0, h = there ? (int)(r - (int64_t)token * a.group) : 0;
            place_of[i] = there ? token : -1;
            row[i] = there ? (const T*)a.q + (item.seq.first + token) * a.q_token + (item.head * a.group + h) * a.q_head : nullptr;
        }
        if constexpr (!S::Q_SHARED) {
#pragma unroll
            for (int k = 0; k < DIM / 16; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int at = 16 * k + 2 * (lane & 3) + (e >= 2 ? 8 : 0);
                    qf[k][e] = row[e & 1] && at < c.dim ? *(const uint32_t*)(row[e & 1] + at) : 0u;
                }
        } else {
            // (every key group writes the same rows the same)
#pragma unroll 1
            for (int k = 0; k < DIM / 16; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int at = 16 * k + 2 * (lane & 3) + (e >= 2 ? 8 : 0), r = rg * 16 + lane / 4 + 8 * (e & 1);
                    const uint32_t x = row[e & 1] && at < c.dim ? *(const uint32_t*)(row[e & 1] + at) : 0u;
                    const uint32_t to = q_shared + r * S::ROW_BYTES + ((at / 8 ^ (r & 7)) << 4) + at % 8 * 2;
                    asm volatile("st.shared.b32 [%0], %1;" ::"r"(to), "r"(x) : "memory");
                }
            __syncthreads();
        }
    };
    begin_item();
    int64_t item_begin = share.lo - item.tile;

    int stage = 0;
#pragma unroll 1
    for (int64_t unit = share.lo; unit < share.hi;) {
        asm volatile("cp.async.wait_group %0;" ::"n"(S::STAGES - 2) : "memory");
        __syncthreads();
        copy(stage == 0 ? S::STAGES - 1 : stage - 1);  // (the stage that the last unit has left)
        const uint32_t keys = stages + stage * 2 * S::TILE_BYTES, values = keys + S::TILE_BYTES;
        const int key0 = kg * (KEYS / S::KEY_GROUPS);  // the warp's first
        float s[NK][4];
#pragma unroll
        for (int n = 0; n < NK; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.0f;
#pragma unroll
        for (int k = 0; k < DIM / 16; ++k) {
            uint32_t q[4];
            if constexpr (S::Q_SHARED)
                load_matrices(q, q_shared + (rg * 16 + (lane & 15)) * S::ROW_BYTES + ((2 * k + (lane >> 4) ^ (lane & 7)) << 4));
            else
                q[0] = qf[k][0], q[1] = qf[k][1], q[2] = qf[k][2], q[3] = qf[k][3];
#pragma unroll
            for (int n = 0; n < NK; n += 2) {
                uint32_t b[4];
                const int row = key0 + 8 * n + (lane & 7) + (lane >> 4 << 3);
                load_matrices(b, keys + row * S::ROW_BYTES + ((2 * k + (lane >> 3 & 1) ^ (lane & 7)) << 4));
                mma_16x8x16<T>(s[n], q, b[0], b[1]);
                mma_16x8x16<T>(s[n + 1], q, b[2], b[3]);
            }
        }
        const uint2 four = *(const uint2*)valid[stage];
        const unsigned long long there = (unsigned long long)four.y << 32 | four.x;
        const bool masked = there != ~0ull || (int64_t)(item.tile + 1) * KEYS > item.seq.start;  // (the same in all threads)
        unsigned long long bad = 0;
        if (masked) {
            unsigned long long see[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                see[i] = place_of[i] < 0 ? 0ull : attend_window(a, item.seq, place_of[i], item.tile) & there;
                see[i] = see[i] >> key0 >> 2 * (lane & 3);
            }
#pragma unroll
            for (int n = 0; n < NK; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!(see[e >> 1] >> (8 * n + (e & 1)) & 1)) s[n][e] = -INFINITY;
            // a value that a row does not see must not touch it, whatever it is: infinities and NaN are taken out and added apart
            for (int i = tid; i < KEYS * CH; i += S::THREADS) {
                const int row = i / CH, ch = i % CH;
                uint4* at = (uint4*)(dynamic + stage * 2 * S::TILE_BYTES + S::TILE_BYTES + row * S::ROW_BYTES + ((ch ^ (row & 7)) << 4));
                const uint4 g = *at;
                if (has_wild<T>(g)) {
                    *at = without_wild<T>(g);
                    atomicOr(&wild[stage], 1ull << row);
                }
            }
            __syncthreads();
            bad = wild[stage];
        }
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int n = 0; n < NK; ++n) {
            top[0] = fmaxf(top[0], fmaxf(s[n][0], s[n][1]));
            top[1] = fmaxf(top[1], fmaxf(s[n][2], s[n][3]));
        }
        float shift[2];
        bool raised = false;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
            top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
            top[i] = fmaxf(m[i], top[i] * a.scale);
            raised = raised || top[i] > m[i];
        }
        if (__any_sync(0xffffffffu, raised)) {
            float f[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                f[i] = top[i] == m[i] ? 1.0f : exp2_unit(m[i] - top[i]);
                m[i] = top[i];
                l[i] *= f[i];
            }
#pragma unroll
            for (int n = 0; n < ND; ++n) o[n][0] *= f[0], o[n][1] *= f[0], o[n][2] *= f[1], o[n][3] *= f[1];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) shift[i] = (m[i] == -INFINITY ? 0.0f : -m[i]) + RAISE<T>;
#pragma unroll
        for (int n = 0; n < NK; ++n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = exp2_unit(__fmaf_rn(s[n][e], a.scale, shift[e >> 1]));
            l[0] += s[n][0] + s[n][1];
            l[1] += s[n][2] + s[n][3];
        }
        // the probabilities are rounded to the values' type, which the product takes: half a step each, as much as the output's own
        // rounding; the norm is that of the unrounded ones
#pragma unroll
        for (int j = 0; j < NK / 2; ++j) {
            const uint32_t p[4] = {pack_two<T>(s[2 * j][0], s[2 * j][1]), pack_two<T>(s[2 * j][2], s[2 * j][3]),
                                   pack_two<T>(s[2 * j + 1][0], s[2 * j + 1][1]), pack_two<T>(s[2 * j + 1][2], s[2 * j + 1][3])};
#pragma unroll
            for (int d = 0; d < DIM / 16; ++d) {
                uint32_t b[4];
                const int row = key0 + 16 * j + (lane & 15);
                load_matrices_turned(b, values + row * S::ROW_BYTES + ((2 * d + (lane >> 4) ^ (lane & 7)) << 4));
                mma_16x8x16<T>(o[2 * d], p, b[0], b[1]);
                mma_16x8x16<T>(o[2 * d + 1], p, b[2], b[3]);
            }
        }
        // (what was taken out: a row that sees it has it, whatever the probability)
        for (unsigned long long left = bad; left; left &= left - 1) {
            const int row = __ffsll((long long)left) - 1, at = row - key0;
            if (at < 0 || at >= KEYS / S::KEY_GROUPS) continue;
            float sees[2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                sees[i] = place_of[i] >= 0 && attend_window(a, item.seq, place_of[i], item.tile) >> row & 1 ? 1.0f : 0.0f;
            int slot = 0;
            const int64_t pg = c.page(item.b, (uint32_t)(item.tile * KEYS + row), slot);
            if (pg < 0) continue;
            const T* v = (const T*)c.values + pg * c.v_page + slot * c.v_slot + item.head * c.v_head + 2 * (lane & 3);
#pragma unroll
            for (int n = 0; n < ND; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float x = 8 * n < c.dim ? cache_value(v[8 * n + e]) : 0.0f;
                    if (!(fabsf(x) < INFINITY)) {
                        if (sees[0] != 0.0f) o[n][e] += x;
                        if (sees[1] != 0.0f) o[n][2 + e] += x;
                    }
                }
        }
        stage = stage + 1 == S::STAGES ? 0 : stage + 1;

        const bool ends = item.tile + 1 == item.tiles;
        unit += ends ? 1 + item.extra_units() : 1;
        if (!ends && unit < share.hi) {
            ++item.tile;
            continue;
        }
        // --- the item's end, or the share's: the key groups' sums together, then out or to the parts
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
            if ((lane & 3) == 0) s_m[warp][lane / 4 + 8 * i] = m[i], s_l[warp][lane / 4 + 8 * i] = l[i];
        }
        __syncthreads();
        const bool whole = ends && item_begin >= share.lo;
        float f[2], all_m[2], all_l[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = lane / 4 + 8 * i;
            float most = m[i], sum = 0.0f;
#pragma unroll
            for (int g = 0; g < S::KEY_GROUPS; ++g) most = fmaxf(most, s_m[g * S::ROW_GROUPS + rg][r]);
#pragma unroll
            for (int g = 0; g < S::KEY_GROUPS; ++g) {
                const float x = s_m[g * S::ROW_GROUPS + rg][r];
                sum += x == most ? s_l[g * S::ROW_GROUPS + rg][r] : s_l[g * S::ROW_GROUPS + rg][r] * exp2_unit(x - most);
            }
            f[i] = m[i] == most ? 1.0f : exp2_unit(m[i] - most);
            if (whole) f[i] = sum == 0.0f ? 0.0f : f[i] / sum;  // (a row that sees nothing is zero)
            all_m[i] = most, all_l[i] = sum;
        }
        const int slot = 2 * blockIdx.x + (item_begin < share.lo ? 0 : 1);
        const int64_t row0 = (int64_t)item.row_tile * ROWS, rows = min((int64_t)ROWS, (int64_t)item.seq.n * a.group - row0);
        if (!whole && kg == 0 && (lane & 3) == 0)
#pragma unroll
            for (int i = 0; i < 2; ++i) a.ml[slot * ROWS + rg * 16 + lane / 4 + 8 * i] = make_float2(all_m[i], all_l[i]);
#pragma unroll
        for (int from = 0; from < DIM; from += S::CHUNK) {
            if (from >= c.dim) break;
            __syncthreads();
#pragma unroll
            for (int n = 0; n < S::CHUNK / 8; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    *(float2*)(region + (warp * 16 + lane / 4 + 8 * i) * S::PITCH + 8 * n + 2 * (lane & 3)) =
                        make_float2(o[from / 8 + n][2 * i] * f[i], o[from / 8 + n][2 * i + 1] * f[i]);
            __syncthreads();
            for (int t = tid; t < ROWS * (S::CHUNK / 4); t += S::THREADS) {
                const int r = t / (S::CHUNK / 4), col = t % (S::CHUNK / 4) * 4;
                if (r >= rows || from + col >= c.dim) continue;
                float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int g = 0; g < S::KEY_GROUPS; ++g) {
                    const float4 y = *(const float4*)(region + ((g * S::ROW_GROUPS + r / 16) * 16 + r % 16) * S::PITCH + col);
                    x.x += y.x, x.y += y.y, x.z += y.z, x.w += y.w;
                }
                if (whole) {
                    const int64_t token = (row0 + r) / a.group;
                    const int h = (int)(row0 + r - token * a.group);
                    T* to = (T*)a.out + (item.seq.first + token) * a.out_token + (item.head * a.group + h) * a.out_head + from + col;
                    *(uint2*)to = make_uint2(pack_two<T>(x.x, x.y), pack_two<T>(x.z, x.w));
                } else
                    *(float4*)(a.part + ((int64_t)slot * ROWS + r) * DIM + from + col) = x;
            }
        }
        if (!ends && item_begin >= share.lo)
            begun = AttendBegun{row0, item.seq.first, item.head, (int)rows, share.last_of(item_begin, item_begin + item.own_units(), 1) - (int)blockIdx.x, 0};
        if (unit < share.hi) {
            item.next<ROWS, KEYS>(a);
            item_begin = unit;
            __syncthreads();
            begin_item();
        }
    }
    if (tid == 0) a.begun[blockIdx.x] = begun;
}

// The parts of items that several CTAs have worked on, two rows by a warp: in the order of the keys, so that the same call gives the same
// bits.  Every such item begins in one CTA, which has said so.  Bound by reads that need each other, three of them: the item; its parts' maxima
// and first sums; the other sums.
constexpr int JOIN_WARPS = 4, JOIN_ROWS = 2, JOIN_PARTS = 32 / JOIN_ROWS;  // rows of a warp, parts that its lanes look at together
template <typename T, int DIM>
__global__ void __launch_bounds__(32 * JOIN_WARPS) k_attend_join(const __grid_constant__ AttendArgs a)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const AttendBegun item = a.begun[blockIdx.x];
    const int lane = threadIdx.x & 31, first = (blockIdx.y * JOIN_WARPS + (threadIdx.x >> 5)) * JOIN_ROWS;
    if (first >= item.rows) return;
    constexpr int EACH = DIM / 32, AHEAD = 4;  // columns of a lane, parts on their way together
    const int parts = item.others + 1, mine = lane / JOIN_PARTS, part = lane % JOIN_PARTS;
    const bool there = lane * EACH < a.cache.dim;
    const auto slot = [&](int i) { return (int64_t)(i == 0 ? 2 * (int)blockIdx.x + 1 : 2 * ((int)blockIdx.x + i)); };
    const auto load = [&](int i) {
        return i < parts && first + mine < item.rows ? __ldcg(&a.ml[slot(i) * a.rows + first + mine]) : make_float2(-INFINITY, 0.0f);
    };
    float2 x[AHEAD][JOIN_ROWS][EACH / 2];
    const auto fetch = [&](int i) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const float* from = a.part + (slot(min(i + k, parts - 1)) * a.rows + first) * DIM + lane * EACH;
#pragma unroll
            for (int j = 0; j < JOIN_ROWS; ++j)
#pragma unroll
                for (int e = 0; e < EACH; e += 2)
                    x[k][j][e / 2] = there && first + j < item.rows ? __ldcg((const float2*)(from + j * DIM + e)) : make_float2(0.0f, 0.0f);
        }
    };
    fetch(0);
    const float2 near = load(part), next = load(JOIN_PARTS + part);
    float most = fmaxf(near.x, next.x);
#pragma unroll 1
    for (int base = 2 * JOIN_PARTS; base < parts; base += JOIN_PARTS) most = fmaxf(most, load(base + part).x);
#pragma unroll
    for (int o = JOIN_PARTS / 2; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    float acc[JOIN_ROWS][EACH] = {}, norm = 0.0f, w = 0.0f;
#pragma unroll 1
    for (int i = 0; i < parts; i += AHEAD) {
        if (i % JOIN_PARTS == 0) {
            const float2 ml = i == 0 ? near : i == JOIN_PARTS ? next : load(i + part);
            w = ml.x == most ? 1.0f : exp2_unit(ml.x - most);
            norm += ml.y * w;
        }
        if (i > 0) fetch(i);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
#pragma unroll
            for (int j = 0; j < JOIN_ROWS; ++j) {
                const float f = __shfl_sync(0xffffffffu, w, j * JOIN_PARTS + (i + k) % JOIN_PARTS);
                if (i + k < parts)
#pragma unroll
                    for (int e = 0; e < EACH; e += 2) acc[j][e] += x[k][j][e / 2].x * f, acc[j][e + 1] += x[k][j][e / 2].y * f;
            }
    }
#pragma unroll
    for (int o = JOIN_PARTS / 2; o > 0; o >>= 1) norm += __shfl_xor_sync(0xffffffffu, norm, o);
    const float inv = norm == 0.0f ? 0.0f : 1.0f / norm;
#pragma unroll
    for (int j = 0; j < JOIN_ROWS; ++j) {
        const float f = __shfl_sync(0xffffffffu, inv, j * JOIN_PARTS);
        if (!there || first + j >= item.rows) continue;
        const int64_t row = item.row0 + first + j, token = attend_quotient(row, a.group);
        T* to = (T*)a.out + (item.first + token) * a.out_token + (item.head * a.group + (int)(row - token * a.group)) * a.out_head + lane * EACH;
#pragma unroll
        for (int e = 0; e < EACH; e += 2) *(uint32_t*)(to + e) = pack_two<T>(acc[j][e] * f, acc[j][e + 1] * f);
    }
}

// --- host ------------------------------------------------------------------------------------------------------------------------

struct AttendPlan {
    bool tc;
    int rows, dim, ctas;          // of a tile; padded; CTAs
    int64_t part, ml, begun, all;  // bytes up to each
    AttendPlan(const lda_paged_cache& cache, int64_t tokens, int32_t heads)
    {
        tc = attend_tc_takes(cache);
        dim = cache.dim <= 64 ? 64 : cache.dim <= 128 ? 128 : 256;
        // Those that a sequence has on average share what is read from shared memory.  Of 32 sequences of up to 4096 slots, all with as many rows, heads of
        // 128, in us: by 32 rows, 64 and 256 with 16 rows a sequence 75, 76, 89, with 24 82, 78, 93, with 40 140, 85, 96, with 96 235, 159, 116 (64 would
        // do up to 64 rows where all have as many; where some have more than the average, 256 read their keys once).  Without tensor memory, pages of 4: by 16,
        // 32 and 64 rows with 16 rows a sequence 95, 103, 121, with 20 170, 107, 124, with 40 248, 192, 125; heads of 256 by 16 and 32 with 16 154, 164, with
        // 20 276, 171.
        const int64_t most = (tokens + cache.n_seqs - 1) / cache.n_seqs * (heads / cache.kv_heads);
        if (tc) rows = most <= 16 ? 32 : most <= 32 ? 64 : 256;
        else rows = most <= 16 ? 16 : most <= 32 || dim == 256 ? 32 : 64;
        ctas = 148 * (tc || dim == 256 ? 1 : dim == 128 ? 2 : 3);
        part = 0;
        ml = (int64_t)2 * ctas * rows * dim * 4;
        begun = ml + (int64_t)2 * ctas * rows * 8;
        all = begun + (int64_t)ctas * sizeof(AttendBegun);
    }
};

template <typename T, int DIM, int ROWS>
static cudaError_t launch_attend(const AttendArgs& a, cudaStream_t st)
{
    using S = AttendShape<DIM, ROWS>;
    static std::atomic<bool> allowed[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !allowed[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(k_attend<T, DIM, ROWS>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SHARED);
        if (e != cudaSuccess) return e;
        if (dev < 64) allowed[dev].store(true, std::memory_order_release);
    }
    k_attend<T, DIM, ROWS><<<a.ctas, S::THREADS, S::SHARED, st>>>(a);
    return cudaGetLastError();
}

template <typename T, int DIM>
static cudaError_t attend_by_rows(const AttendArgs& a, const AttendPlan& plan, const lda_paged_cache& cache, cudaStream_t st)
{
    cudaError_t e;
    if (plan.tc) e = attend_tc(a, cache, st);
    else if (plan.rows == 16) e = launch_attend<T, DIM, 16>(a, st);
    else if (plan.rows == 32 || DIM == 256) e = launch_attend<T, DIM, 32>(a, st);
    else e = launch_attend<T, DIM, DIM == 256 ? 32 : 64>(a, st);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3((unsigned)a.ctas, (unsigned)(a.rows / (JOIN_WARPS * JOIN_ROWS)));
    c.blockDim = dim3(32 * JOIN_WARPS);
    c.stream = st;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    c.attrs = &at;
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, k_attend_join<T, DIM>, a);
}

template <typename T>
static cudaError_t attend_by_dim(const AttendArgs& a, const AttendPlan& plan, const lda_paged_cache& cache, cudaStream_t st)
{
    return plan.dim == 64    ? attend_by_rows<T, 64>(a, plan, cache, st)
           : plan.dim == 128 ? attend_by_rows<T, 128>(a, plan, cache, st)
                             : attend_by_rows<T, 256>(a, plan, cache, st);
}

static int attend_check(const lda_paged_cache* cache, int64_t tokens, int32_t heads, CacheView& view)
{
    const int rc = cache_view(cache, tokens, view);
    if (rc != LDA_OK) return rc;
    if (heads < 1 || heads % cache->kv_heads) return LDA_EINVAL;
    return heads > LDA_HEADS_MAX ? LDA_ERANGE : LDA_OK;
}

}  // namespace lda

extern "C" int64_t lda_tree_attention_workspace(const lda_paged_cache* cache, int64_t tokens, int32_t heads)
{
    using namespace lda;
    CacheView view;
    const int rc = attend_check(cache, tokens, heads, view);
    if (rc != LDA_OK) return rc;
    if (tokens == 0 || cache->n_seqs == 0) return 0;
    return AttendPlan(*cache, tokens, heads).all;
}

extern "C" int lda_tree_attention(const lda_paged_cache* cache, int64_t tokens, const void* q_dev, int64_t q_token_stride,
                                  int64_t q_head_stride, int32_t heads, const int64_t* mask_dev, int64_t mask_stride, int32_t mask_words,
                                  double scale, void* out_dev, int64_t out_token_stride, int64_t out_head_stride, void* workspace_dev,
                                  int64_t workspace_bytes, void* cuda_stream)
{
    using namespace lda;
    AttendArgs a{};
    const int rc = attend_check(cache, tokens, heads, a.cache);
    if (rc != LDA_OK) return rc;
    if (!(scale >= 1e-6 && scale <= 1e6)) return LDA_EINVAL;
    if (mask_dev && (mask_words < 1 || mask_stride < 0 || !aligned(mask_dev, 8))) return LDA_EINVAL;
    if (mask_dev && (mask_words > LDA_MASK_MAX_WORDS || mask_stride > (1ll << 31))) return LDA_ERANGE;
    if (tokens == 0 || cache->n_seqs == 0) return LDA_OK;
    if (!heads_ok(q_dev, q_token_stride, q_head_stride) || !heads_ok(out_dev, out_token_stride, out_head_stride)) return LDA_EINVAL;
    const int64_t most = 1ll << 31;
    if (q_token_stride > most || q_head_stride > most || out_token_stride > most || out_head_stride > most) return LDA_ERANGE;
    if (!heads_apart(q_dev, q_token_stride, q_head_stride, out_dev, out_token_stride, out_head_stride, tokens, heads, cache->dim)) return LDA_EINVAL;
    const AttendPlan plan(*cache, tokens, heads);
    if (!workspace_dev || !aligned(workspace_dev, 32) || workspace_bytes < plan.all) return LDA_EINVAL;
    a.ctas = plan.ctas, a.rows = plan.rows;
    a.q = q_dev, a.out = out_dev;
    a.q_token = q_token_stride, a.q_head = q_head_stride, a.out_token = out_token_stride, a.out_head = out_head_stride;
    a.mask = mask_dev, a.mask_stride = mask_stride, a.mask_words = mask_words;
    a.heads = heads, a.group = heads / cache->kv_heads;
    a.scale = (float)(scale * 1.4426950408889634);
    a.part = (float*)((char*)workspace_dev + plan.part);
    a.ml = (float2*)((char*)workspace_dev + plan.ml);
    a.begun = (AttendBegun*)((char*)workspace_dev + plan.begun);
    const cudaError_t e = cache->dtype == LDA_F16 ? attend_by_dim<__half>(a, plan, *cache, (cudaStream_t)cuda_stream)
                                                  : attend_by_dim<__nv_bfloat16>(a, plan, *cache, (cudaStream_t)cuda_stream);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return LDA_ECUDA;
    }
    return LDA_OK;
}
