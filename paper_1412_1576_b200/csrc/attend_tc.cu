// Attention over a paged cache on the tensor cores' own memory: heads of up to 128 values, pages of a multiple of 8 slots.
//
// A tile has 128 keys and 128 rows.  S = Q K^T and O += P V are matrix products of a tile, or of half its keys (PIECES), each issued by one thread
// of a warp of its own: K and V from shared memory, where tensor copies bring them page by page, S, P and O in tensor memory (P in S's place).
// There are two teams of four warps, each with an S and an O of its own; a thread has a row: it reads the row's scores, makes probabilities of
// them and writes these back, while the products of the other team run.
//   items of more than 128 rows  the teams have 128 rows each, and every tile of keys serves both
//   others                       the teams take the tiles of keys in turn, and the two O are added up at the item's end.  Of 64 or 32 rows
//                                (ROWS) every one stands in the tile twice or four times, and each of its copies has the probabilities of
//                                its own half or fourth of the keys (zeros for the others), so that all warps work.
// The products cost the same, 128 rows or 4: 1024 cycles of the tensor cores for a tile of 128 values a head, whose keys and values take 2800
// cycles to come from memory.
// Measured (bf16, heads of 128, 32 query heads on 8 of the cache; replayed graphs of five calls, a call being this kernel and the join):
//   64 sequences of up to 8192 slots, one token each   212 to 230 us on different cards, 5.8 to 6.3 TB/s (the copy's rate is 6.5): memory.  A long
//                                                      run of calls draws 1000 W and takes 229 to 252, at 1.5 to 1.6 GHz
//   16 sequences of up to 8192, trees of up to 64      127 to 130 us, 420 TFLOP/s: the warps that issue products and their waits (a piece of 64
//                                                      keys: 1200 cycles of its warp, 400 of the tensor cores), then starting up and the join
//   one sequence of 32 768, 8 tokens                   40 us: 20 of memory, 9 to the first tile's end, 8 the join
// With one warp for all products 44, 225 and 147 us; with one for each team's scores and outputs (four, 128 registers a thread) 48, 223 and
// 137; the scores of a tile in one piece 153 (trees); the matrix instructions of the other kernel (attend.cu) 51, 277 and 297.
#include <cuda.h>

#include "attend.cuh"

namespace lda {

constexpr int TC_KEYS = 128, TC_ROWS = 128;
constexpr int TC_TEAM = 128, TC_THREADS = 3 * TC_TEAM;  // two teams; two warps that issue products, two that copy
constexpr uint32_t TC_S = 0, TC_O = 256;                     // columns of tensor memory: S twice, O twice

template <int DIM, int ROWS>
struct TcShape {
    static constexpr bool PAIR = ROWS == 256;                    // the teams may have rows of their own
    static constexpr int HALVES = DIM / 64;                      // 128 bytes of every row at a time
    static constexpr int TILE = TC_KEYS * DIM * 2;               // bytes of keys, values or queries
    static constexpr int K_STAGES = DIM == 128 ? 2 : 4, V_STAGES = DIM == 128 ? (PAIR ? 2 : 3) : 4;  // (a tile's values are needed later and longer)
    static constexpr int RT = PAIR ? 128 : ROWS;                 // rows of a team
    static constexpr int GROUPS = TC_ROWS / RT;                  // of keys
    // A tile's scores come and its probabilities go in one piece, or (PAIR) in two of 64 keys, so that a team has one to work on while the products
    // of its other one run.  A piece's probabilities stand in the second half of its scores' columns.
    static constexpr int PIECES = PAIR ? 2 : 1, PIECE = TC_KEYS / PIECES;
    static constexpr int COLS = PAIR ? 64 : ROWS;                // of a piece that a thread looks at
    static constexpr int TOGETHER = 16 / GROUPS, PITCH = DIM + 4;  // rows whose parts are added up at a time
    static constexpr int K_AT = 0, V_AT = K_STAGES * TILE, Q_AT = V_AT + V_STAGES * TILE, REGION_AT = Q_AT + (PAIR ? 2 : 1) * TILE;
    static constexpr int SHARED = REGION_AT + 2 * GROUPS * TOGETHER * PITCH * 4 + 1024;  // (its start is moved up to a multiple of 1024)
};

struct TcBars {
    uint64_t k_full[4], k_empty[4], v_full[4], v_empty[4], s_full[4], p_full[4], o_done[4], q_full, q_empty, cleaned[2], last[2];  // (S, P and O: of a team's piece)
};

__device__ __forceinline__ uint32_t tc_smem(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void tc_init(uint64_t& bar, uint32_t arrivals)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(tc_smem(&bar)), "r"(arrivals) : "memory");
}
__device__ __forceinline__ void tc_arrive(uint64_t& bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(tc_smem(&bar)) : "memory"); }
__device__ __forceinline__ void tc_expect(uint64_t& bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(tc_smem(&bar)), "r"(bytes) : "memory");
}
// Waits for a phase.  Every wait here ends by itself, within microseconds; one that has not after so many polls (how long the hardware holds each
// of them is its own affair) gives up and tells the others, which then do not wait any more, and the rows concerned become NaN.  A build with 0 polls
// shows that: every wait gives up at once.
#ifndef LDA_WAIT_POLLS
#define LDA_WAIT_POLLS (1 << 22)
#endif
constexpr int TC_POLLS = LDA_WAIT_POLLS, TC_POLLS_LAST = 1 << 22;  // (of what is under way at the end, in any build)
__device__ __forceinline__ bool tc_wait(uint64_t& bar, uint32_t parity, volatile int* failed, int polls = TC_POLLS)
{
    const uint32_t at = tc_smem(&bar);
    for (int i = 0; i < polls; ++i) {
        uint32_t done;
        asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                     : "=r"(done)
                     : "r"(at), "r"(parity)
                     : "memory");
        if (done) return true;
        if (*failed) return false;
    }
    *failed = 1;
    return false;
}
// Arrives, and waits for all others of the phase.  A barrier that the threads of a team meet at wherever they are, and unlike bar.sync none that
// hangs where a wait before it gave up in some of them only.  (The phase goes by what the arrival returns: a count of phases is one register
// more in loops that have none left, 8 us of the trees' 127.)
__device__ __forceinline__ void tc_meet(uint64_t& bar, volatile int* failed)
{
    const uint32_t at = tc_smem(&bar);
    uint64_t phase;
    asm volatile("mbarrier.arrive.shared::cta.b64 %0, [%1];" : "=l"(phase) : "r"(at) : "memory");
    for (int i = 0; i < TC_POLLS; ++i) {
        uint32_t done;
        asm volatile("{ .reg .pred p; mbarrier.try_wait.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }" : "=r"(done) : "r"(at), "l"(phase) : "memory");
        if (done || *failed) break;
        if (i + 1 == TC_POLLS) *failed = 1;
    }
}
// What a product reads or has written, seen by the other side of a barrier.
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint64_t& bar, bool leads)
{
    asm volatile("{ .reg .pred q; setp.ne.u32 q, %1, 0; @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0]; }" ::"r"(tc_smem(&bar)),
                 "r"((uint32_t)leads)
                 : "memory");
}
// An operand in shared memory, rows of 128 bytes swizzled among eight, in units of 16 bytes: its place, and what is the same for all places.
// `across`: bytes from one group of 64 elements to the next where the contiguous dimension is not the one that is summed over.
__device__ __forceinline__ uint32_t tc_operand_at(uint32_t at) { return at >> 4; }
__device__ __forceinline__ constexpr uint32_t tc_operand_low(uint32_t across) { return across >> 4 << 16; }
constexpr uint32_t TC_OPERAND_HIGH = 1024 >> 4 | 1u << 14 | 2u << 29;
// Types (fp16 0, bf16 1; sums of single precision), whether B is contiguous in the columns, columns; 128 rows.
__device__ __forceinline__ constexpr uint32_t tc_kind(bool bf16, bool turned, uint32_t columns)
{
    return 1u << 4 | (uint32_t)bf16 << 7 | (uint32_t)bf16 << 10 | (uint32_t)turned << 16 | columns / 8 << 17 | (uint32_t)(TC_ROWS / 16) << 24;
}
// By a whole warp, of which the lane `leads` issues: what the product needs is the same in all lanes then, and stays in uniform registers.
__device__ __forceinline__ void tc_product_shared(uint32_t d, uint32_t a, uint32_t b, uint32_t kind, bool add, bool leads)
{
    asm volatile("{ .reg .pred p, q; .reg .b64 x, y; setp.ne.u32 p, %5, 0; setp.ne.u32 q, %6, 0; mov.b64 x, {%1, %4}; mov.b64 y, {%2, %4}; "
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p; }" ::"r"(d),
                 "r"(a), "r"(b), "r"(kind), "r"(TC_OPERAND_HIGH), "r"((uint32_t)add), "r"((uint32_t)leads)
                 : "memory");
}
__device__ __forceinline__ void tc_product_tensor(uint32_t d, uint32_t a, uint32_t b, uint32_t kind, bool add, bool leads)
{
    asm volatile("{ .reg .pred p, q; .reg .b64 y; setp.ne.u32 p, %5, 0; setp.ne.u32 q, %6, 0; mov.b64 y, {%2, %4}; "
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p; }" ::"r"(d),
                 "r"(a), "r"(b), "r"(kind), "r"(TC_OPERAND_HIGH), "r"((uint32_t)add), "r"((uint32_t)leads)
                 : "memory");
}
// 32 columns of a thread's row of tensor memory.
__device__ __forceinline__ void tc_load(uint32_t (&r)[32], uint32_t at)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
                 "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
                   "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
                   "=r"(r[31])
                 : "r"(at));
}
// The registers of a load may be looked at behind this only.
__device__ __forceinline__ void tc_loaded(uint32_t (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]),
                   "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]),
                   "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]),
                   "+r"(r[31])::"memory");
}
__device__ __forceinline__ void tc_loaded(uint32_t (&r)[8])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7])::"memory");
}
__device__ __forceinline__ void tc_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_store(uint32_t at, const uint32_t (&r)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
                 "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(at),
                 "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                 "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
                 "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
                 : "memory");
}
__device__ __forceinline__ void tc_store(uint32_t at, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(at),
                 "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                 "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
__device__ __forceinline__ void tc_load(uint32_t (&r)[8], uint32_t at)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(at));
}
__device__ __forceinline__ void tc_store(uint32_t at, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
// 64 columns of `rows` slots of a page's head; every coordinate is inside the cache, the first one a multiple of 64.
__device__ __forceinline__ void tc_copy(uint32_t to, const CUtensorMap* map, int column, int slot, int head, int page, uint64_t& bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(to),
                 "l"(map), "r"(column), "r"(slot), "r"(head), "r"(page), "r"(tc_smem(&bar))
                 : "memory");
}
__device__ __forceinline__ void tc_rows_sync() { asm volatile("bar.sync 3, 256;" ::: "memory"); }
__device__ __forceinline__ uint4 tc_shared16(uint32_t at)
{
    uint4 x;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at) : "memory");
    return x;
}
__device__ __forceinline__ void tc_put16(uint32_t at, uint4 x)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
}

struct TcMaps {
    CUtensorMap k, v;
    int32_t group_bits;  // 2^group_bits slots come in a copy: a power of two that divides a page, 8 to 128
};

// How far a row's largest exponent may rise above what its probabilities are relative to before its sums are moved: they need no more
// digits up to there (2^8 times the probability, fp16 2^15), and most rows never do it after their first tile.
constexpr float TC_SLACK = 8.0f;
template <typename T>
constexpr float TC_RAISE = T_is_bf16<T> ? 0.0f : 7.0f;

// Of four columns of a row's sums, what is NaN although the row's norm is a number: what the infinities and NaN among the values of the keys of
// `count` tiles that the row sees make of it.  An infinity that all rows see stays in its tile, and times the zeros that a row's copies have for
// each other's keys it is NaN.  (A function of its own: a call that needs it is rare, and the others do not fetch its code.)
template <typename T>
__device__ __noinline__ float4 tc_wild(const AttendArgs& a, float4 of, int b, int head, int64_t row0, int row, int tile, int count, int keys, int column)
{
    const CacheView& c = a.cache;
    const CacheSeq seq = c.seq(b);
    const int place = (int)attend_quotient(row0 + row, a.group);
    const int64_t first = (int64_t)tile * TC_KEYS, end = min((int64_t)(tile + count) * TC_KEYS, (int64_t)keys);
#pragma unroll 1
    for (int i = 0; i < 4; ++i) {
        float& x = i == 0 ? of.x : i == 1 ? of.y : i == 2 ? of.z : of.w;
        if (!isnan(x)) continue;
        const T* values = (const T*)c.values + head * c.v_head + column + i;
        float sum = 0.0f;
        unsigned long long see = 0;
#pragma unroll 1
        for (int64_t key = first; key < end && sum == sum; key += 8) {  // (eight slots of a page at a time)
            if (key % 64 == 0) see = attend_window(a, seq, place, (int)(key / 64));
            uint32_t bits = (uint32_t)(see >> (key % 64)) & 0xFFu;
            if (end - key < 8) bits &= (1u << (end - key)) - 1;
            int slot = 0;
            const int64_t page = bits ? c.page(b, (uint32_t)key, slot) : -1;
            if (page < 0) continue;
            const T* from = values + page * c.v_page + slot * c.v_slot;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = bits >> e & 1 ? cache_value(from[e * c.v_slot]) : 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (!(fabsf(v[e]) < INFINITY)) sum += v[e];
        }
        if (sum != 0.0f) x = sum;
    }
    return of;
}

// A copying warp's walk over its CTA's units, for keys or for values: a lane has one of the tile's groups of slots.
template <int DIM, int ROWS, int STAGES>
__device__ __forceinline__ void tc_copies(const AttendArgs& a, const CUtensorMap* map, int bits, AttendItem item, int64_t units, uint32_t to,
                                          uint64_t* full, uint64_t* empty, uint32_t* valid, unsigned long long (*wild)[2], volatile int* failed)
{
    const int lane = threadIdx.x & 31, groups = TC_KEYS >> bits;
    int page = -1, place = 0;
    const auto look = [&] {
        const int key = item.tile * TC_KEYS + (lane << bits);
        page = lane < groups && key < item.keys ? a.cache.page(item.b, (uint32_t)key, place) : -1;
    };
    look();
    int it = 0;
#pragma unroll 1
    for (; units > 0; ++it) {
        const int p = page, at = place, head = item.head, s = it % STAGES;
        const uint32_t there = __ballot_sync(0xffffffffu, p >= 0);
        const bool ok = tc_wait(empty[s], it / STAGES & 1 ^ 1, failed);
        if (__any_sync(0xffffffffu, !ok)) break;
        if (lane == 0) {
            if (valid) valid[it & 15] = there;
            if (wild) wild[s][0] = wild[s][1] = 0;
            tc_expect(full[s], (__popc(there) << bits) * DIM * 2);
        }
        __syncwarp();
        if (p >= 0)
#pragma unroll
            for (int h = 0; h < DIM / 64; ++h)
                tc_copy(to + s * (TC_KEYS * DIM * 2) + h * (TC_KEYS * 128) + (lane << bits) * 128, map, 64 * h, at, head, p, full[s]);
        units -= item.tile + 1 == item.tiles ? item.weight + item.extra_units() : item.weight;
        if (units > 0) {
            item.template next<ROWS, TC_KEYS>(a);
            look();
        }
    }
    if (units > 0) {  // gave up: what is under way still lands
        int quit = 0;
        for (int i = max(0, it - STAGES); i < it; ++i) tc_wait(full[i % STAGES], i / STAGES & 1, (volatile int*)&quit, TC_POLLS_LAST);
    }
}

template <typename T, int DIM, int ROWS>
__global__ void __launch_bounds__(TC_THREADS, 1) k_attend_tc(const __grid_constant__ AttendArgs a, const __grid_constant__ TcMaps maps)
{
    using S = TcShape<DIM, ROWS>;
    constexpr bool PAIR = S::PAIR;
    constexpr int GROUPS = S::GROUPS, COLS = S::COLS, RT = S::RT, PIECES = S::PIECES, PIECE = S::PIECE;
    extern __shared__ uint8_t dynamic[];
    __shared__ TcBars bars;
    __shared__ unsigned long long red[TC_THREADS / 32], wild[4][2];  // (wild: of a stage's keys, those whose values are not all finite)
    __shared__ uint32_t s_tmem, valid[16];
    __shared__ int s_failed;
    __shared__ float s_m[2 * TC_ROWS], s_l[2 * TC_ROWS];
    const uint32_t base = (tc_smem(dynamic) + 1023) & ~1023u;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const CacheView& c = a.cache;
    volatile int* failed = &s_failed;
    if (tid == 0) {
        for (int i = 0; i < 4; ++i) tc_init(bars.k_full[i], 1), tc_init(bars.k_empty[i], 1), tc_init(bars.v_full[i], 1), tc_init(bars.v_empty[i], 1);
        for (int i = 0; i < 4; ++i) tc_init(bars.s_full[i], 1), tc_init(bars.p_full[i], TC_TEAM), tc_init(bars.o_done[i], 1);
        tc_init(bars.q_full, 2 * TC_TEAM), tc_init(bars.q_empty, 1);
        for (int i = 0; i < 2; ++i) tc_init(bars.cleaned[i], TC_TEAM), tc_init(bars.last[i], 1);
        s_failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    AttendShare share;
    AttendItem item;
    AttendBegun begun{};
    if (!attend_share<ROWS, TC_KEYS>(a, blockIdx.x, share, item, red)) {
        if (tid == 0) a.begun[blockIdx.x] = begun;
        return;
    }
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(tc_smem(&s_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        tc_before();
    }
    __syncthreads();
    tc_after();
    const uint32_t tmem = s_tmem;
    const int64_t units = share.hi - share.lo;
    // whether the teams have rows of their own of an item
    const auto splits = [&](const AttendItem& of) { return PAIR && of.weight == 2; };

    if (warp >= 8) {
        if (warp == 9) {
            tc_copies<DIM, ROWS, S::K_STAGES>(a, &maps.k, maps.group_bits, item, units, base + S::K_AT, bars.k_full, bars.k_empty, valid, nullptr,
                                                  failed);
        } else if (warp == 10) {
            tc_copies<DIM, ROWS, S::V_STAGES>(a, &maps.v, maps.group_bits, item, units, base + S::V_AT, bars.v_full, bars.v_empty, nullptr, wild,
                                                  failed);
        } else {
            // --- products, a piece's for a team at a time (a job): one warp issues those of the scores, as soon as the outputs of the job before
            // in the same place are done, another those of the outputs (one alone is the slowest part of a tile: an issue takes it as long
            // as the tensor cores take for the product)
            constexpr uint32_t KIND_S = tc_kind(T_is_bf16<T>, false, PIECE), KIND_O = tc_kind(T_is_bf16<T>, true, DIM);
            constexpr uint32_t JOB_PIECE = 1, JOB_TEAM = 2, JOB_FIRST = 4, JOB_LAST = 8, JOB_FRESH = 16, JOB_STEPS = 32;  // (first, last: of its tile)
            const bool leads = lane == 0;
            const uint32_t at = __shfl_sync(0xffffffffu, base, 0), tensor = __shfl_sync(0xffffffffu, tmem, 0);
            bool go = leads;  // (products and barriers are this lane's; none where a wait gave up)
            const auto wait = [&](uint64_t& bar, uint32_t parity) { go = tc_wait(bar, parity, failed) && go; };
            uint32_t stage = 0, round = 0, rounds = 0, q_round = 0;  // of keys or values, and parities of the next phases
            const uint32_t q_operand = tc_operand_low(16) + tc_operand_at(at + S::Q_AT), k_operand = tc_operand_low(16) + tc_operand_at(at + S::K_AT),
                           v_operand = tc_operand_low(TC_KEYS * 128) + tc_operand_at(at + S::V_AT);
            const auto scores = [&](uint32_t job) {
                const uint32_t piece = job & 1, team = job >> 1 & 1, place = team * PIECES + piece;
                if (job & JOB_FIRST) wait(bars.k_full[stage], round);
                wait(bars.o_done[place], rounds >> place & 1 ^ 1);
                rounds ^= 1u << place;
                tc_after();
                const uint32_t q = q_operand + (PAIR ? team * (S::TILE / 16) : 0), k = k_operand + stage * (S::TILE / 16) + piece * (PIECE * 128 / 16),
                               to = tensor + TC_S + team * TC_KEYS + piece * PIECE;
#pragma unroll
                for (int i = 0; i < DIM / 16; ++i) {
                    const uint32_t step = (i / 4 * (TC_KEYS * 128) + i % 4 * 32) / 16;
                    tc_product_shared(to, q + step, k + step, KIND_S, i > 0, go);
                }
                tc_commit(bars.s_full[place], go);
                if (!(job & JOB_LAST)) return;
                tc_commit(bars.k_empty[stage], go);
                if (++stage == S::K_STAGES) stage = 0, round ^= 1;
            };
            const auto outputs = [&](uint32_t job) {
                const uint32_t piece = job & 1, team = job >> 1 & 1, place = team * PIECES + piece;
                const int steps = (int)(job / JOB_STEPS);
                if (job & JOB_FIRST) wait(bars.v_full[stage], round);
                wait(bars.p_full[place], rounds >> place & 1);
                rounds ^= 1u << place;
                tc_after();
                const uint32_t v = v_operand + stage * (S::TILE / 16) + piece * (PIECE * 128 / 16),
                               from = tensor + TC_S + team * TC_KEYS + piece * PIECE + PIECE / 2, to = tensor + TC_O + team * 128;
                if (steps == PIECE / 16) {
#pragma unroll
                    for (int i = 0; i < PIECE / 16; ++i) tc_product_tensor(to, from + 8 * i, v + i * (2048 / 16), KIND_O, i > 0 || !(job & JOB_FRESH), go);
                } else
#pragma unroll 1
                    for (int i = 0; i < steps; ++i) tc_product_tensor(to, from + 8 * i, v + i * (2048 / 16), KIND_O, i > 0 || !(job & JOB_FRESH), go);
                tc_commit(bars.o_done[place], go);
                if (!(job & JOB_LAST)) return;
                tc_commit(bars.v_empty[stage], go);
                if (++stage == S::V_STAGES) stage = 0, round ^= 1;
            };
            int64_t unit = share.lo;
            uint32_t turn = 0;  // the team of the next tile that one team has
            while (true) {
                const int tiles = __shfl_sync(0xffffffffu, (int)min((int64_t)(item.tiles - item.tile), (share.hi - unit) >> (item.weight - 1)), 0);
                const bool split = __any_sync(0xffffffffu, splits(item)), ends = __any_sync(0xffffffffu, item.tile + tiles == item.tiles);
                // of the item's last tile the sixteens of keys that there are
                const int last_steps = ends ? __shfl_sync(0xffffffffu, max(1, (item.keys - (item.tiles - 1) * TC_KEYS + 15) / 16), 0) : TC_KEYS / 16;
                if (warp == 8) {
                    wait(bars.q_full, q_round);
                    q_round ^= 1;
                }
#pragma unroll 1
                for (int i = 0; i < tiles; ++i) {
                    const int steps = i + 1 < tiles ? TC_KEYS / 16 : last_steps, n = split ? 2 * PIECES : PIECES;
                    const bool fresh = i < (split ? 1 : 2);
#pragma unroll 1
                    for (int x = 0; x < n; ++x) {
                        const int piece = split ? x >> 1 : x, here = min(PIECE / 16, max(0, steps - piece * (PIECE / 16)));
                        const uint32_t job = piece * JOB_PIECE | (split ? x & 1 : turn) * JOB_TEAM | (x == 0) * JOB_FIRST | (x + 1 == n) * JOB_LAST |
                                             (fresh && piece == 0) * JOB_FRESH | here * JOB_STEPS;
                        if (warp == 8) scores(job);
                        else outputs(job);
                    }
                    turn ^= 1;
                }
                if (ends && warp == 8) tc_commit(bars.q_empty, go);
                unit += (int64_t)tiles * item.weight + (ends ? item.extra_units() : 0);
                if (!__any_sync(0xffffffffu, unit < share.hi)) break;
                item.tile = item.tiles - 1;
                item.template next<ROWS, TC_KEYS>(a);
            }
        }
        __syncwarp();
    } else {
        // --- rows (they go on where a wait gave up, so that all of them meet at an item's end; outputs are NaN then)
        const int team = warp >> 2, kg = tid % TC_TEAM / RT;
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
        const uint32_t at_s = tmem + lanes + TC_S + team * TC_KEYS, at_o = tmem + lanes + TC_O + team * 128;
        const uint32_t at_q = base + S::Q_AT + (PAIR ? team * S::TILE : 0) + tid % TC_TEAM * 128;
        // a thread's row of an item
        const auto row_of = [&](const AttendItem& of) { return splits(of) ? tid : tid % RT; };
        // a row's queries, once for each of its copies, a half by each team (PAIR: each team has a place for its own); an item's first are put down
        // where the last one's have been read, which `ready` waits for
        constexpr int Q_EACH = DIM / 16;
        const auto put_q = [&](const AttendItem& of, auto ready) {
            const int64_t row = (int64_t)of.row_tile * ROWS + row_of(of);
            const bool there = row < (int64_t)of.seq.n * a.group;
            const int token = there ? (int)attend_quotient(row, a.group) : 0, h = there ? (int)(row - (int64_t)token * a.group) : 0;
            const T* from = (const T*)a.q + (of.seq.first + token) * a.q_token + (of.head * a.group + h) * a.q_head;
#pragma unroll 1
            for (int half = PAIR ? 0 : team; half < (PAIR ? 2 : team + 1); ++half) {
                uint4 q[Q_EACH];
#pragma unroll
                for (int i = 0; i < Q_EACH; ++i) {
                    const int ch = half * Q_EACH + i;
                    q[i] = there && ch * 8 < c.dim ? __ldg((const uint4*)(from + ch * 8)) : make_uint4(0, 0, 0, 0);
                }
                if (!PAIR || half == 0) ready();
#pragma unroll
                for (int i = 0; i < Q_EACH; ++i) {
                    const int ch = half * Q_EACH + i;
                    tc_put16(at_q + ch / 8 * (TC_KEYS * 128) + ((ch % 8 ^ tid % 8) << 4), q[i]);
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            tc_arrive(bars.q_full);
        };
        put_q(item, [] {});
        int it = 0;
        int64_t unit = share.lo;
        uint32_t n_s = 0, n_q = 0;  // pieces of the team, queries put down
        // barrier and parity of a piece of the team by its number
        const auto place_of = [&](uint32_t n) { return team * PIECES + (PIECES == 2 ? n & 1 : 0); };
        const auto phase_of = [&](uint32_t n) { return (PIECES == 2 ? n >> 1 : n) & 1; };
#pragma unroll 1
        while (unit < share.hi) {
            const int count = (int)min((int64_t)(item.tiles - item.tile), (share.hi - unit) >> (item.weight - 1)), end = it + count;
            const bool ends = item.tile + count == item.tiles, split = splits(item);
            const int64_t unit_after = unit + (int64_t)count * item.weight + (ends ? item.extra_units() : 0);
            const bool last = unit_after == share.hi;
            const int r = row_of(item);
            const int64_t item_begin = unit - (int64_t)item.tile * item.weight, row0 = (int64_t)item.row_tile * ROWS, all_rows = (int64_t)item.seq.n * a.group - row0;
            const int rows = (int)min((int64_t)ROWS, all_rows), place = r < rows ? (int)attend_quotient(row0 + r, a.group) : -1;
            float m = -INFINITY, l = 0.0f;
            bool any = false;
#pragma unroll 1
            for (int u = split ? it : it + ((it ^ team) & 1); u < end; u += split ? 1 : 2) {
                const int tile = item.tile + u - it;
                tc_wait(bars.s_full[place_of(n_s)], phase_of(n_s), failed);
                tc_after();
                const uint32_t there = *(volatile uint32_t*)&valid[u & 15];
                // the tile's keys, and whether all their pages have come
                const int keys = min(TC_KEYS, item.keys - tile * TC_KEYS), groups = (keys + (1 << maps.group_bits) - 1) >> maps.group_bits;
                const bool full = there == (uint32_t)((1ull << groups) - 1);
                unsigned long long bad[2] = {0, 0}, see[2] = {~0ull, ~0ull};
                const bool masked = !full || tile * TC_KEYS + keys > item.seq.start || keys < TC_KEYS;
                if (masked) {
                    // what the row sees of the keys (in loops that stay loops: this runs once or twice in a call)
#pragma unroll 1
                    for (int i = 0; i < 2; ++i) {
                        const int left = keys - 64 * i;
                        unsigned long long w = place < 0 || left <= 0 ? 0ull : attend_window(a, item.seq, place, 2 * tile + i);
                        if (left < 64 && left > 0) w &= (1ull << left) - 1;
                        if (!full)
#pragma unroll 1
                            for (int g = 0; g < 64; g += 8)
                                if (!(there >> ((64 * i + g) >> maps.group_bits) & 1)) w &= ~(0xFFull << g);
                        if (i == 0) see[0] = w;
                        else see[1] = w;
                    }
                    // a value that a row does not see must not touch it, whatever it is: infinities and NaN are taken out and added apart, and
                    // what stands where no key is, up to the last sixteen that the product takes, becomes zero
                    const int vs = u % S::V_STAGES;
                    tc_wait(bars.v_full[vs], u / S::V_STAGES & 1, failed);
                    const int from = full ? max(0, min(keys, item.seq.start - tile * TC_KEYS)) : 0, to = max(16, (keys + 15) & ~15);
#pragma unroll 1
                    for (int key = from + tid % TC_TEAM / 8; key < to; key += TC_TEAM / 8) {
                        const bool known = key < keys && (there >> (key >> maps.group_bits) & 1);
#pragma unroll
                        for (int h = 0; h < S::HALVES; ++h) {
                            const uint32_t at = base + S::V_AT + vs * S::TILE + (h * TC_KEYS + key) * 128 + tid % 8 * 16;
                            uint4 g = make_uint4(0, 0, 0, 0);
                            if (known) {
                                g = tc_shared16(at);
                                if (!has_wild<T>(g)) continue;
                                g = without_wild<T>(g);
                                // (said before it is taken out: where the teams have the same tile, both look)
                                atomicOr(&wild[vs][key / 64], 1ull << (key & 63));
                                __threadfence_block();
                            }
                            tc_put16(at, g);
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    tc_meet(bars.cleaned[team], failed);
                    // (the same in the warp, also where a wait gave up)
                    for (int i = 0; i < 2; ++i) bad[i] = __shfl_sync(0xffffffffu, *(volatile unsigned long long*)&wild[vs][i], 0);
                }
#pragma unroll 1
                for (int piece = 0; piece < PIECES; ++piece) {
                if (piece > 0) {
                    tc_wait(bars.s_full[place_of(n_s)], phase_of(n_s), failed);
                    tc_after();
                }
                const uint32_t at_piece = at_s + piece * PIECE;
                // the scores come 32 columns at a time; the probabilities go behind them, from the last to the first: over scores that have
                // been read
                constexpr int CHUNKS = COLS / 32;
                uint32_t even[32], odd[32];
                const auto fetch = [&](uint32_t (&s)[32], int chunk) { tc_load(s, at_piece + kg * COLS + 32 * chunk); };
                const auto hide = [&](uint32_t (&s)[32], int chunk) {
                    if (!masked) return;
                    const int k = piece * PIECE + kg * COLS + 32 * chunk;
                    const uint32_t w = (uint32_t)((k & 64 ? see[1] : see[0]) >> (k & 32));
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (!(w >> j & 1)) s[j] = 0xFF800000u;  // minus infinity
                };
                float top = -INFINITY;
                const auto largest = [&](const uint32_t (&s)[32]) {
                    float x[4] = {top, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int j = 0; j < 32; j += 8)
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[i] = fmaxf(x[i], fmaxf(__uint_as_float(s[j + 2 * i]), __uint_as_float(s[j + 2 * i + 1])));
                    top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
                };
                fetch(even, 0);
#pragma unroll
                for (int chunk = 0; chunk < CHUNKS; ++chunk) {
                    if (chunk & 1) tc_loaded(odd);
                    else tc_loaded(even);
                    if (chunk + 1 < CHUNKS) {
                        if (chunk & 1) fetch(even, chunk + 1);
                        else fetch(odd, chunk + 1);
                    }
                    if (chunk & 1) hide(odd, chunk), largest(odd);
                    else hide(even, chunk), largest(even);
                }
                top *= a.scale;
                // (minus infinity is no reason; the first number is)
                const bool raise = top > (m == -INFINITY ? -INFINITY : m + TC_SLACK);
                if (__any_sync(0xffffffffu, raise)) {
                    const float to = fmaxf(m, top), f = to == m ? 1.0f : exp2_unit(m - to);
                    m = to;
                    l *= f;
                    if (any) {  // (O holds something)
                        tc_wait(bars.o_done[place_of(n_s - 1)], phase_of(n_s - 1), failed);
                        tc_after();
#pragma unroll 1
                        for (int d = 0; d < DIM; d += 32) {
                            uint32_t o[32];
                            tc_load(o, at_o + d);
                            tc_loaded(o);
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                            tc_store(at_o + d, o);
                        }
                    }
                }
                // (places of no row have no probabilities: products with zeros take less power, and a long call is bound by that)
                const float shift = place < 0 ? -INFINITY : (m == -INFINITY ? 0.0f : -m) + TC_RAISE<T>;
                // the probabilities are rounded to the values' type, which the product takes: half a step each, as much as the output's own
                // rounding; the norm is that of the unrounded ones
                float2 sum = make_float2(0.0f, 0.0f);
                const auto put = [&](const uint32_t (&s)[32], int chunk) {
                    uint32_t p[16];
                    const float2 by = make_float2(a.scale, a.scale), plus = make_float2(shift, shift);
#pragma unroll
                    for (int j = 0; j < 32; j += 2) {
                        const float2 y = fma_two(make_float2(__uint_as_float(s[j]), __uint_as_float(s[j + 1])), by, plus);
                        const float2 x = make_float2(exp2_unit(y.x), exp2_unit(y.y));
                        sum = add_two(sum, x);
                        p[j / 2] = pack_two<T>(x.x, x.y);
                    }
                    tc_store(at_piece + PIECE / 2 + (kg * COLS + 32 * chunk) / 2, p);
                };
                if constexpr (CHUNKS == 2) put(odd, 1);
                put(even, 0);
                if (GROUPS > 1) {
                    const uint32_t zero[16] = {};
#pragma unroll
                    for (int g = 1; g < GROUPS; ++g)
#pragma unroll
                        for (int from = 0; from < COLS; from += 32) tc_store(at_piece + PIECE / 2 + (((kg + g) % GROUPS) * COLS + from) / 2, zero);
                }
                l += sum.x + sum.y;
                tc_stored();
                tc_before();
                tc_arrive(bars.p_full[place_of(n_s)]);
                any = true;
                // (what was taken out: a row that sees it has it, whatever the probability, which cannot be read any more: the outputs being done, the
                // next scores may stand in its place)
                if (bad[0] | bad[1]) {
                    tc_wait(bars.o_done[place_of(n_s)], phase_of(n_s), failed);
                    tc_after();
#pragma unroll 1
                    for (int i = 0; i < COLS; ++i) {
                        const int k = piece * PIECE + kg * COLS + i;
                        if (!((k < 64 ? bad[0] : bad[1]) >> (k & 63) & 1)) continue;  // (the same in the warp)
                        const bool sees = (k < 64 ? see[0] : see[1]) >> (k & 63) & 1;
                        int slot = 0;
                        const int64_t pg = c.page(item.b, (uint32_t)(tile * TC_KEYS + k), slot);
                        const T* v = (const T*)c.values + pg * c.v_page + slot * c.v_slot + item.head * c.v_head;
#pragma unroll 1
                        for (int d = 0; d < c.dim && pg >= 0; d += 8) {
                            float x[8];
                            unpack<T>(*(const uint4*)(v + d), x);
                            uint32_t o[8];
                            tc_load(o, at_o + d);
                            tc_loaded(o);
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (sees && !(fabsf(x[e]) < INFINITY)) o[e] = __float_as_uint(__uint_as_float(o[e]) + x[e]);
                            tc_store(at_o + d, o);
                            tc_stored();
                        }
                    }
                    tc_before();
                }
                ++n_s;
                }
            }
            // --- the item's end, or the share's: the next item's queries, then the sums out or to the parts
            AttendItem after = item;
            if (!last) {
                after.tile = after.tiles - 1;
                after.template next<ROWS, TC_KEYS>(a);
                put_q(after, [&] { tc_wait(bars.q_empty, n_q++ & 1, failed); });
            }
            if (any) tc_wait(bars.o_done[place_of(n_s - 1)], phase_of(n_s - 1), failed);
            tc_after();
            if (*failed) l = NAN;  // (and with the norm all of the row, here or where the parts are put together)
            const bool whole = ends && item_begin >= share.lo;
            const int slot = 2 * blockIdx.x + (item_begin < share.lo ? 0 : 1);
            const auto out_at = [&](int row) {
                const int64_t token = attend_quotient(row0 + row, a.group);
                const int h = (int)(row0 + row - token * a.group);
                return (T*)a.out + (item.seq.first + token) * a.out_token + (item.head * a.group + h) * a.out_head;
            };
            if (split) {
                const float f = !whole ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;  // (a row that sees nothing is zero)
                if (!whole) a.ml[(int64_t)slot * ROWS + r] = make_float2(m, l);
                T* to = r < rows ? out_at(r) : nullptr;
                float* part = a.part + ((int64_t)slot * ROWS + r) * DIM;
#pragma unroll 1
                for (int d = 0; d < c.dim; d += 32) {
                    uint32_t o[32];
                    tc_load(o, at_o + d);
                    tc_loaded(o);
#pragma unroll
                    for (int i = 0; i < 32; i += 8)
                        if (r < rows && d + i < c.dim) {
                            float x[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(o[i + e]) * f;
                            if (whole) *(uint4*)(to + d + i) = pack<T>(x);
                            else  // (32 bytes at a time: a thread's row lies by itself)
                                asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(part + d + i), "f"(x[0]), "f"(x[1]), "f"(x[2]),
                                             "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7])
                                             : "memory");
                        }
                    __syncwarp();
                }
            } else {
                // the teams' and key groups' parts: of a few rows at a time, or, behind the CTA's last unit, of all of them, where its keys and
                // values were
                constexpr int ALL = RT < (S::K_STAGES + S::V_STAGES + (PAIR ? 2 : 1)) * S::TILE / (2 * GROUPS * S::PITCH * 4)
                                        ? RT
                                        : (S::K_STAGES + S::V_STAGES + (PAIR ? 2 : 1)) * S::TILE / (2 * GROUPS * S::PITCH * 4);
                const int together = last ? ALL : S::TOGETHER;
                s_m[tid] = m, s_l[tid] = l;
                tc_rows_sync();
                float most = -INFINITY, norm = 0.0f;
#pragma unroll
                for (int g = 0; g < 2 * GROUPS; ++g) most = fmaxf(most, s_m[g * RT + r]);
#pragma unroll
                for (int g = 0; g < 2 * GROUPS; ++g) {
                    const float x = s_m[g * RT + r];
                    norm += x == most ? s_l[g * RT + r] : s_l[g * RT + r] * exp2_unit(x - most);
                }
                float f = m == most ? 1.0f : exp2_unit(m - most);
                if (whole) f = norm == 0.0f ? 0.0f : f / norm;  // (a row that sees nothing is zero)
                if (!whole && tid < RT) a.ml[(int64_t)slot * ROWS + r] = make_float2(most, norm);
                const uint32_t region = base + (last ? S::K_AT : S::REGION_AT);
#pragma unroll 1
                for (int first = 0; first < rows; first += together) {
                    const bool here = r >= first && r < first + together && r < rows;
                    if (first > 0) tc_rows_sync();
                    // (behind a row's sums of the first part, its norm)
                    if (GROUPS > 1 && here && tid < RT)
                        tc_put16(region + ((r - first) * S::PITCH + DIM) * 4, make_uint4(__float_as_uint(norm), 0, 0, 0));
                    if (__any_sync(0xffffffffu, here))
#pragma unroll 1
                        for (int d = 0; d < c.dim; d += 32) {
                            uint32_t o[32];
                            tc_load(o, at_o + d);
                            tc_loaded(o);
                            const uint32_t to = region + ((tid / RT * together + r - first) * S::PITCH + d) * 4;
                            if (here)
#pragma unroll
                                for (int i = 0; i < 32; i += 4)
                                    tc_put16(to + 4 * i, any ? make_uint4(__float_as_uint(__uint_as_float(o[i]) * f), __float_as_uint(__uint_as_float(o[i + 1]) * f),
                                                                          __float_as_uint(__uint_as_float(o[i + 2]) * f), __float_as_uint(__uint_as_float(o[i + 3]) * f))
                                                             : make_uint4(0, 0, 0, 0));
                            __syncwarp();
                        }
                    tc_rows_sync();
#pragma unroll 1
                    for (int t = tid; t < together * (DIM / 4); t += 2 * TC_TEAM) {
                        const int rr = t / (DIM / 4), col = t % (DIM / 4) * 4;
                        if (first + rr >= rows || col >= c.dim) continue;
                        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                        for (int g = 0; g < 2 * GROUPS; ++g) {
                            const uint4 y = tc_shared16(region + ((g * together + rr) * S::PITCH + col) * 4);
                            x.x += __uint_as_float(y.x), x.y += __uint_as_float(y.y), x.z += __uint_as_float(y.z), x.w += __uint_as_float(y.w);
                        }
                        if constexpr (GROUPS > 1) {
                            const float all = x.x + x.y + x.z + x.w;
                            if (all != all && !isnan(__uint_as_float(tc_shared16(region + (rr * S::PITCH + DIM) * 4).x)))
                                x = tc_wild<T>(a, x, item.b, item.head, row0, first + rr, item.tile, count, item.keys, col);
                        }
                        if (whole) *(uint2*)(out_at(first + rr) + col) = make_uint2(pack_two<T>(x.x, x.y), pack_two<T>(x.z, x.w));
                        else *(float4*)(a.part + ((int64_t)slot * ROWS + first + rr) * DIM + col) = x;
                    }
                }
            }
            tc_before();
            if (!ends && item_begin >= share.lo)
                begun = AttendBegun{row0, item.seq.first, item.head, rows, share.last_of(item_begin, item_begin + item.own_units(), item.weight) - (int)blockIdx.x, 0};
            it = end;
            unit = unit_after;
            item = after;
        }
        if (tid == 0) a.begun[blockIdx.x] = begun;
    }
    // what the two warps have issued, arrivals among it, ends before the tensor memory is given back and the CTA goes (here, and not at the end of
    // their branch: there it costs the products' loops registers, and trees take 8 us more)
    if (const int issuer = threadIdx.x >> 5; issuer == 8 || issuer == 11) {
        uint64_t& mine = bars.last[issuer & 1];
        int quit = 0;
        tc_commit(mine, threadIdx.x % 32 == 0);
        tc_wait(mine, 0, (volatile int*)&quit, TC_POLLS_LAST);
    }
    tc_before();
    __syncthreads();
    if (warp == 8) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

// --- host ------------------------------------------------------------------------------------------------------------------------

// The largest power of two that divides a page, 128 at most.
static int tc_group(int page_size)
{
    const int g = page_size & -page_size;
    return g < TC_KEYS ? g : TC_KEYS;
}

// Whether a tensor map can describe one side of the cache: a dimension that is stepped over has a stride.
static bool tc_strides_ok(const int64_t (&s)[3], const lda_paged_cache& c)
{
    return (s[0] > 0 || c.pages <= 1) && (s[1] > 0 || c.page_size == 1) && (s[2] > 0 || c.kv_heads == 1);
}

bool attend_tc_takes(const lda_paged_cache& c)
{
    return c.dim <= 128 && c.pages > 0 && tc_group(c.page_size) >= 8 && tc_strides_ok(c.key_strides, c) && tc_strides_ok(c.value_strides, c);
}

using TcEncode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                              CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static TcEncode tc_encode()
{
    static std::atomic<void*> known;
    void* fn = known.load(std::memory_order_acquire);
    if (!fn) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess)
            return nullptr;
        known.store(fn, std::memory_order_release);
    }
    return (TcEncode)fn;
}

static bool tc_map(CUtensorMap& map, void* at, const int64_t (&strides)[3], const lda_paged_cache& c, int group)
{
    const TcEncode encode = tc_encode();
    if (!encode) return false;
    const auto bytes = [](int64_t stride) { return (cuuint64_t)(stride > 0 ? 2 * stride : 16); };  // (of a dimension of one: never taken)
    const cuuint64_t sizes[4] = {(cuuint64_t)c.dim, (cuuint64_t)c.page_size, (cuuint64_t)c.kv_heads, (cuuint64_t)c.pages};
    const cuuint64_t steps[3] = {bytes(strides[1]), bytes(strides[2]), bytes(strides[0])};
    const cuuint32_t box[4] = {64, (cuuint32_t)group, 1, 1}, each[4] = {1, 1, 1, 1};
    return encode(&map, c.dtype == LDA_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, at, sizes, steps, box, each,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int DIM, int ROWS>
static cudaError_t launch_tc(const AttendArgs& a, const TcMaps& maps, cudaStream_t st)
{
    using S = TcShape<DIM, ROWS>;
    static std::atomic<bool> allowed[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !allowed[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(k_attend_tc<T, DIM, ROWS>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SHARED);
        if (e != cudaSuccess) return e;
        if (dev < 64) allowed[dev].store(true, std::memory_order_release);
    }
    k_attend_tc<T, DIM, ROWS><<<a.ctas, TC_THREADS, S::SHARED, st>>>(a, maps);
    return cudaGetLastError();
}

template <typename T, int DIM>
static cudaError_t tc_by_rows(const AttendArgs& a, const TcMaps& maps, cudaStream_t st)
{
    return a.rows == 32 ? launch_tc<T, DIM, 32>(a, maps, st) : a.rows == 64 ? launch_tc<T, DIM, 64>(a, maps, st) : launch_tc<T, DIM, 256>(a, maps, st);
}

cudaError_t attend_tc(const AttendArgs& a, const lda_paged_cache& cache, cudaStream_t st)
{
    TcMaps maps;
    const int group = tc_group(cache.page_size);
    maps.group_bits = 0;
    while (1 << maps.group_bits < group) ++maps.group_bits;
    if (!tc_map(maps.k, cache.keys, cache.key_strides, cache, group) || !tc_map(maps.v, cache.values, cache.value_strides, cache, group))
        return cudaErrorInvalidValue;
    if (cache.dtype == LDA_F16) return cache.dim <= 64 ? tc_by_rows<__half, 64>(a, maps, st) : tc_by_rows<__half, 128>(a, maps, st);
    return cache.dim <= 64 ? tc_by_rows<__nv_bfloat16, 64>(a, maps, st) : tc_by_rows<__nv_bfloat16, 128>(a, maps, st);
}

}  // namespace lda
