// Attention of one new token a sequence over a paged cache:  o = sum_j softmax_j(c q . k_j) v_j  for the heads that share a key head.
//
// One pass over the rows with the running maximum and sum of the softmax (weights 2^(s - M), s the score times log2 e), on the tensor cores with the rows of the
// cache as the rows of the products: S^T (16 rows x 8 heads) = K Q^T and O^T (16 values x 8 heads) += V^T P^T.  So a warp's products are full for up to 8
// heads of a key head, twice as wide for up to 16, and more heads are so many items.  Both products' inner dimension may be in any order
// as long as their two operands agree on it, and so may the values' order: a lane's operands of K are then 16 neighbouring bytes of a row, those of V^T 8 or 16
// neighbouring values of four rows, put in pairs by byte permutes.  P^T comes from S^T by transposing 8 x 8 blocks among the lanes.
//
// Bound by the cache's bytes.  Each warp has rows of its own and a ring of its own in shared memory that it fills by asynchronous copies of 16 bytes, rows outside the
// sequence and values beyond head_size as zeros: nothing in the loop waits for another warp.  About 128 KB are under way on an SM: 32 sequences of up to 32768 tokens of
// 8 key heads of 128 values, 2.84 GB, in 422 us, 6.7 TB/s (a kernel that does nothing but read as much: 387 us, 7.3); one of 131071, 537 MB, in 90 us, 6.0 TB/s; 64 of up to 8192 of
// 4 key heads in 8 bits, 331 MB, in 71 us, 4.7 TB/s; 33 of up to 4099 of 12 heads of 80 values, 328 MB, in 74 us, 4.4 TB/s.  The last two wait for dependent instructions (47 and 41 %
// of issue slots; two warps a scheduler): queries of one or seven heads fill an eighth of the products or nearly all, at the same cost in instructions, and 80 values cost what 128 do,
// three eighths of both products, of the copies and of the ring being zeros.  16-byte
// chunks of a row are permuted by the row's number, so that reads by 8 lanes, of two rows or of four, fall into different banks.
//
// Few short items have a cluster each (ranks_of), whose CTAs add their parts up out of one another's shared memory.  Else the
// work is cut evenly, whatever the lengths: steps of WARPS * ROWS rows, of all sequences and key heads one after another, in as many equal runs as there are CTAs. A
// run's first and last item may be a part of one: its sums go to the workspace, and the join kernel adds an item's parts in order.  No atomics: the
// same bits every time.
//
// Weights are rounded to 16 bits for the second product, whose operands have one type: that of the cache's values.  A weight is off by half a step of it at most, so a result by as much
// of the sum of weight times |value|, which is what rounding the result to that type costs where values have one sign.  As two numbers in 16 bits each it would take a second product and as
// many instructions more, of which shapes in 8 bits and of one head have too many as it is.  They are at most 2^12, not 1, in f16: what lies below f16's smallest number is then 2^-37 of the
// largest, too little to matter in 2^17 rows.  Rows in 8 bits are exact in f16: s is scaled by the key row's scale, a weight by the value row's, and M is the
// largest of s + log2(value scale), so that scaled weights keep within f16's range whatever the scales are.  Queries in bf16 are brought into f16's by a
// power of two a head: exactly down to 2^-17 of the head's largest value; what is smaller is off by 2^-25 of that at most, as a sum in 32 bits is by 2^-24 of its largest term.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "attention.h"
#include "llm.h"

namespace strassen {
namespace decode {

constexpr int WARPS = 4, STAGES = 3, THREADS = 32 * WARPS;
constexpr int HALF_STAGE = 4096, STAGE = 2 * HALF_STAGE;       // a warp's rows of K, then of V
enum { BF16 = 0, F16 = 1, E4M3 = 2 };                          // what the cache holds

// A part of an item: sums, then per head M and the sum of weights.
__host__ __device__ constexpr int part_floats(int dp, int nt) { return 8 * nt * (dp + 2); }

struct Meta {
    int b, item;          // the item that begins in this run and does not end in it, or (by_item) this item
    int last;             // the run it ends in; -1: there is no such item, or it is in one run
    int first;            // the run it begins in
};

struct Args {
    AttentionArgs a;
    int items;            // key heads * blocks of heads
    int blocks, group;    // blocks of heads of a key head; heads of a key head
    int ranks;            // CTAs of a cluster, where one has an item
    bool wide;            // q's rows start at multiples of 16 bytes
    bool by_item;         // a Meta for each item; else for each run
    Meta *meta;
    float *parts;
};

// What a sequence's token sees: rows lo .. end - 1.
struct Span {
    int64_t lo, end;
};
__device__ __forceinline__ Span span_of(const AttentionArgs &a, int b)
{
    const int64_t length = a.seq.lengths[b], most = int64_t(a.seq.width) << a.cache.page_shift;
    Span s;
    s.end = length < most ? length : most;
    s.lo = a.window && length > a.window ? length - a.window : 0;
    if (s.lo > s.end) s.lo = s.end;
    if (s.end < 0) s.lo = s.end = 0;
    return s;
}

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ float exp2_of(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float log2_of(float x)
{
    float y;
    asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <bool BF> __device__ __forceinline__ uint32_t two_16_bits(float lo, float hi)
{
    uint32_t d;
    if (BF) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
template <bool BF> __device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if (BF)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v)
{
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}
// Two e4m3 as two f16, exactly.
__device__ __forceinline__ uint32_t two_of_e4m3(uint32_t v)
{
    uint32_t d;
    asm("{\n .reg .b16 h;\n cvt.u16.u32 h, %1;\n cvt.rn.f16x2.e4m3x2 %0, h;\n}" : "=r"(d) : "r"(v));
    return d;
}
__device__ __forceinline__ void copy16(uint32_t to, const void *from, uint32_t bytes)        // bytes 0: zeros
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t to, const void *from, uint32_t bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}

// KIND: of the cache; DP: head_size, padded with zeros; NT: blocks of 8 heads.
template <int KIND, int DP, int NT> struct Shape {
    static constexpr int SIZE = KIND == E4M3 ? 1 : 2, ROW = DP * SIZE, CHUNKS = ROW / 16;
    static constexpr int ROWS = HALF_STAGE / ROW;              // of a warp's stage: 16, 32 or 64
    static constexpr int STEP = WARPS * ROWS;                  // rows of a step
    static constexpr int SCALES = KIND == E4M3 ? 8 * ROWS : 0; // bytes of the rows' scales in a stage, of K, then of V
    static constexpr int RING = STAGES * STAGE, SMEM = WARPS * STAGES * (STAGE + SCALES);
    static constexpr int MT = DP / 16;                         // tiles of 16 values in O^T
    // where chunk c of row r is
    static __device__ __forceinline__ int place(int r, int c)
    {
        const int f = CHUNKS == 4 ? r >> 1 & 3 : (r & 2) | ((r >> 2 ^ r) & 1) << 2;
        return r * ROW + (c ^ f) * 16;
    }
};

// Which value of a row is number g (half 0) or g + 8 (half 1) of tile i of O^T.
template <int KIND, int DP> __device__ __forceinline__ int value_of(int i, int g, int half)
{
    if (DP == 64) return 8 * g + 4 * half + i;
    return KIND == E4M3 ? 16 * g + 8 * half + i : 64 * half + 8 * g + i;
}

// a / b for numbers that are not negative.  Nearly always both have 32 bits, and the division that takes five times as long is not made: four of them were
// 3000 clocks of the 4000 that pass before a CTA knows what to do.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b)
{
    if (((a | b) >> 32) == 0) return uint32_t(a) / uint32_t(b);
    return a / b;
}
// `total` steps in `runs` runs: the first ones have one more.
struct Runs {
    int64_t size, longer;
    __device__ __forceinline__ Runs(int64_t total, int runs) : size(quotient(total, runs)), longer(total - size * runs) {}
    __device__ __forceinline__ int64_t begin(int run) const { return size * run + (run < longer ? run : longer); }
    // the run that has step n
    __device__ __forceinline__ int of(int64_t n) const
    {
        const int64_t in_longer = longer * (size + 1);
        return int(n < in_longer ? quotient(n, size + 1) : longer + quotient(n - in_longer, size));
    }
};

// Steps of all sequences, and which of them is step `at`.  All threads of the CTA take part; every thread gets the answer.
template <int STEP> struct Plan {
    int64_t total, first;                    // first: of the thread's first sequence
    __device__ __forceinline__ static int64_t steps(const AttentionArgs &a, int b)
    {
        const Span s = span_of(a, b);
        return int64_t(uint64_t(s.end - s.lo + STEP - 1) / STEP);
    }
    __device__ __forceinline__ static int64_t block_sum(int64_t v, int64_t *sh)
    {
        for (int i = 16; i > 0; i >>= 1) v += __shfl_xor_sync(~0u, v, i);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0;
        for (int w = 0; w < WARPS; ++w) v += sh[w];
        return v;
    }
    __device__ Plan(const AttentionArgs &a, int64_t *sh)
    {
        int64_t mine = 0;
        first = threadIdx.x < a.seq.batch ? steps(a, threadIdx.x) : 0;
        mine = first;
        for (int b = threadIdx.x + THREADS; b < a.seq.batch; b += THREADS) mine += steps(a, b);
        total = block_sum(mine, sh);
    }
    // The sequence that holds step `at` of total, and the steps before it.
    __device__ void find(const AttentionArgs &a, int64_t at, int64_t *sh, int *b, int64_t *before) const
    {
        int64_t base = 0;
        for (int b0 = 0; b0 < a.seq.batch; b0 += THREADS) {
            const int mine = b0 + int(threadIdx.x);
            const int64_t n = b0 == 0 ? first : mine < a.seq.batch ? steps(a, mine) : 0;
            int64_t upto = n;
            for (int i = 1; i < 32; i <<= 1) {
                const int64_t other = __shfl_up_sync(~0u, upto, i);
                if ((threadIdx.x & 31) >= i) upto += other;
            }
            __syncthreads();
            if ((threadIdx.x & 31) == 31) sh[threadIdx.x >> 5] = upto;
            if (threadIdx.x == 0) sh[WARPS] = -1;
            __syncthreads();
            int64_t all = 0;
            for (int w = 0; w < WARPS; ++w) {
                if (w < int(threadIdx.x >> 5)) upto += sh[w];
                all += sh[w];
            }
            const int64_t from = base + upto - n;
            if (n > 0 && at >= from && at < from + n) {
                sh[WARPS] = mine;
                sh[WARPS + 1] = from;
            }
            __syncthreads();
            if (sh[WARPS] >= 0) break;
            base += all;
        }
        *b = int(sh[WARPS]);
        *before = sh[WARPS + 1];
        __syncthreads();
    }
};

__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The number at `at` in the shared memory of a CTA of the cluster.
__device__ __forceinline__ float of_rank(const float *at, uint32_t rank)
{
    uint32_t there;
    float v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(smem_addr(at)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(there) : "memory");
    return v;
}

// TOGETHER: a cluster has one item, whose parts its CTAs add up at the end, out of one another's shared memory.
template <int KIND, int DP, int NT, bool TOGETHER> __global__ void __launch_bounds__(THREADS, 2) decode_kernel(const Args p)
{
    using S = Shape<KIND, DP, NT>;
    constexpr bool BF = KIND == BF16;
    constexpr int ROWS = S::ROWS, SUB = ROWS / 16, MT = S::MT, KS = DP / 16;
    constexpr float RAISE = BF ? 0.f : 12.f;             // weights are 2^(s - M + RAISE)
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int64_t scratch[WARPS + 2];
    __shared__ float sh_m[WARPS][8 * NT], sh_l[WARPS][8 * NT], all_sums[2 * 8 * NT];
    const AttentionArgs &a = p.a;
    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    uint8_t *const ring = smem + warp * S::RING;
    uint8_t *const scales = smem + WARPS * S::RING + warp * STAGES * S::SCALES;

    after_work_before();
    // A place in the order of all steps; one for the copies, which run ahead, one for the products.
    struct Place {
        int b, item;
        int64_t step, steps, lo, end;
        __device__ __forceinline__ void sequence(const AttentionArgs &a, int which)
        {
            b = which;
            const Span s = span_of(a, b);
            lo = s.lo;
            end = s.end;
            steps = int64_t(uint64_t(end - lo + S::STEP - 1) / S::STEP);
        }
        __device__ __forceinline__ void next(const Args &p)
        {
            if (++step < steps) return;
            step = 0;
            if (++item < p.items) return;
            item = 0;
            do {
                if (++b >= p.a.seq.batch) {
                    steps = lo = end = 0;
                    return;
                }
                sequence(p.a, b);
            } while (steps == 0);
        }
    } ahead, at;
    int64_t from, to;
    Runs runs(0, 1);
    if (TOGETHER) {
        const int which = blockIdx.x / p.ranks, rank = blockIdx.x % p.ranks;
        at.sequence(a, p.items == 1 ? which : which / p.items);
        at.item = which - at.b * p.items;
        runs = Runs(at.steps, p.ranks);
        from = runs.begin(rank), to = runs.begin(rank + 1);
        at.step = from;
        ahead = at;
    } else {
        // sequences that see nothing
        for (int b = blockIdx.x; b < a.seq.batch; b += gridDim.x) {
            if (Plan<S::STEP>::steps(a, b) > 0) continue;
            for (int i = threadIdx.x; p.by_item && i < p.items; i += THREADS) p.meta[b * p.items + i].last = -1;
            for (int i = threadIdx.x; i < a.heads * a.cache.d; i += THREADS)
                static_cast<uint16_t *>(a.out)[b * a.out_row + i / a.cache.d * a.out_head + i % a.cache.d] = 0;
        }
        const Plan<S::STEP> plan(a, scratch);
        // no run is empty: an item's parts are in neighbouring ones
        const int64_t total = plan.total * p.items;
        if (!p.by_item && threadIdx.x == 0) p.meta[blockIdx.x].last = -1;
        if (blockIdx.x >= total) return;
        runs = Runs(total, int(total < gridDim.x ? total : gridDim.x));
        from = runs.begin(blockIdx.x), to = runs.begin(blockIdx.x + 1);
        int b;
        int64_t before;
        plan.find(a, quotient(from, p.items), scratch, &b, &before);
        // steps of sequence b: item after item
        at.sequence(a, b);
        const int64_t inside = from - before * p.items;
        at.item = int(quotient(inside, at.steps));
        at.step = inside - at.item * at.steps;
        ahead = at;
    }

    // ---- queries ----------------------------------------------------------------------------------------------------
    uint32_t q[NT][KS][2];
    float factor[NT][2], m[NT][2], l[NT][2], o[NT][MT][4];
    int64_t first_step = 0;                              // of the item, in this run
    // queries of the item that `at` is in, and nothing summed up yet
    const auto begin_item = [&] {
        first_step = at.step;
        const int kv = p.blocks == 1 ? at.item : at.item / p.blocks, head0 = kv * p.group + (p.blocks == 1 ? 0 : (at.item % p.blocks) * 8 * NT);
        const int heads = (kv + 1) * p.group - head0;          // of them, up to 8 * NT
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            // lane (g, t): head g's values beside the rows' chunks 4 c + t
            const bool there = 8 * nt + g < heads;
            const uint16_t *row = static_cast<const uint16_t *>(a.q.p) + at.b * a.q.row + (head0 + 8 * nt + g) * a.q.head;
            uint32_t w[KS][2];
            constexpr int LOADS = DP / 32;                      // of 8 values
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int first = KIND == E4M3 ? 16 * (4 * (i / 2) + t) + 8 * (i & 1) : 8 * (4 * i + t);
                uint4 u = make_uint4(0, 0, 0, 0);
                if (there && first < a.cache.d) {
                    if (p.wide) {
                        u = *reinterpret_cast<const uint4 *>(row + first);
                    } else {
                        u.x = row[first] | uint32_t(row[first + 1]) << 16;
                        u.y = row[first + 2] | uint32_t(row[first + 3]) << 16;
                        u.z = row[first + 4] | uint32_t(row[first + 5]) << 16;
                        u.w = row[first + 6] | uint32_t(row[first + 7]) << 16;
                    }
                }
                w[2 * i][0] = u.x;
                w[2 * i][1] = u.y;
                w[2 * i + 1][0] = u.z;
                w[2 * i + 1][1] = u.w;
            }
            float back = 1.f;
            if (KIND == E4M3 && a.type == STRASSEN_BF16) {
                float most = 0.f;
#pragma unroll
                for (int i = 0; i < KS; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        most = fmaxf(most, fmaxf(fabsf(__uint_as_float(w[i][e] << 16)), fabsf(__uint_as_float(w[i][e] & 0xffff0000u))));
                most = fmaxf(most, __shfl_xor_sync(~0u, most, 1));
                most = fmaxf(most, __shfl_xor_sync(~0u, most, 2));
                // the power of two that brings the largest to 1 .. 2; queries that are 0 or no numbers are left alone
                const uint32_t e = __float_as_uint(most) >> 23;
                const bool turn = e > 1 && e < 253;
                const float down = turn ? __uint_as_float((254 - e) << 23) : 1.f;
                back = turn ? __uint_as_float(e << 23) : 1.f;
#pragma unroll
                for (int i = 0; i < KS; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) w[i][e] = two_16_bits<false>(__uint_as_float(w[i][e] << 16) * down, __uint_as_float(w[i][e] & 0xffff0000u) * down);
            }
#pragma unroll
            for (int i = 0; i < KS; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) q[nt][i][e] = w[i][e];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                factor[nt][e] = a.scale * 1.4426950408889634f * __shfl_sync(~0u, back, 4 * (2 * t + e));
                m[nt][e] = -INFINITY;
                l[nt][e] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nt][i][e] = 0.f;
        }
    };

    // ---- copies ------------------------------------------------------------------------------------------------------
    const int64_t count = to - from;
    int64_t copied = 0;
    constexpr int MINE = (ROWS + 31) / 32;
    int pages[MINE];                                     // of the rows lane, lane + 32 of the next stage, as the table has them: not looked at before they are used,
                                                         // so that nothing waits for the table (1300 clocks of a step's 2400 otherwise)
    auto look_up = [&](int (&pages)[MINE], int64_t copied) {
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const int r = lane + 32 * i;
            const int64_t j = ahead.lo + (ahead.step * WARPS + warp) * ROWS + r;
            pages[i] = -1;
            if (copied < count && r < ROWS && j < ahead.end) pages[i] = a.seq.table[ahead.b * a.seq.ld_table + (j >> a.cache.page_shift)];
        }
    };
    auto start = [&](int stage, const Place &ahead, const int (&pages)[MINE]) {
        {
            const int h = p.blocks == 1 ? ahead.item : ahead.item / p.blocks;
            const int j0 = int(ahead.lo + (ahead.step * WARPS + warp) * ROWS), mask = (1 << a.cache.page_shift) - 1;
            const uint32_t k_to = smem_addr(ring + stage * STAGE), v_to = k_to + HALF_STAGE;
            // where the lane's rows begin; -1: nowhere
            int64_t place[MINE];
#pragma unroll
            for (int i = 0; i < MINE; ++i) {
                const int slot = (j0 + lane + 32 * i) & mask;
                const bool there = uint32_t(pages[i]) < uint64_t(a.cache.pages);
                place[i] = there ? pages[i] * a.cache.page_stride + h * a.cache.head_stride + slot * a.cache.row_stride : -1;
                if (KIND == E4M3 && lane + 32 * i < ROWS) {
                    const int64_t from = there ? ((int64_t(pages[i]) * a.cache.kv_heads + h) << a.cache.page_shift) + slot : 0;
                    const uint32_t to = smem_addr(scales + stage * S::SCALES) + 4 * (lane + 32 * i);
                    copy4(to, a.cache.k_scale + from, there ? 4 : 0);
                    copy4(to + 4 * ROWS, a.cache.v_scale + from, there ? 4 : 0);
                }
            }
            const int chunk = lane % S::CHUNKS;
            const bool inside = chunk * 16 < a.cache.d * S::SIZE;
#pragma unroll
            for (int i = 0; i < ROWS * S::CHUNKS / 32; ++i) {
                const int r = i * (32 / S::CHUNKS) + lane / S::CHUNKS;
                const int64_t at = __shfl_sync(~0u, place[ROWS > 32 ? (i * (32 / S::CHUNKS)) >> 5 : 0], r & 31);
                const bool there = at >= 0 && inside;
                const int64_t off = there ? at + chunk * 16 : 0;
                const uint32_t to = S::place(r, chunk), bytes = there ? 16 : 0;
                copy16(k_to + to, a.cache.k + off, bytes);
                copy16(v_to + to, a.cache.v + off, bytes);
            }
        }
    };
    auto copy = [&](int stage) {
        if (copied < count) {
            start(stage, ahead, pages);
            ahead.next(p);
            ++copied;
            look_up(pages, copied);
            if (warp == 0 && ahead.step == 0 && copied < count) {
                // the next item's queries on their way to the second cache, in time before they are asked for
                const int kv = p.blocks == 1 ? ahead.item : ahead.item / p.blocks, head = kv * p.group + (p.blocks == 1 ? 0 : (ahead.item % p.blocks) * 8 * NT) + lane / 2;
                if (lane < 16 * NT && head < (kv + 1) * p.group && 64 * (lane & 1) < a.cache.d)
                    asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const uint16_t *>(a.q.p) + ahead.b * a.q.row + head * a.q.head + 64 * (lane & 1)));
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // the pages of the first steps are looked up together
    static_assert(STAGES == 3, "two steps ahead");
    {
        int first[MINE];
        const Place before = ahead;
        look_up(first, 0);
        ahead.next(p);
        look_up(pages, 1);
        begin_item();                    // before the copies: behind them it would wait for 3 us
        start(0, before, first);
        copied = 1;
        asm volatile("cp.async.commit_group;" ::: "memory");
        copy(1);
    }

    // ---- products ----------------------------------------------------------------------------------------------------
    int stage = 0;
#pragma unroll 1
    for (int64_t n = 0; n < count; ++n) {
        if (n > 0 && at.step == 0) begin_item();
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
        __syncwarp();                                    // the stage's copies of all lanes are here, and the one before has been read by all
        copy(stage == 0 ? STAGES - 1 : stage - 1);
        const uint8_t *const k_at = ring + stage * STAGE, *const v_at = k_at + HALF_STAGE;
        const int64_t left = at.end - (at.lo + (at.step * WARPS + warp) * ROWS);       // rows of this stage that are seen
        if (left > 0) {
            float s[NT][SUB][4];
#pragma unroll
            for (int sub = 0; sub < SUB; ++sub) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[nt][sub][e] = 0.f;
#pragma unroll
                for (int c = 0; c < S::CHUNKS / 4; ++c) {
                    const uint4 u = *reinterpret_cast<const uint4 *>(k_at + S::place(16 * sub + g, 4 * c + t)), v = *reinterpret_cast<const uint4 *>(k_at + S::place(16 * sub + g + 8, 4 * c + t));
                    const uint32_t lo[4] = {u.x, u.y, u.z, u.w}, hi[4] = {v.x, v.y, v.z, v.w};
                    if (KIND == E4M3) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t a0 = two_of_e4m3(lo[i]), a2 = two_of_e4m3(lo[i] >> 16), a1 = two_of_e4m3(hi[i]), a3 = two_of_e4m3(hi[i] >> 16);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) mma<BF>(s[nt][sub], a0, a1, a2, a3, q[nt][4 * c + i][0], q[nt][4 * c + i][1]);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) mma<BF>(s[nt][sub], lo[2 * i], hi[2 * i], lo[2 * i + 1], hi[2 * i + 1], q[nt][2 * c + i][0], q[nt][2 * c + i][1]);
                    }
                }
            }
            // scores in powers of two; rows that are not there: none
            float vs[SUB][2];
            const float *const ks_at = reinterpret_cast<const float *>(scales + stage * S::SCALES);
            float most[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) most[nt][0] = most[nt][1] = -INFINITY;
#pragma unroll
            for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int r = 16 * sub + 8 * half + g;
                    const bool there = r < left;
                    float ks = 1.f, more = 0.f;
                    if (KIND == E4M3) {
                        ks = ks_at[r];
                        vs[sub][half] = there ? ks_at[ROWS + r] : 0.f;
                        more = log2_of(fmaxf(fabsf(vs[sub][half]), kMinRowScale));       // of a page that is not there 0: M stays within 2^64 of s
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float &x = s[nt][sub][2 * half + e];
                            x = there ? x * (factor[nt][e] * ks) : -INFINITY;
                            most[nt][e] = fmaxf(most[nt][e], KIND == E4M3 ? x + more : x);
                        }
                }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                bool grows = false;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float &x = most[nt][e];
                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 4));
                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 8));
                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 16));
                    grows |= x > m[nt][e];
                }
                if (__any_sync(~0u, grows)) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float next = fmaxf(m[nt][e], most[nt][e]), back = m[nt][e] == next ? 1.f : exp2_of(m[nt][e] - next);
                        m[nt][e] = next;
                        l[nt][e] *= back;
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            o[nt][i][e] *= back;
                            o[nt][i][2 + e] *= back;
                        }
                    }
                }
            }
            uint32_t w[NT][SUB][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                // nothing but -inf so far: weights of 0
                const float off[2] = {m[nt][0] == -INFINITY ? 0.f : m[nt][0] - RAISE, m[nt][1] == -INFINITY ? 0.f : m[nt][1] - RAISE};
                float sum[2] = {0.f, 0.f};
#pragma unroll
                for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        float x[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            x[e] = exp2_of(s[nt][sub][2 * half + e] - off[e]);
                            sum[e] += x[e];
                            if (KIND == E4M3) x[e] *= vs[sub][half];
                        }
                        w[nt][sub][half] = transpose8(two_16_bits<BF>(x[0], x[1]));
                    }
                l[nt][0] += sum[0];
                l[nt][1] += sum[1];
            }
            // V^T: rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9 of 16; two rows' values in pairs
#pragma unroll
            for (int sub = 0; sub < SUB; ++sub) {
                const int r = 16 * sub + 2 * t;
                if (KIND != E4M3) {
                    constexpr int PER = DP / 64;               // chunks of a row that a lane has
                    uint32_t rows[4][PER][4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int c = 0; c < PER; ++c) {
                            const uint4 u = *reinterpret_cast<const uint4 *>(v_at + S::place(r + (i & 1) + 8 * (i >> 1), g + 8 * c));
                            rows[i][c][0] = u.x;
                            rows[i][c][1] = u.y;
                            rows[i][c][2] = u.z;
                            rows[i][c][3] = u.w;
                        }
                    // tile i: value 8 g + i and, DP 128: 64 + 8 g + i; DP 64: 8 g + 4 + i
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        const int lw = i / 2, hc = PER - 1, hw = PER == 2 ? i / 2 : 2 + i / 2;
                        const uint32_t pick = i & 1 ? 0x7632 : 0x5410;
                        const uint32_t a0 = __byte_perm(rows[0][0][lw], rows[1][0][lw], pick), a1 = __byte_perm(rows[0][hc][hw], rows[1][hc][hw], pick),
                                       a2 = __byte_perm(rows[2][0][lw], rows[3][0][lw], pick), a3 = __byte_perm(rows[2][hc][hw], rows[3][hc][hw], pick);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma<BF>(o[nt][i], a0, a1, a2, a3, w[nt][sub][0], w[nt][sub][1]);
                    }
                } else {
                    // values 16 g + i and 16 g + 8 + i (DP 64: 8 g + i and 8 g + 4 + i) in tile i
                    constexpr int WORDS = DP / 32;
                    uint32_t rows[4][WORDS];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int row = r + (i & 1) + 8 * (i >> 1);
                        if (DP == 128) {
                            const uint4 u = *reinterpret_cast<const uint4 *>(v_at + S::place(row, g));
                            rows[i][0] = u.x;
                            rows[i][1] = u.y;
                            rows[i][WORDS - 2] = u.z;
                            rows[i][WORDS - 1] = u.w;
                        } else {
                            const uint2 u = *reinterpret_cast<const uint2 *>(v_at + S::place(row, g >> 1) + 8 * (g & 1));
                            rows[i][0] = u.x;
                            rows[i][1] = u.y;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < MT; i += 2) {
                        // bytes i and i + 1 of two rows: values i of both, then i + 1 of both
                        const int lw = i / 4, hw = WORDS / 2 + i / 4;
                        const uint32_t pick = i % 4 == 0 ? 0x5140 : 0x7362;
                        const uint32_t x0 = __byte_perm(rows[0][lw], rows[1][lw], pick), x1 = __byte_perm(rows[0][hw], rows[1][hw], pick), x2 = __byte_perm(rows[2][lw], rows[3][lw], pick),
                                       x3 = __byte_perm(rows[2][hw], rows[3][hw], pick);
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const uint32_t a0 = two_of_e4m3(x0 >> 16 * k), a1 = two_of_e4m3(x1 >> 16 * k), a2 = two_of_e4m3(x2 >> 16 * k), a3 = two_of_e4m3(x3 >> 16 * k);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) mma<BF>(o[nt][i + k], a0, a1, a2, a3, w[nt][sub][0], w[nt][sub][1]);
                        }
                    }
                }
            }
        }

        // ---- the end of an item, or of the run -----------------------------------------------------------------------
        const bool ends = at.step + 1 == at.steps;
        if (ends || n + 1 == count) {
            // the warps' sums on one scale, added up in order through the stage that has just been read
            const auto part = [&](int w) { return reinterpret_cast<float *>(smem + w * S::RING + stage * STAGE); };
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float &x = l[nt][e];
                    x += __shfl_xor_sync(~0u, x, 4);
                    x += __shfl_xor_sync(~0u, x, 8);
                    x += __shfl_xor_sync(~0u, x, 16);
                    if (g == 0) {
                        sh_m[warp][8 * nt + 2 * t + e] = m[nt][e];
                        sh_l[warp][8 * nt + 2 * t + e] = x;
                    }
                }
            __syncthreads();
            float all_m[NT][2], all_l[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int h = 8 * nt + 2 * t + e;
                    float most = -INFINITY, sum = 0.f;
#pragma unroll
                    for (int w = 0; w < WARPS; ++w) most = fmaxf(most, sh_m[w][h]);
#pragma unroll
                    for (int w = 0; w < WARPS; ++w) sum += sh_l[w][h] * (sh_m[w][h] == most ? 1.f : exp2_of(sh_m[w][h] - most));
                    const float back = m[nt][e] == most ? 1.f : exp2_of(m[nt][e] - most);
                    all_m[nt][e] = most;
                    all_l[nt][e] = sum;
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        o[nt][i][e] *= back;
                        o[nt][i][2 + e] *= back;
                    }
                }
            const auto put = [&](float *to) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) to[((nt * MT + i) * 4 + e) * 32 + lane] = o[nt][i][e];
            };
            const auto add = [&](const float *from) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[nt][i][e] += from[((nt * MT + i) * 4 + e) * 32 + lane];
            };
            if (warp >= 2) put(part(warp));
            __syncthreads();
            if (warp < 2) add(part(warp + 2));
            if (warp == 1) put(part(1));
            __syncthreads();
            if (warp == 0) {
                add(part(1));
                if (!TOGETHER && ends && first_step == 0) {
                    const int kv = p.blocks == 1 ? at.item : at.item / p.blocks, head0 = kv * p.group + (p.blocks == 1 ? 0 : (at.item % p.blocks) * 8 * NT);
                    uint16_t *const out = static_cast<uint16_t *>(a.out) + at.b * a.out_row;
                    if (p.by_item && lane == 0) p.meta[at.b * p.items + at.item].last = -1;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int head = head0 + 8 * nt + 2 * t + e;
                            const float inv = all_l[nt][e] == 0.f ? 0.f : 1.f / all_l[nt][e];
                            if (head >= (kv + 1) * p.group) continue;
#pragma unroll
                            for (int i = 0; i < MT; ++i)
#pragma unroll
                                for (int half = 0; half < 2; ++half) {
                                    const int at_value = value_of<KIND, DP>(i, g, half);
                                    const float y = o[nt][i][2 * half + e] * inv;
                                    if (at_value < a.cache.d)
                                        out[head * a.out_head + at_value] = uint16_t(a.type == STRASSEN_BF16 ? two_16_bits<true>(y, 0.f) : two_16_bits<false>(y, 0.f));
                                }
                        }
                } else {
                    // the run's first item, begun in another run, or its last
                    float *const to = TOGETHER ? reinterpret_cast<float *>(smem) : p.parts + (2 * int64_t(blockIdx.x) + (first_step == 0 ? 1 : 0)) * part_floats(DP, NT);
                    float *const sums = TOGETHER ? all_sums : to + 8 * NT * DP;
                    put(to);
                    if (g == 0) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                sums[8 * nt + 2 * t + e] = all_m[nt][e];
                                sums[8 * NT + 8 * nt + 2 * t + e] = all_l[nt][e];
                            }
                    }
                    if (!TOGETHER && lane == 0 && first_step == 0) {
                        const int64_t last = from + n + (at.steps - at.step) - 1;            // the item's last step
                        p.meta[p.by_item ? at.b * p.items + at.item : int(blockIdx.x)] = {at.b, at.item, runs.of(last), int(blockIdx.x)};
                    }
                }
            }
            __syncthreads();
        }
        at.next(p);
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    if (TOGETHER) {
        // each CTA adds up some of the tiles of 16 values of 8 heads, a thread a number of one; ranks beyond the steps have none
        cluster_barrier();
        const int which = blockIdx.x / p.ranks, item = p.items == 1 ? 0 : which % p.items, b = p.items == 1 ? which : which / p.items, parts = int(runs.size > 0 ? p.ranks : runs.longer), n = threadIdx.x, head = 2 * t + (warp & 1);
        for (int tile = blockIdx.x % p.ranks; tile < NT * MT; tile += p.ranks) {
            const int nt = tile / MT, i = tile % MT;
            float m[MOST_RANKS], l[MOST_RANKS], v[MOST_RANKS], most = -INFINITY, sum = 0.f, y = 0.f;
#pragma unroll
            for (int k = 0; k < MOST_RANKS; ++k) {
                m[k] = -INFINITY, l[k] = v[k] = 0.f;
                if (k >= parts) continue;
                m[k] = of_rank(all_sums + 8 * nt + head, k);
                l[k] = of_rank(all_sums + 8 * NT + 8 * nt + head, k);
                v[k] = of_rank(reinterpret_cast<const float *>(smem) + tile * 128 + n, k);
            }
#pragma unroll
            for (int k = 0; k < MOST_RANKS; ++k) most = fmaxf(most, m[k]);
#pragma unroll
            for (int k = 0; k < MOST_RANKS; ++k) {
                const float f = m[k] == most ? 1.f : exp2_of(m[k] - most);
                sum += f * l[k];
                y += f * v[k];
            }
            const int kv = p.blocks == 1 ? item : item / p.blocks, h = kv * p.group + (p.blocks == 1 ? 0 : item % p.blocks * 8 * NT) + 8 * nt + head, at_value = value_of<KIND, DP>(i, g, warp >> 1);
            y = sum == 0.f ? 0.f : y / sum;
            if (h < (kv + 1) * p.group && at_value < a.cache.d)
                static_cast<uint16_t *>(a.out)[b * a.out_row + h * a.out_head + at_value] = uint16_t(a.type == STRASSEN_BF16 ? two_16_bits<true>(y, 0.f) : two_16_bits<false>(y, 0.f));
        }
        cluster_barrier();                               // no CTA leaves while another reads its sums
    }
}

// The parts of an item that begins in one run and ends in a later one, added up in order.  A CTA has tiles of 16 values of 8 heads, a thread one number of
// one; its GROUPS of four warps take every GROUPS-th part, and their sums are added in order.
template <int KIND, int DP, int NT, int GROUPS> __global__ void __launch_bounds__(128 * GROUPS) join_kernel(const Args p)
{
    constexpr int MT = DP / 16;
    __shared__ float sh[GROUPS][3][128];
    after_work_before();
    const Meta meta = p.meta[blockIdx.x];
    if (meta.last < 0) return;
    const int count = meta.last - meta.first + 1, group = threadIdx.x / 128, n = threadIdx.x % 128, lane = n & 31, e = n >> 5, head = 2 * (lane & 3) + (e & 1);
    for (int tile = blockIdx.y; tile < NT * MT; tile += gridDim.y) {
        const int nt = tile / MT, i = tile % MT;
        float m = -INFINITY, l = 0.f, o = 0.f;
#pragma unroll 8
        for (int k = group; k < count; k += GROUPS) {
            const float *const part = p.parts + (2 * int64_t(meta.first + k) + (k == 0 ? 1 : 0)) * part_floats(DP, NT);
            const float here = part[8 * NT * DP + 8 * nt + head], sum = part[8 * NT * DP + 8 * NT + 8 * nt + head], v = part[tile * 128 + n];
            const float next = fmaxf(m, here), back = m == next ? 1.f : exp2_of(m - next), w = here == next ? 1.f : exp2_of(here - next);
            m = next;
            l = l * back + w * sum;
            o = o * back + w * v;
        }
        __syncthreads();
        sh[group][0][n] = m;
        sh[group][1][n] = l;
        sh[group][2][n] = o;
        __syncthreads();
        const int kv = meta.item / p.blocks, h = kv * p.group + (meta.item % p.blocks) * 8 * NT + 8 * nt + head, at = value_of<KIND, DP>(i, lane >> 2, e >> 1);
        if (group != 0 || h >= (kv + 1) * p.group || at >= p.a.cache.d) continue;
        float most = m, sum = 0.f, y = 0.f;
#pragma unroll
        for (int k = 1; k < GROUPS; ++k) most = fmaxf(most, sh[k][0][n]);
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) {
            const float f = sh[k][0][n] == most ? 1.f : exp2_of(sh[k][0][n] - most);
            sum += f * sh[k][1][n];
            y += f * sh[k][2][n];
        }
        y = sum == 0.f ? 0.f : y / sum;
        static_cast<uint16_t *>(p.a.out)[meta.b * p.a.out_row + h * p.a.out_head + at] = uint16_t(p.a.type == STRASSEN_BF16 ? two_16_bits<true>(y, 0.f) : two_16_bits<false>(y, 0.f));
    }
}

// CTAs of the largest cluster of Kernel that the current device holds: 16, which has to fit one of its GPU processing clusters, as every device allows 8.  Asked once a device.
template <auto Kernel> int most_ranks(int bytes)
{
    static std::atomic<uint64_t> asked{0}, sixteen{0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 8;
    const uint64_t bit = uint64_t(1) << dev;
    if (!(asked.load(std::memory_order_acquire) & bit)) {
        if (allow_shared<Kernel>(bytes, true) != cudaSuccess) return 8;
        cudaLaunchAttribute size = {};
        size.id = cudaLaunchAttributeClusterDimension;
        size.val.clusterDim.x = MOST_RANKS;
        size.val.clusterDim.y = size.val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(MOST_RANKS);
        cfg.blockDim = dim3(THREADS);
        cfg.dynamicSmemBytes = size_t(bytes);
        cfg.attrs = &size;
        cfg.numAttrs = 1;
        int clusters = 0;
        if (cudaOccupancyMaxActiveClusters(&clusters, Kernel, &cfg) != cudaSuccess) {
            cudaGetLastError();
            clusters = 0;
        }
        if (clusters > 0) sixteen.fetch_or(bit, std::memory_order_release);
        asked.fetch_or(bit, std::memory_order_release);
    }
    return sixteen.load(std::memory_order_acquire) & bit ? MOST_RANKS : 8;
}
template <int KIND, int DP, int NT> int ranks_for(const AttentionArgs &a, int64_t heads, int sm_count)
{
    using S = Shape<KIND, DP, NT>;
    const int ranks = ranks_of(a, S::STEP, heads, sm_count, MOST_RANKS);
    return ranks < MOST_RANKS ? ranks : ranks_of(a, S::STEP, heads, sm_count, most_ranks<decode_kernel<KIND, DP, NT, true>>(S::SMEM));
}

template <int KIND, int DP, int NT> cudaError_t launch(Args p, int sm_count, cudaStream_t stream)
{
    using S = Shape<KIND, DP, NT>;
    cudaError_t e;
    const int64_t steps = steps_of(p.a, S::STEP), all = steps * p.items * p.a.seq.batch;
    const unsigned runs = unsigned(all < 2 * sm_count ? all : 2 * sm_count);
    p.ranks = ranks_for<KIND, DP, NT>(p.a, p.items, sm_count);
    if (p.ranks > 0) {
        e = allow_shared<decode_kernel<KIND, DP, NT, true>>(S::SMEM, true);
        if (e != cudaSuccess) return e;
        return launch_after(decode_kernel<KIND, DP, NT, true>, dim3(unsigned(p.ranks * p.items * p.a.seq.batch)), dim3(THREADS), S::SMEM, stream, dim3(unsigned(p.ranks), 1), p);
    }
    e = allow_shared<decode_kernel<KIND, DP, NT, false>>(S::SMEM);
    if (e != cudaSuccess) return e;
    const int64_t items = p.items * int64_t(p.a.seq.batch);
    p.by_item = runs >= 8 * items;
    e = launch_after(decode_kernel<KIND, DP, NT, false>, dim3(runs), dim3(THREADS), S::SMEM, stream, dim3(1, 1), p);
    // items of a single step are never cut
    if (e != cudaSuccess || steps == 1) return e;
    // many parts an item: a thread has an eighth of them, so that their latencies add up to less, and there is a CTA for each item's tile (one sequence of 131071
    // rows, 32 heads over 8: 89.9 us, 94.0 with quarters and four CTAs for each run; of 20000 rows, 16 heads over one: 19.8, 93.7); few: a CTA for each run and tile (33 sequences of 4099: 77.3 us, 80.8 with
    // eighths)
    if (p.by_item) return launch_after(join_kernel<KIND, DP, NT, 8>, dim3(unsigned(items), NT * DP / 16), dim3(1024), 0, stream, dim3(1, 1), p);
    return launch_after(join_kernel<KIND, DP, NT, 1>, dim3(runs, NT * DP / 16), dim3(128), 0, stream, dim3(1, 1), p);
}

cudaError_t launch_bf16(const Args &p, int dp, int nt, int sm_count, cudaStream_t stream);
cudaError_t launch_f16(const Args &p, int dp, int nt, int sm_count, cudaStream_t stream);
cudaError_t launch_e4m3(const Args &p, int dp, int nt, int sm_count, cudaStream_t stream);
int ranks_bf16(const AttentionArgs &a, int dp, int nt, int64_t heads, int sm_count);
int ranks_f16(const AttentionArgs &a, int dp, int nt, int64_t heads, int sm_count);
int ranks_e4m3(const AttentionArgs &a, int dp, int nt, int64_t heads, int sm_count);

}  // namespace decode
}  // namespace strassen
