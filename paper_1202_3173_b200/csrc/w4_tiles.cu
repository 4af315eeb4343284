// Products of many rows with a matrix of 4-bit weights on the fifth-generation tensor cores.
//
// The weights are the rows of the product, so few rows of x make a narrow product and not a padded one:
//     D (128 rows of weights a CTA x up to 256 rows of x, 32 bits, tensor memory) += A (tensor memory) . B (shared memory)
// Where there are tiles enough, a pair of CTAs (CTAS = 2, tcgen05 cta_group::2) owns 256 rows of weights, and each of the two brings in
// HALF of the rows of x, which both tensor cores read: for single CTAs the rows of x alone would cross L2 -> SM at 64 bytes a clock and
// SM.  Where there are few, single CTAs (CTAS = 1) spread over more of the GPU.  A CTA of 19 warps:
//   * warp 16 streams the laid-out weights with their scales into a ring of shared memory (bulk copies), from before the CTA is set up;
//   * warp 18 brings its part of the rows of x to the same ring (tensor-map copies, which swizzle and fill with zeros past the inner size
//     and the last row);
//   * warps 0-15 turn weights into 16-bit floats in registers, a thread one row of a 128 x 128 tile, and store them to tensor memory as
//     the A operand: they never go back to shared memory, whose bandwidth the B operand needs.  Four groups of four warps take the tiles
//     in turn; four to seven A buffers, as many as D leaves room for;
//   * one thread of warp 17 (of the pair's first CTA) issues the products, eight for each 128 of the inner dimension;
//   * warps 0-15 read D back, multiply by the row's power of two and x's scale in 32 bits, and write.
// The CTAs stay and take tile after tile; the first A buffers of a tile are filled before the tile before it is read back.
//
// A weight is held in 16 bits as S 2^-e (Q - Z) (e: w4_pack.cu): this rounding, to bf16 beside bf16 rows and to f16 beside f16 and
// e4m3 rows, is the price of one chain of products over the whole inner dimension; sums of a group scaled apart in 32 bits would
// cross tensor memory once per group.  It is one rounding of each weight, as large as that of the result to the same type (in f16 down to weights of
// 2^-20 of their row's largest scale).  As in the kernel for few rows, a masked nibble is a subnormal number, and one or two packed instructions
// make a pair of weights of two of them (Num).
//
// Where even single CTAs' tiles are too few to fill the GPU, the CTAs of a cluster split the inner dimension and add their sums in a
// fixed order over distributed shared memory.  Rows of x that a tensor map cannot take as they are (e4m3, other alignments, the rows of an
// expert's tokens) are first written to the workspace in order, in 16 bits (rows_kernel).
//
// Bound by the tensor cores for prompts (4096 x 16384 x 4096, e4m3 with zero points, with the rows' conversion: 348 us in a run of calls on one input,
// 1.6 PFLOP/s, and 409 to 413 where the inputs change from call to call, 1.3 PFLOP/s: the power cap).  For tens of rows by latency: 48 x 4096 x 16384 in 16.4 us, 2.4 TB/s.
// Of the 26 900 clocks of a CTA there, 2 900 pass until its first weights are in shared memory, 18 100 in its 32 steps (a group of warps turns every fourth;
// from one of its steps to the next it takes 2 260, waits included), 400 to read the results back, 2 000 for the cluster's barrier, 2 200 to
// add and write the splits' sums, 1 300 for the barrier after that.
//
// Every wait has a limit, after which the CTA gives up, frees its tensor memory and raises a flag (wait_for).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <atomic>

#include "llm.h"
#include "pieces.cuh"
#include "strassen_b200.h"

namespace strassen {

namespace {

constexpr int TOKENS = 256;                 // most rows of x in a tile of a pair
constexpr int ALONE_TOKENS = 176;           // ... of a single CTA, which brings them all in: three steps fit in shared memory
constexpr int STEP = 16;                    // rows of x that a CTA brings in: a multiple of this
constexpr int GROUPS = 4;                   // groups of four warps that turn weights; at least as many A buffers
constexpr int TURN_WARPS = 4 * GROUPS, WEIGHT_WARP = TURN_WARPS, MMA_WARP = TURN_WARPS + 1, X_WARP = TURN_WARPS + 2, THREADS = 32 * (TURN_WARPS + 3);
// 128-deep steps g = 0, 1, .. over all tiles of a CTA: their weights and their barriers are in rings of RING, at g % RING.  A group sees every
// RING / GROUPS-th of them, always at the same places, so it never takes a phase of a barrier for the one two later.  The rows of x, which are
// larger, have a ring of x_stages, and the A buffers one of a_buffers.
constexpr int RING = 8, MAX_SPLITS = 8;
static_assert(RING % GROUPS == 0, "");
constexpr int A_WIDTH = 64;                 // tensor-memory columns of an A buffer: 128 rows x 128 values of 16 bits; the last of 512, D comes first
constexpr int64_t kWaitLimit = int64_t(1) << 31;      // clocks of a wait, about a second

// Set by a CTA that gave up on a wait; read and cleared by strassen_device_status.
__device__ int g_gave_up;

struct Args {
    const uint8_t *packed;
    const float *exponents;
    const float *x_scale;
    void *out;
    int64_t ldo, depth_tiles;
    int n, m;
    int row_tiles;           // of one matrix
    int group_shift;         // a group is 1 << group_shift words of a row's 16 bytes
    int tile_bytes, zero_off;
    int tokens;              // rows of x in a tile, a multiple of CTAS * STEP
    int box;                 // rows of x in one copy; a CTA brings in whole boxes
    int x_stages, x_bytes;   // up to RING
    int a_buffers;           // GROUPS .. RING
    int out_type;
    bool scale_bf16, has_zeros, out_pairs;
    const W4Tile *table;     // experts: the tiles of rows and their number; NULL: every `tokens` rows a tile
    const int *table_size;
    const int *order;        // experts: which pair a row of x is
    int scale_div;           // experts: x_scale of pair i is x_scale[i / scale_div]
};

// Barriers of step g: full_w / empty_w: its weights have arrived / have been read; ready: the pair's rows of x are in place, and its
// weights are in their A buffers; used: the products that read those are done.  done: all products of a tile of results are; d_free: the
// pair has read them back.  ready and d_free count in the pair's first CTA.
struct Shared {
    uint64_t full_w[RING], empty_w[RING], ready[RING], used[RING], done, d_free;
    uint32_t tmem;
    int dead;
};

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ uint32_t of_rank(const void *p, uint32_t rank)
{
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ uint32_t of_address(uint32_t at, uint32_t rank)
{
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(at), "r"(rank));
    return a;
}
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ float4 remote_float4(uint32_t at)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void bar_init(uint64_t *b, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(b)), "r"(count)); }
__device__ __forceinline__ void bar_arrive(uint64_t *b) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(b)) : "memory"); }
// At the pair's first CTA, after tcgen05 loads and stores that tcgen05.fence::before_thread_sync orders.  Relaxed: a release at cluster scope waits for
// all that the thread has under way, its results' stores among them, and took some thousand clocks of each step (64 tokens, 8 of 64 experts of
// 2048 x 2048: 80 us, 54 without; 4096 x 16384 x 4096: 372 and 360).
__device__ __forceinline__ void bar_arrive_at(uint32_t b) { asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(b) : "memory"); }
__device__ __forceinline__ void bar_expect(uint64_t *b, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(b)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t *b, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(smem_addr(b)), "r"(parity) : "memory");
    return ok != 0;
}
// Whether it is over, without waiting.
__device__ __forceinline__ bool bar_test(uint64_t *b, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(smem_addr(b)), "r"(parity) : "memory");
    return ok != 0;
}
// Waits until phase `parity` of the barrier is over.  False: the limit was reached, here or elsewhere in the CTA, and the caller leaves
// its loop; nothing that comes later waits long, and the results of the call are not valid.
__device__ __forceinline__ bool wait_for(uint64_t *b, uint32_t parity, Shared *sh)
{
    if (bar_try(b, parity)) return true;
    for (const int64_t start = clock64(); clock64() - start < kWaitLimit;) {
#pragma unroll 1
        for (int i = 0; i < 64; ++i)
            if (bar_try(b, parity)) return true;
        if (*reinterpret_cast<volatile int *>(&sh->dead)) return false;
    }
    *reinterpret_cast<volatile int *>(&sh->dead) = 1;
    g_gave_up = 1;
    return false;
}
// For whole warps: the same answer in every lane, so that a warp leaves its loop as one.
__device__ __forceinline__ bool warp_wait_for(uint64_t *b, uint32_t parity, Shared *sh) { return __all_sync(~0u, wait_for(b, parity, sh)); }
// One lane of a whole warp, known as such to the compiler: tensor instructions and bulk copies issued by a lane that a comparison
// picked cost 105 clocks each and more, whatever their size; by an elected one, what the tensor cores take.
__device__ __forceinline__ bool elected()
{
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(ok));
    return ok != 0;
}
__device__ __forceinline__ void bulk_copy(void *dst, const void *src, uint32_t bytes, uint64_t *bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_addr(dst)), "l"(src), "r"(bytes), "r"(smem_addr(bar)) : "memory");
}
// A box of 64 values x p.box rows; the barrier may be the other CTA's of the pair.  k is a multiple of 64 (128 bytes).
template <int CTAS> __device__ __forceinline__ void box_copy(uint32_t dst, const CUtensorMap *map, int k, int row, uint32_t bar)
{
    if constexpr (CTAS == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(k), "r"(row), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(k), "r"(row), "r"(bar) : "memory");
}
// Arrives at the barrier, in both CTAs of a pair, when the products issued so far are done.
template <int CTAS> __device__ __forceinline__ void commit(uint64_t *bar)
{
    if constexpr (CTAS == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_addr(bar)), "h"(uint16_t(3)) : "memory");
}
template <int CTAS> __device__ __forceinline__ void mma(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    if constexpr (CTAS == 1)
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
template <int CTAS> __device__ __forceinline__ void tmem_alloc(uint32_t *to)
{
    if constexpr (CTAS == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(to)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(to)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
}
// After giving up: the copies that are under way end before the CTA does.
__device__ __noinline__ void give_copies_time()
{
    for (int i = 0; i < 10000; ++i) __nanosleep(100);
}
template <int CTAS> __device__ __forceinline__ void tmem_free(uint32_t at)
{
    if constexpr (CTAS == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(at) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(at) : "memory");
}
// Shared-memory descriptor of a K-major operand whose rows of 64 values (128 bytes) are swizzled in groups of 8 (1024 bytes).
__device__ __forceinline__ uint64_t operand(uint32_t addr)
{
    return uint64_t((addr & 0x3ffff) >> 4) | (uint64_t(1) << 16) | (uint64_t(1024 >> 4) << 32) | (uint64_t(1) << 46) | (uint64_t(2) << 61);
}
__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void st_tmem32(uint32_t at, const uint32_t (&v)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(at),
                 "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]),
                 "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]),
                 "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
                 : "memory");
}
__device__ __forceinline__ void ld_tmem16(uint32_t (&v)[16], uint32_t at)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]),
                   "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(at)
                 : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// What a 16-bit weight is made of, from the pairs of a masked nibble and the scale S 2^-e, below 2^16 and near it for the row's largest (w4_pack.cu):
//   one step   FMA(pair, scale FACTOR, scale -8 UNIT): one step of q becomes scale UNIT.  For bf16 without zero points, where 8 S is exact
//   two steps  MUL(FMA(pair, BIG or SMALL, -z STEP), scale): (q - z) STEP first, exactly.  With zero points S z need not be exact; and in f16 the scale
//              has to stay at the upper end of the range (one step leaves UNIT at 2^-10 of it, where scales below a sixteenth of the row's largest
//              make subnormal weights): so it does down to 2^-20 of the row's largest
//   and for f16 scales beside bf16 rows, whose 11 bits are two bf16 numbers of 8 and 3 (the product of the second is exact), d = (q - z) STEP:
//              FMA(d, first, MUL(d, second)), so that the weight is rounded once
// Nibbles in bits 4..7 take a sixteenth of the factor.
template <bool BF16> struct Num;
template <> struct Num<true> {
    // a masked nibble is q 2^-133
    static constexpr float UNIT = 1.f / 4194304, STEP = 1.f / 64;
    static constexpr uint32_t BIG_FACTOR = 0x77007700, SMALL_FACTOR = 0x75007500, MINUS_EIGHT = 0xb600b600;       // 2^111, 2^107, -2^-19
    static constexpr uint32_t BIG = 0x7f007f00, SMALL = 0x7d007d00;                                               // 2^127, 2^123
    static __device__ __forceinline__ uint32_t both(float v)
    {
        const uint32_t b = __bfloat16_as_ushort(__float2bfloat16_rn(v));
        return b | (b << 16);
    }
    static __device__ __forceinline__ uint32_t fma(uint32_t a, uint32_t b, uint32_t c)
    {
        uint32_t d;
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
        return d;
    }
    static __device__ __forceinline__ uint32_t mul(uint32_t a, uint32_t b)
    {
        uint32_t d;
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
        return d;
    }
};
template <> struct Num<false> {
    // a masked nibble is q 2^-24
    static constexpr float UNIT = 0.f, STEP = 1.f / 512;                                                          // always two steps
    static constexpr uint32_t BIG_FACTOR = 0, SMALL_FACTOR = 0, MINUS_EIGHT = 0;
    static constexpr uint32_t BIG = 0x78007800, SMALL = 0x68006800;                                               // 2^15, 2^11
    static __device__ __forceinline__ uint32_t both(float v)
    {
        const uint32_t b = __half_as_ushort(__float2half_rn(v));
        return b | (b << 16);
    }
    static __device__ __forceinline__ uint32_t fma(uint32_t a, uint32_t b, uint32_t c)
    {
        uint32_t d;
        asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
        return d;
    }
    static __device__ __forceinline__ uint32_t mul(uint32_t a, uint32_t b)
    {
        uint32_t d;
        asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
        return d;
    }
};

__device__ __forceinline__ float scale_value(uint32_t bits, bool bf16)
{
    return bf16 ? __uint_as_float(bits << 16) : __half2float(__ushort_as_half(uint16_t(bits)));
}


// Two values as 16 bits each, the first in the low half.
__device__ __forceinline__ uint32_t two_16_bits(float lo, float hi, bool bf16)
{
    uint32_t d;
    if (bf16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}

enum { PLAIN = 0, SPLIT = 1, EXPERTS = 2 };
// How weights are made: without zero points; with them; of f16 scales for bf16 rows, with or without zero points.
enum { EIGHT = 0, ZEROS = 1, FINE = 2 };

// BF16: x and weights are bf16, else f16.
template <bool BF16, int WEIGHTS, int CTAS, int MODE> __global__ void __launch_bounds__(THREADS, 1) w4_tile_kernel(const Args p, const __grid_constant__ CUtensorMap map)
{
    using N = Num<BF16>;
    constexpr bool TWO_STEPS = WEIGHTS != EIGHT || !BF16;
    constexpr float BACK = 1.f / (TWO_STEPS ? N::STEP : N::UNIT);             // what a sum is multiplied by beside 2^e
    extern __shared__ uint8_t raw[];
    __shared__ Shared sh;
    uint8_t *const ring = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);      // the swizzle's groups start at multiples of 1024; the same place in every CTA
    uint8_t *const weight_ring = ring + p.x_stages * p.x_bytes;
    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;     // the shuffle: known to be one value per warp
    const int side = CTAS == 2 ? blockIdx.x & 1 : 0, splits = MODE == SPLIT ? int(gridDim.y) : 1;
    const int kb0 = MODE == SPLIT ? int(p.depth_tiles * blockIdx.y / splits) : 0;
    const int depth = (MODE == SPLIT ? int(p.depth_tiles * (blockIdx.y + 1) / splits) : int(p.depth_tiles)) - kb0;
    const int columns = (p.row_tiles + CTAS - 1) / CTAS;                      // tiles of results side by side

    after_work_before();
    // tiles of results: those of one run of rows of x side by side, so that its CTAs share the rows in L2
    const int runs = MODE == EXPERTS ? *p.table_size : (p.m + p.tokens - 1) / p.tokens;
    const int first = int(blockIdx.x) / CTAS, stride = int(gridDim.x) / CTAS, tile_count = columns * runs;
    const int mine = first < tile_count ? (tile_count - first + stride - 1) / stride : 0;
    struct Tile {
        int64_t nt;              // this CTA's tile of 128 rows of weights, over all matrices; past the last: the last again, not written
        int row0;                // its first row in its matrix
        int t0;                  // first row of x
        int count, tokens;       // rows of x, and what they are padded to
    };
    auto tile_at = [&](int i) {
        const int at = first + i * stride, run = at / columns, rt = (at - run * columns) * CTAS + side;
        Tile t;
        t.nt = rt < p.row_tiles ? rt : p.row_tiles - 1;
        if (MODE == EXPERTS) {
            const W4Tile e = p.table[run];
            t.nt += int64_t(e.expert) * p.row_tiles;
            t.t0 = e.first;
            t.count = e.count;
            t.tokens = (e.count + CTAS * STEP - 1) / (CTAS * STEP) * (CTAS * STEP);
        } else {
            t.t0 = run * p.tokens;
            t.count = p.m - t.t0 < p.tokens ? p.m - t.t0 : p.tokens;
            t.tokens = p.tokens;
        }
        t.row0 = rt * kW4Rows;
        return t;
    };
    // the weights of the first tile's first steps are on their way before anything else is
    const auto weights = [&](int64_t tile, int s) {
        bar_expect(&sh.full_w[s], uint32_t(p.tile_bytes));
        bulk_copy(weight_ring + s * p.tile_bytes, p.packed + tile * p.tile_bytes, uint32_t(p.tile_bytes), &sh.full_w[s]);
    };
    const int ahead = mine == 0 ? 0 : depth < RING ? depth : RING;
    if (warp == WEIGHT_WARP && elected()) {
        for (int i = 0; i < RING; ++i) {
            bar_init(&sh.full_w[i], 1);
            bar_init(&sh.empty_w[i], 4);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        if (ahead > 0) {
            const int64_t from = tile_at(0).nt * p.depth_tiles + kb0;
            for (int j = 0; j < ahead; ++j) weights(from + j, j);
        }
    }
    if (warp == X_WARP && elected()) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map) : "memory");
        for (int i = 0; i < RING; ++i) {
            bar_init(&sh.ready[i], 4 * CTAS + 1);
            bar_init(&sh.used[i], 1);
        }
        bar_init(&sh.done, 1);
        bar_init(&sh.d_free, TURN_WARPS * CTAS);
        sh.dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == MMA_WARP) tmem_alloc<CTAS>(&sh.tmem);
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (CTAS == 2) cluster_barrier();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = sh.tmem;

    if (warp < TURN_WARPS) {
        const int group = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t lanes = tmem + (uint32_t((warp & 3) * 32) << 16);
        const int place = W4Layout::row_place(r);
        const uint32_t ready = of_rank(sh.ready, CTAS == 2 ? 0 : cluster_rank()), d_free = of_rank(&sh.d_free, CTAS == 2 ? 0 : cluster_rank());
        const bool bf16_out = p.out_type == STRASSEN_BF16;

        // ---- results of tile i; with splits this CTA's part of the sums stays in the ring ------------------------------------
        auto read_back = [&](int i) {
            const Tile t = tile_at(i);
            const int row = t.row0 + r;
            const float back = BACK * p.exponents[t.nt * kW4Rows + r];
            // where this group's rows of x (16 of every 64) go and their scales, two a lane, read before the wait
            int place[2] = {0, 0};
            float scale[2] = {1.f, 1.f};
            if (MODE != SPLIT) {
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int at = 16 * group + 128 * b + (lane >> 4) * 64 + (lane & 15);
                    if (at < t.count) {
                        place[b] = t.t0 + at;
                        if (MODE == EXPERTS) place[b] = p.order[place[b]];
                        if (p.x_scale) scale[b] = p.x_scale[MODE == EXPERTS ? place[b] / p.scale_div : place[b]];
                    }
                }
            }
            if (!warp_wait_for(&sh.done, i & 1, &sh)) return false;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const int end = MODE == SPLIT ? t.tokens : t.count;
            // D is free for the products of the next tile as soon as its last rows are in registers
            const auto free_d = [&] {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) bar_arrive_at(d_free);
            };
            if (16 * group >= end) free_d();
            // Not unrolled, and in one place in the code: it is run once a tile, and its instructions, fetched anew each time, are what
            // it takes (2000 clocks for 16 rows of x; 2048 tokens of 64 experts: 151 us unrolled, 147 so).
#pragma unroll 1
            for (int q = 0; q < TOKENS / (16 * GROUPS); ++q) {
                const int c = 16 * group + 16 * GROUPS * q;
                if (c >= end) break;
                uint32_t v[16];
                ld_tmem16(v, lanes + c);
                if (c + 16 * GROUPS >= end) free_d();
                if (MODE == SPLIT) {
                    float *sums = reinterpret_cast<float *>(ring) + c * kW4Rows + r;
#pragma unroll
                    for (int b = 0; b < 16; ++b) sums[b * kW4Rows] = __uint_as_float(v[b]);
                    continue;
                }
                const int left = t.count - c;            // rows of x from here on
                const int places = q & 2 ? place[1] : place[0];
                const float scales = q & 2 ? scale[1] : scale[0];
                int to[16];                              // where they go
                float y[16];
#pragma unroll
                for (int b = 0; b < 16; ++b) {
                    to[b] = MODE == EXPERTS ? __shfl_sync(~0u, places, 16 * (q & 1) + b) : t.t0 + c + b;
                    y[b] = __uint_as_float(v[b]) * back;
                    if (p.x_scale) y[b] *= __shfl_sync(~0u, scales, 16 * (q & 1) + b);
                }
                if (MODE == EXPERTS && p.out_type == STRASSEN_F32) {
#pragma unroll
                    for (int b = 0; b < 16; ++b)
                        if (b < left && row < p.n) static_cast<float *>(p.out)[to[b] * p.ldo + row] = y[b];
                } else if (p.out_pairs && row - r + kW4Rows <= p.n) {
                    // neighbouring rows of weights are neighbours in memory: two lanes trade halves so that each writes two of them in one
                    // word, the even lane for one row of x, the odd lane for the next
                    const int odd = lane & 1;
                    uint16_t *const out = static_cast<uint16_t *>(p.out) + (row & ~1);
#pragma unroll
                    for (int b = 0; b < 16; b += 2) {
                        const uint32_t own = two_16_bits(y[b], y[b + 1], bf16_out), got = __shfl_xor_sync(~0u, own, 1);
                        const uint32_t word = odd ? __byte_perm(got, own, 0x7632) : __byte_perm(own, got, 0x5410);
                        if (b + odd < left) *reinterpret_cast<uint32_t *>(out + (odd ? to[b + 1] : to[b]) * p.ldo) = word;
                    }
                } else if (row < p.n) {
#pragma unroll
                    for (int b = 0; b < 16; ++b)
                        if (b < left) static_cast<uint16_t *>(p.out)[to[b] * p.ldo + row] = uint16_t(two_16_bits(y[b], 0.f, bf16_out));
                }
            }
            return true;
        };

        // ---- weights to tensor memory: every GROUPS-th of the 128-deep tiles of all tiles of results ------------------------------
        int read = 0;            // tiles of results read back
        int i = group / depth, j = group % depth;        // tile of results, and its step
        int a = group;                                   // A buffer (a_buffers >= GROUPS)
        int g = group;
        bool alive = true;
        while (alive) {
            // the first A buffers of a tile are filled before the tile before it is read back
            if (i >= mine ? read < mine : read < i && (j >= GROUPS - 1 || read < i - 1)) {
                alive = read_back(read++);
                continue;
            }
            if (i >= mine) break;
            const int s = g % RING;
            if (!warp_wait_for(&sh.full_w[s], (g / RING) & 1, &sh)) break;
            const uint8_t *stage = weight_ring + s * p.tile_bytes;
            uint32_t w[4][4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint4 u = *reinterpret_cast<const uint4 *>(stage + W4Layout::chunk_place(r, c));
                w[c][0] = u.x;
                w[c][1] = u.y;
                w[c][2] = u.z;
                w[c][3] = u.w;
            }
            uint32_t sc[4], z[4];                    // of each word's group
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                if (b & ((1 << p.group_shift) - 1)) {
                    sc[b] = sc[b - 1];
                    z[b] = z[b - 1];
                } else {
                    const int at = (b >> p.group_shift) * kW4Rows + place;
                    sc[b] = *reinterpret_cast<const uint16_t *>(stage + kW4NibbleBytes + at * 2);
                    z[b] = WEIGHTS == ZEROS || (WEIGHTS == FINE && p.has_zeros) ? stage[p.zero_off + at] : 8;
                }
            }
            __syncwarp();
            if (lane == 0) bar_arrive(&sh.empty_w[s]);
            uint32_t v[2][32];                       // column 16 w + 4 c + pair
            uint32_t big = 0, small = 0, minus = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                if (!(b & ((1 << p.group_shift) - 1))) {
                    if (WEIGHTS == FINE) {
                        const float scale = scale_value(sc[b], false);
                        big = N::both(scale);
                        small = N::both(scale - __uint_as_float(big & 0xffff0000u));
                    } else if (p.scale_bf16 == BF16) {
                        big = sc[b] | sc[b] << 16;
                    } else {
                        big = N::both(scale_value(sc[b], p.scale_bf16));
                    }
                    if (TWO_STEPS) {
                        minus = N::both(-N::STEP * float(z[b]));
                    } else {
                        small = N::mul(big, N::SMALL_FACTOR);
                        minus = N::mul(big, N::MINUS_EIGHT);
                        big = N::mul(big, N::BIG_FACTOR);
                    }
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t *const to = v[b >> 1] + 16 * (b & 1) + 4 * c;
                    const uint32_t u = w[c][b], uu = u >> 8;
                    if (TWO_STEPS) {
                        const auto weight = [&](uint32_t d) { return WEIGHTS == FINE ? N::fma(d, big, N::mul(d, small)) : N::mul(d, big); };
                        to[0] = weight(N::fma(u & 0x000f000f, N::BIG, minus));
                        to[1] = weight(N::fma(u & 0x00f000f0, N::SMALL, minus));
                        to[2] = weight(N::fma(uu & 0x000f000f, N::BIG, minus));
                        to[3] = weight(N::fma(uu & 0x00f000f0, N::SMALL, minus));
                    } else {
                        to[0] = N::fma(u & 0x000f000f, big, minus);
                        to[1] = N::fma(u & 0x00f000f0, small, minus);
                        to[2] = N::fma(uu & 0x000f000f, big, minus);
                        to[3] = N::fma(uu & 0x00f000f0, small, minus);
                    }
                }
            }
            // the buffer is free when the products of the step that used it are done
            const int before = g - p.a_buffers;
            if (before >= 0 && !warp_wait_for(&sh.used[before % RING], (before / RING) & 1, &sh)) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t to = lanes + 512 - (p.a_buffers - a) * A_WIDTH;
            st_tmem32(to, v[0]);
            st_tmem32(to + 32, v[1]);
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                if (CTAS == 2) bar_arrive_at(ready + 8 * s);
                else bar_arrive(&sh.ready[s]);
            }
            g += GROUPS;
            a += GROUPS;
            if (a >= p.a_buffers) a -= p.a_buffers;
            for (j += GROUPS; j >= depth; j -= depth) ++i;
        }
    } else if (warp == WEIGHT_WARP) {
        // ---- weights to shared memory -------------------------------------------------------------------------------------------
        if (elected()) {
            int g = ahead;
            bool alive = true;
            for (int i = 0; i < mine && alive; ++i) {
                const int64_t from = tile_at(i).nt * p.depth_tiles + kb0;
                for (int j = i == 0 ? ahead : 0; j < depth; ++j, ++g) {
                    if (g >= RING && !(alive = wait_for(&sh.empty_w[g % RING], (g / RING - 1) & 1, &sh))) break;
                    weights(from + j, g % RING);
                }
            }
            if (!alive) give_copies_time();
        }
    } else if (warp == X_WARP) {
        // ---- rows of x to shared memory -----------------------------------------------------------------------------------------
        if (elected()) {
            const uint32_t ring_at = smem_addr(ring);
            int g = 0, at = 0;                       // step, and its place in the ring of rows of x
            bool alive = true;
            for (int i = 0; i < mine && alive; ++i) {
                const Tile t = tile_at(i);
                const int rows = t.tokens / CTAS, row = t.t0 + side * rows, brought = (rows + p.box - 1) / p.box * p.box;
                for (int j = 0; j < depth; ++j, ++g) {
                    const int before = g - p.x_stages, s = g % RING;
                    if (before >= 0 && !(alive = wait_for(&sh.used[before % RING], (before / RING) & 1, &sh))) break;
                    const uint32_t ready = CTAS == 2 ? of_rank(&sh.ready[s], 0) : smem_addr(&sh.ready[s]), to = ring_at + at * p.x_bytes;
                    if (side == 0) bar_expect(&sh.ready[s], uint32_t(brought * CTAS) * 256);       // of both CTAs
                    const int k = (kb0 + j) * kW4Depth;
                    for (int b = 0; b < rows; b += p.box) {
                        box_copy<CTAS>(to + b * 128, &map, k, row + b, ready);
                        box_copy<CTAS>(to + brought * 128 + b * 128, &map, k + 64, row + b, ready);
                    }
                    at = at + 1 == p.x_stages ? 0 : at + 1;
                }
            }
            // the last products' arrivals at `used`, which may come from the other CTA, are here before this one leaves
            for (int before = g > p.x_stages ? g - p.x_stages : 0; before < g && alive; ++before) alive = wait_for(&sh.used[before % RING], (before / RING) & 1, &sh);
            if (!alive) give_copies_time();
        }
    } else if (side == 0 && elected()) {
        // ---- products -----------------------------------------------------------------------------------------------------------
        constexpr uint32_t format = BF16 ? 1 : 0;
        int g = 0, at = 0, a = 0;
        bool alive = true, here = false;         // here: the next step was found ready while products were being issued
        for (int i = 0; i < mine && alive; ++i) {
            const int tokens = tile_at(i).tokens, brought = (tokens / CTAS + p.box - 1) / p.box * p.box;
            const uint32_t idesc = (1u << 4) | (format << 7) | (format << 10) | (uint32_t(tokens >> 3) << 17) | (uint32_t(128 * CTAS >> 4) << 24);
            if (i > 0 && !(alive = wait_for(&sh.d_free, (i - 1) & 1, &sh))) break;
            for (int j = 0; j < depth; ++j, ++g) {
                if (!here && !(alive = wait_for(&sh.ready[g % RING], (g / RING) & 1, &sh))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t x_addr = smem_addr(ring) + at * p.x_bytes;
                const uint64_t b0 = operand(x_addr), b1 = operand(x_addr + brought * 128);
                const uint32_t from = tmem + 512 - (p.a_buffers - a) * A_WIDTH;
                here = bar_test(&sh.ready[(g + 1) % RING], ((g + 1) / RING) & 1);
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) mma<CTAS>(tmem, from + kk * 8, (kk < 4 ? b0 : b1) + (kk & 3) * 2, idesc, j > 0 || kk > 0);
                commit<CTAS>(&sh.used[g % RING]);
                at = at + 1 == p.x_stages ? 0 : at + 1;
                a = a + 1 == p.a_buffers ? 0 : a + 1;
            }
            commit<CTAS>(&sh.done);
        }
    }
    __syncwarp();
    __syncthreads();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    if (CTAS == 2 || MODE == SPLIT) cluster_barrier();       // the pair is through with its shared and tensor memory; the sums of all splits are in place
    if (MODE == SPLIT) {
        const Tile t = mine > 0 ? tile_at(0) : Tile{};
        // CTA y of the cluster writes every splits-th row of x, a thread four rows of weights
        if (mine > 0 && threadIdx.x < TURN_WARPS * 32) {
            const int c = (threadIdx.x & 31) * 4;
            const float4 back = *reinterpret_cast<const float4 *>(p.exponents + t.nt * kW4Rows + c);
            const bool bf16_out = p.out_type == STRASSEN_BF16;
            const bool wide = p.out_pairs && p.ldo % 4 == 0 && reinterpret_cast<uintptr_t>(p.out) % 8 == 0 && t.row0 + c + 4 <= p.n;
            for (int i = int(blockIdx.y) + splits * int(threadIdx.x / 32); i < t.count; i += splits * TURN_WARPS) {
                float4 part[MAX_SPLITS];
#pragma unroll
                for (int b = 0; b < MAX_SPLITS; ++b)
                    if (b < splits) part[b] = remote_float4(of_address(smem_addr(ring) + uint32_t(i * kW4Rows + c) * 4, uint32_t(b)));
                float4 y = part[0];
#pragma unroll
                for (int b = 1; b < MAX_SPLITS; ++b)
                    if (b < splits) {
                        y.x += part[b].x;
                        y.y += part[b].y;
                        y.z += part[b].z;
                        y.w += part[b].w;
                    }
                const float factor = p.x_scale ? BACK * p.x_scale[t.t0 + i] : BACK;
                const uint32_t lo = two_16_bits(y.x * back.x * factor, y.y * back.y * factor, bf16_out), hi = two_16_bits(y.z * back.z * factor, y.w * back.w * factor, bf16_out);
                uint16_t *out = static_cast<uint16_t *>(p.out) + (t.t0 + i) * p.ldo + t.row0 + c;
                if (wide) {
                    *reinterpret_cast<uint2 *>(out) = make_uint2(lo, hi);
                } else {
#pragma unroll
                    for (int b = 0; b < 4; ++b)
                        if (t.row0 + c + b < p.n) out[b] = uint16_t((b < 2 ? lo : hi) >> (16 * (b & 1)));
                }
            }
        }
        __syncwarp();
        cluster_barrier();           // no CTA leaves while another reads its sums
    }
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == MMA_WARP) tmem_free<CTAS>(tmem);
}

// Rows of x in 16 bits, one after another, `width` (a multiple of 8) values apart, zeros past the inner size: e4m3 becomes f16, exactly.
struct RowsArgs {
    const char *x;
    int64_t ldx_bytes, rows, k, width;
    bool e4m3;
    uintptr_t x_end;         // of the memory of x
    uint16_t *out;
    // experts: the pair of each row in order, pairs per row of x; the pairs' ids, to write zeros to the results of those without an expert
    const int *order, *count, *ids;
    int per_row, experts;
    uint16_t *results;       // NULL: not those
    int64_t ldo, n;
};

// A warp has a row's piece of PIECES x 256 values at a time, all its loads under way at once: what a row's place costs (order, divisions) is paid once for them.
// 16384 rows of 2048 out of 2048 in e4m3: 17.6 us, 23 us with a division for every 8 values.
constexpr int PIECES = 4;
__global__ void __launch_bounds__(256) rows_kernel(const RowsArgs p)
{
    after_work_before();
    const int64_t count = p.count ? int64_t(*p.count) : p.rows;
    const int warp = int(threadIdx.x >> 5), lane = int(threadIdx.x & 31);
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p.x);
    for (int64_t i = int64_t(blockIdx.x) * 8 + warp; i < count; i += int64_t(gridDim.x) * 8) {
        const char *const x = p.x + (p.order ? int64_t(p.order[i] / p.per_row) : i) * p.ldx_bytes;
        uint16_t *const out = p.out + i * p.width;
        for (int64_t piece = blockIdx.y; piece * (PIECES * 256) < p.width; piece += gridDim.y) {
            const int64_t c0 = piece * (PIECES * 256) + lane * 8;
            uint4 v[PIECES];
            if (p.e4m3) {
                uint2 u[PIECES];
#pragma unroll
                for (int j = 0; j < PIECES; ++j)
                    if (c0 + j * 256 < p.width) u[j] = load_bytes8(reinterpret_cast<const uint8_t *>(x), c0 + j * 256, p.k, lo, p.x_end);
#pragma unroll
                for (int j = 0; j < PIECES; ++j) {
                    uint32_t w[4];
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t((b < 2 ? u[j].x : u[j].y) >> (16 * (b & 1))), __NV_E4M3);
                        w[b] = uint32_t(h.x) | (uint32_t(h.y) << 16);
                    }
                    v[j] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < PIECES; ++j)
                    if (c0 + j * 256 < p.width) {
                        Words<__half> w;
                        load(w, reinterpret_cast<const __half *>(x), c0 + j * 256, p.k, lo, p.x_end);
                        v[j] = make_uint4(w.w[0], w.w[1], w.w[2], w.w[3]);
                    }
            }
#pragma unroll
            for (int j = 0; j < PIECES; ++j)
                if (c0 + j * 256 < p.width) *reinterpret_cast<uint4 *>(out + c0 + j * 256) = v[j];
        }
    }
    if (p.results && *p.count < p.rows)
        for (int64_t i = (int64_t(blockIdx.y) * gridDim.x + blockIdx.x) * 8 + warp; i < p.rows; i += int64_t(gridDim.x) * gridDim.y * 8)
            if (p.ids[i] < 0 || p.ids[i] >= p.experts)
                for (int64_t c = lane; c < p.n; c += 32) p.results[i * p.ldo + c] = 0;
}

// Pairs (a token and one of its ids) in order of their experts, pairs of one expert in their own order: CTA e counts the ids of all experts,
// and with them knows where its own begin.  Every CTA reads all ids, a few kilobytes from L2, and nothing has to be waited for.
// 16384 ids of 64 experts: 7 us, 17 us with one load at a time.
__global__ void __launch_bounds__(1024) order_kernel(const int *ids, int pairs, int experts, int most, int *order, int *count, int *table_size, W4Tile *table)
{
    __shared__ int counts[kMostExperts], part[2][32];
    __shared__ int start, tiles;
    const int e = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    after_work_before();
    for (int i = threadIdx.x; i < experts; i += blockDim.x) counts[i] = 0;
    __syncthreads();
    // a warp has neighbouring ids, 32 * EACH of them at a time, whose loads are all under way at once
    constexpr int EACH = 16;
    const int share = (pairs + 32 * 32 - 1) / (32 * 32) * 32, from = warp * share, to = from + share < pairs ? from + share : pairs;
    int own = 0;
    for (int i = from; i < to; i += 32 * EACH) {
        int id[EACH];
#pragma unroll
        for (int j = 0; j < EACH; ++j) id[j] = i + 32 * j + lane < to ? ids[i + 32 * j + lane] : -1;
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            if (id[j] >= 0 && id[j] < experts) atomicAdd(&counts[id[j]], 1);
            own += __popc(__ballot_sync(~0u, id[j] == e));
        }
    }
    __syncthreads();
    // rows and tiles of rows before this expert, and of all
    int before[2] = {0, 0}, all[2] = {0, 0};
    if (int(threadIdx.x) < experts) {
        const int n = counts[threadIdx.x], t = (n + most - 1) / most;
        all[0] = n;
        all[1] = t;
        if (int(threadIdx.x) < e) {
            before[0] = n;
            before[1] = t;
        }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        before[b] = __reduce_add_sync(~0u, before[b]);
        all[b] = __reduce_add_sync(~0u, all[b]);
        if (lane == 0) part[b][warp] = before[b];
    }
    __syncthreads();
    if (warp == 0) {
        const int rows = __reduce_add_sync(~0u, part[0][lane]), t = __reduce_add_sync(~0u, part[1][lane]);
        if (lane == 0) {
            start = rows;
            tiles = t;
        }
    }
    __syncthreads();
    if (lane == 0) {
        part[0][warp] = all[0];
        part[1][warp] = all[1];
    }
    __syncthreads();
    if (e == 0 && warp == 0) {
        const int rows = __reduce_add_sync(~0u, part[0][lane]), t = __reduce_add_sync(~0u, part[1][lane]);
        if (lane == 0) {
            *count = rows;
            *table_size = t;
        }
    }
    // rows of x: as few tiles as hold them, evenly filled
    const int mine = counts[e], runs = (mine + most - 1) / most, even = runs ? (mine + runs - 1) / runs : 0;
    for (int i = threadIdx.x; i < runs; i += blockDim.x) table[tiles + i] = {e, start + i * even, mine - i * even < even ? mine - i * even : even, 0};
    __syncthreads();
    // its own ids' places: after those of the warps before it, of its ids before and of the lanes below
    if (lane == 0) part[0][warp] = own;
    __syncthreads();
    int at = start + __reduce_add_sync(~0u, lane < warp ? part[0][lane] : 0);
    if (own > 0)
        for (int i = from; i < to; i += 32 * EACH) {
            int id[EACH];
#pragma unroll
            for (int j = 0; j < EACH; ++j) id[j] = i + 32 * j + lane < to ? ids[i + 32 * j + lane] : -1;
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                const uint32_t those = __ballot_sync(~0u, id[j] == e);
                if (id[j] == e) order[at + __popc(those & ((1u << lane) - 1))] = i + 32 * j + lane;
                at += __popc(those);
            }
        }
}

// out_t = sum_j weights_tj part_tj, in the order of j; pairs without an expert add nothing.
__global__ void __launch_bounds__(256) weighted_sum_kernel(const float *part, const int *ids, const float *weights, int64_t tokens, int top, int experts, int64_t n, int64_t width, void *out, int64_t ldo, bool bf16)
{
    after_work_before();
    const int64_t chunks = width / 4, total = tokens * chunks;
    for (int64_t e = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; e < total; e += int64_t(gridDim.x) * blockDim.x) {
        const int64_t t = e / chunks, c = (e - t * chunks) * 4;
        float y[4] = {0.f, 0.f, 0.f, 0.f};
        for (int j = 0; j < top; ++j) {
            const int id = ids[t * top + j];
            if (id < 0 || id >= experts) continue;
            const float w = weights[t * top + j];
            const float4 v = *reinterpret_cast<const float4 *>(part + (t * top + j) * width + c);
            y[0] += w * v.x;
            y[1] += w * v.y;
            y[2] += w * v.z;
            y[3] += w * v.w;
        }
#pragma unroll
        for (int b = 0; b < 4; ++b)
            if (c + b < n) static_cast<uint16_t *>(out)[t * ldo + c + b] = uint16_t(two_16_bits(y[b], 0.f, bf16));
    }
}

constexpr int kDynamicLimit = 225 * 1024;         // of 227 KB: the rest holds Shared

// What a launch is made of beside the kernel's arguments.
struct Shape {
    int ctas, mode, columns, splits, bytes;
};

template <bool BF16, int WEIGHTS, int CTAS, int MODE> cudaError_t launch_one(const Args &p, const CUtensorMap &map, const Shape &shape, cudaStream_t stream)
{
    static std::atomic<uint64_t> opted_in{0};        // devices that this kernel has been given its shared memory on
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (!(opted_in.load(std::memory_order_relaxed) >> dev & 1)) {
        e = cudaFuncSetAttribute(w4_tile_kernel<BF16, WEIGHTS, CTAS, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, kDynamicLimit);
        if (e != cudaSuccess) return e;
        opted_in.fetch_or(uint64_t(1) << dev, std::memory_order_relaxed);
    }
    return launch_after(w4_tile_kernel<BF16, WEIGHTS, CTAS, MODE>, dim3(unsigned(shape.columns * CTAS), unsigned(shape.splits)), dim3(THREADS), size_t(shape.bytes), stream, dim3(CTAS, unsigned(shape.splits)), p, map);
}

template <bool BF16, int WEIGHTS> cudaError_t launch_shape(const Args &p, const CUtensorMap &map, const Shape &s, cudaStream_t stream)
{
    if (s.mode == EXPERTS) return launch_one<BF16, WEIGHTS, 2, EXPERTS>(p, map, s, stream);
    if (s.ctas == 2) return launch_one<BF16, WEIGHTS, 2, PLAIN>(p, map, s, stream);
    return s.mode == SPLIT ? launch_one<BF16, WEIGHTS, 1, SPLIT>(p, map, s, stream) : launch_one<BF16, WEIGHTS, 1, PLAIN>(p, map, s, stream);
}

// How many clusters of `size` of these CTAs, one to an SM, the current device holds at a time: less than SMs / size, since a cluster lies within
// one group of SMs (33 of 4 and 15 of 8 on a B200 with 148 SMs).  Devices differ in how their SMs are grouped, so each has its own answer, and with it
// its own order of sums, whichever device was used first.
int clusters_of(int size)
{
    constexpr int DEVICES = 64;              // as many as the entry points take
    static std::atomic<int> known[DEVICES][MAX_SPLITS + 1];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= DEVICES) return 0;
    if ((n = known[dev][size].load(std::memory_order_relaxed)) > 0) return n;
    const auto kernel = w4_tile_kernel<true, EIGHT, 1, SPLIT>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kDynamicLimit) != cudaSuccess) return 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(64, unsigned(size));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = kDynamicLimit;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 1;
    attr[0].val.clusterDim.y = unsigned(size);
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) return 0;
    known[dev][size].store(n, std::memory_order_relaxed);
    return n;
}

using EncodeTiled = decltype(&cuTensorMapEncodeTiled);

// The driver's function that fills a tensor map, looked up once.
EncodeTiled encode_tiled()
{
    static std::atomic<EncodeTiled> found{nullptr};
    EncodeTiled f = found.load(std::memory_order_acquire);
    if (!f) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) return nullptr;
        f = reinterpret_cast<EncodeTiled>(p);
        found.store(f, std::memory_order_release);
    }
    return f;
}

bool map_takes(const W4Args &a)
{
    return a.type != STRASSEN_E4M3 && reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && a.ldx % 8 == 0;
}

RowsArgs rows_args(const W4Args &a, void *to)
{
    const int size = a.type == STRASSEN_E4M3 ? 1 : 2;
    RowsArgs r = {};
    r.x = static_cast<const char *>(a.x);
    r.ldx_bytes = a.ldx * size;
    r.rows = a.m;
    r.k = a.lay.k;
    r.width = (a.lay.k + 7) / 8 * 8;
    r.e4m3 = a.type == STRASSEN_E4M3;
    r.x_end = reinterpret_cast<uintptr_t>(a.x) + uintptr_t(((a.ids && a.each ? a.m * a.top : a.m) - 1) * r.ldx_bytes + a.lay.k * size);
    r.out = static_cast<uint16_t *>(to);
    r.per_row = 1;
    return r;
}

cudaError_t launch_rows(const RowsArgs &r, int sm_count, cudaStream_t stream)
{
    const int64_t pieces = (r.width + PIECES * 256 - 1) / (PIECES * 256), y = pieces < 65535 ? pieces : 65535;
    const int64_t blocks = (r.rows + 7) / 8, most = (int64_t(sm_count) * 32 + y - 1) / y;
    return launch_after(rows_kernel, dim3(unsigned(blocks < most ? blocks : most), unsigned(y)), dim3(256), 0, stream, dim3(1, 1), r);
}

// What does not depend on how the rows of x are cut into tiles.
Args common_args(const W4Args &a)
{
    Args p = {};
    p.packed = a.packed;
    p.exponents = reinterpret_cast<const float *>(a.packed + a.lay.exponent_off);
    p.x_scale = a.x_scale;
    p.out = a.out;
    p.n = int(a.lay.n);
    p.ldo = a.ldo;
    p.depth_tiles = a.lay.depth_tiles;
    p.row_tiles = int(a.lay.row_tiles);
    p.group_shift = a.lay.group == 32 ? 0 : a.lay.group == 64 ? 1 : 2;
    p.tile_bytes = a.lay.tile_bytes;
    p.zero_off = a.lay.zero_off();
    p.scale_bf16 = a.lay.scale_type == STRASSEN_BF16;
    p.has_zeros = a.lay.has_zeros;
    p.out_type = a.out_type;
    p.out_pairs = reinterpret_cast<uintptr_t>(p.out) % 4 == 0 && p.ldo % 2 == 0;
    p.scale_div = 1;
    return p;
}

// Rings and shared memory for p.tokens rows of x, and the launch.
cudaError_t launch_tiles(Args p, Shape shape, const W4Args &a, const void *x, int64_t ldx, int64_t rows, cudaStream_t stream)
{
    p.x_bytes = p.tokens * 256 / shape.ctas;
    const int stages = (kDynamicLimit - 1024 - RING * p.tile_bytes) / p.x_bytes;
    p.x_stages = stages > RING ? RING : stages;
    p.a_buffers = (512 - p.tokens) / A_WIDTH;
    if (p.a_buffers > RING) p.a_buffers = RING;
    static_assert((512 - TOKENS) / A_WIDTH >= GROUPS, "at least an A buffer for each group");
    static_assert((kDynamicLimit - 1024 - RING * (kW4NibbleBytes + 4 * kW4Rows * 3)) / (ALONE_TOKENS * 256) >= 3 &&
                      (kDynamicLimit - 1024 - RING * (kW4NibbleBytes + 4 * kW4Rows * 3)) / (TOKENS * 128) >= 3,
                  "rows of x three steps deep at least");
    shape.bytes = p.x_stages * p.x_bytes + RING * p.tile_bytes;
    if (shape.mode == SPLIT && shape.bytes < p.tokens * kW4Rows * 4) shape.bytes = p.tokens * kW4Rows * 4;
    shape.bytes += 1024;

    const EncodeTiled encode = encode_tiled();
    if (!encode) return cudaErrorSymbolNotFound;
    CUtensorMap map;
    const cuuint64_t dims[2] = {cuuint64_t(a.lay.k), cuuint64_t(rows)}, strides[1] = {cuuint64_t(ldx) * 2};
    const cuuint32_t box[2] = {64, cuuint32_t(p.box)}, steps[2] = {1, 1};
    if (encode(&map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void *>(x), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;
    if (a.type == STRASSEN_BF16 && !p.scale_bf16) return launch_shape<true, FINE>(p, map, shape, stream);
    if (a.type == STRASSEN_BF16) return a.lay.has_zeros ? launch_shape<true, ZEROS>(p, map, shape, stream) : launch_shape<true, EIGHT>(p, map, shape, stream);
    return a.lay.has_zeros ? launch_shape<false, ZEROS>(p, map, shape, stream) : launch_shape<false, EIGHT>(p, map, shape, stream);
}

// Workspace of the products of experts: the order and its tables, the rows of x in order, and with weights the pairs' results in 32 bits.
struct ExpertsSpace {
    int64_t pairs, most_tiles;
    int tokens;              // most rows of x in a tile
    size_t count_off, table_off, rows_off, part_off, bytes;
    int64_t width;           // of the pairs' results
};
ExpertsSpace experts_space(const W4Args &a)
{
    constexpr int LEAST = 64;
    const auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    ExpertsSpace s;
    s.pairs = a.m * a.top;
    // Twice the average run, so that few runs take two tiles, and however uneven they are, there are at most half as many tiles again as experts: 8 of 64
    // experts of 2048 x 2048, 64 tokens 52.5 us, 53.4 with tiles of 256, whose ring holds fewer steps; 512 tokens 64.0 and 66.4; 16 tokens 51 and 50.
    const int64_t twice = (2 * s.pairs / a.lay.experts + 2 * STEP - 1) / (2 * STEP) * (2 * STEP);
    s.tokens = int(twice < LEAST ? LEAST : twice > TOKENS ? TOKENS : twice);
    s.most_tiles = s.pairs / s.tokens + (s.pairs < a.lay.experts ? s.pairs : a.lay.experts);
    s.width = (a.lay.n + 3) / 4 * 4;
    s.count_off = up(size_t(s.pairs) * 4);
    s.table_off = s.count_off + 256;
    s.rows_off = s.table_off + up(size_t(s.most_tiles) * sizeof(W4Tile));
    s.part_off = s.rows_off + up(size_t(s.pairs) * size_t((a.lay.k + 7) / 8 * 8) * 2);
    s.bytes = s.part_off + (a.weights ? up(size_t(s.pairs) * size_t(s.width) * 4) : 0);
    return s;
}

}  // namespace

int64_t w4_tiles_workspace(const W4Args &a) { return map_takes(a) ? 0 : a.m * ((a.lay.k + 7) / 8 * 8) * 2; }

cudaError_t launch_w4_tiles(const W4Args &a, int sm_count, cudaStream_t stream)
{
    const void *x = a.x;
    int64_t ldx = a.ldx;
    if (!map_takes(a)) {
        const RowsArgs r = rows_args(a, a.workspace);
        const cudaError_t e = launch_rows(r, sm_count, stream);
        if (e != cudaSuccess) return e;
        x = a.workspace;
        ldx = r.width;
    }
    Args p = common_args(a);
    p.m = int(a.m);
    // Single CTAs while their tiles fill no more than the GPU, pairs beyond: 4096 x 4096, 64 rows 8.8 us and 15.0 in pairs, 256 rows 13.0 and 26.0;
    // 16384 x 4096, 176 rows 24.7 and 26.4.  Rows of x: as few tiles as hold them, evenly filled.
    Shape shape = {2, PLAIN, 0, 1, 0};
    if (int64_t(p.row_tiles) * ((p.m + ALONE_TOKENS - 1) / ALONE_TOKENS) <= sm_count) shape.ctas = 1;
    const int full = shape.ctas == 1 ? ALONE_TOKENS : TOKENS, runs = (p.m + full - 1) / full, even = (p.m + runs - 1) / runs;
    const int step = shape.ctas * STEP;
    p.tokens = (even + step - 1) / step * step;
    p.box = p.tokens / shape.ctas;
    const int64_t tiles = int64_t(p.row_tiles + shape.ctas - 1) / shape.ctas * runs;
    if (tiles > 0x7fffffff) return cudaErrorInvalidValue;
    // 64 rows, 4096 x 4096: 8.8 us, 13.7 with the inner dimension in one piece; 4096 x 16384: 16.6 and 44.3
    if (shape.ctas == 1)
        while (shape.splits < MAX_SPLITS && tiles <= clusters_of(shape.splits + 1) && p.depth_tiles >= 2 * (shape.splits + 1)) ++shape.splits;
    if (shape.splits > 1) shape.mode = SPLIT;
    shape.columns = int(tiles < sm_count / shape.ctas ? tiles : sm_count / shape.ctas);
    return launch_tiles(p, shape, a, x, ldx, a.m, stream);
}

int64_t w4_experts_workspace(const W4Args &a) { return int64_t(experts_space(a).bytes); }

cudaError_t launch_w4_experts_tiles(const W4Args &a, int sm_count, cudaStream_t stream)
{
    const ExpertsSpace s = experts_space(a);
    uint8_t *const ws = static_cast<uint8_t *>(a.workspace);
    int *const order = reinterpret_cast<int *>(ws), *const count = reinterpret_cast<int *>(ws + s.count_off);
    W4Tile *const table = reinterpret_cast<W4Tile *>(ws + s.table_off);
    const int experts = int(a.lay.experts);
    cudaError_t e = launch_after(order_kernel, dim3(unsigned(experts)), dim3(1024), 0, stream, dim3(1, 1), a.ids, int(s.pairs), experts, s.tokens, order, count, count + 1, table);
    if (e != cudaSuccess) return e;

    RowsArgs r = rows_args(a, ws + s.rows_off);
    r.rows = s.pairs;
    r.order = order;
    r.count = count;
    r.ids = a.ids;
    r.per_row = a.each ? 1 : int(a.top);
    r.experts = experts;
    if (!a.weights) r.results = static_cast<uint16_t *>(a.out);
    r.ldo = a.ldo;
    r.n = a.lay.n;
    e = launch_rows(r, sm_count, stream);
    if (e != cudaSuccess) return e;

    Args p = common_args(a);
    p.m = int(s.pairs);
    p.table = table;
    p.table_size = count + 1;
    p.order = order;
    p.scale_div = r.per_row;
    if (a.weights) {
        p.out = ws + s.part_off;
        p.out_type = STRASSEN_F32;
        p.ldo = s.width;
    }
    p.tokens = s.tokens;
    // Boxes as large as the runs are on average: a copy costs the thread that issues it more than the rows that it brings in beyond a run's end cost L2.
    const int64_t average = s.pairs / experts / 2;
    p.box = STEP;
    while (p.box < 64 && p.box * 2 <= average && p.box * 4 <= p.tokens) p.box *= 2;
    p.tokens = (p.tokens + 2 * p.box - 1) / (2 * p.box) * (2 * p.box);
    Shape shape = {2, EXPERTS, 0, 1, 0};
    const int64_t tiles = int64_t(p.row_tiles + 1) / 2 * s.most_tiles;
    if (tiles > 0x7fffffff) return cudaErrorInvalidValue;
    shape.columns = int(tiles < sm_count / 2 ? tiles : sm_count / 2);
    e = launch_tiles(p, shape, a, r.out, r.width, s.pairs, stream);
    if (e != cudaSuccess || !a.weights) return e;
    const int64_t blocks = (a.m * (s.width / 4) + 255) / 256, most = int64_t(sm_count) * 16;
    return launch_after(weighted_sum_kernel, dim3(unsigned(blocks < most ? blocks : most)), dim3(256), 0, stream, dim3(1, 1), reinterpret_cast<const float *>(ws + s.part_off), a.ids, a.weights, a.m, int(a.top), experts,
                        a.lay.n, s.width, a.out, a.ldo, a.out_type == STRASSEN_BF16);
}

cudaError_t read_gave_up(int *flag)
{
    cudaError_t e = cudaMemcpyFromSymbol(flag, g_gave_up, sizeof(int));
    if (e != cudaSuccess || !*flag) return e;
    const int zero = 0;
    return cudaMemcpyToSymbol(g_gave_up, &zero, sizeof(int));
}

}  // namespace strassen
