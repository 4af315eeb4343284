// Products of many rows with a matrix of 4-bit weights on the fifth-generation tensor cores.
//
// The weights are the 128-row operand of tcgen05.mma, so few rows of x make a narrow product and not a padded one:
//     D (128 rows of weights x up to 128 rows of x, 32 bits, tensor memory) += A (tensor memory) . B (shared memory)
// A CTA of 18 warps owns HALVES x 128 rows of weights and up to 128 rows of x:
//   * warp 17 streams the laid-out weights and their scales into a ring of shared memory (bulk copies);
//   * warps 0-7 turn them into 16-bit floats in registers, a thread one row of the tile, and store them to tensor memory as the
//     A operand: the weights never go back to shared memory, whose bandwidth the B operand needs;
//   * warps 8-15 bring the rows of x into the 128-byte swizzled form of the B operand, from any alignment, as 16-bit or e4m3 values, zeros past
//     the inner size and past the last row;
//   * one thread of warp 16 issues the products, 8 x HALVES for each 128 of the inner dimension;
//   * warps 0-7 read D back, multiply by the row's power of two and x's scale in 32 bits, and write through shared memory.
//
// A weight is held in 16 bits as S 2^-e (Q - Z) (e: llm.h, w4_pack.cu): this rounding, to bf16 beside bf16 rows and to f16 beside f16 and
// e4m3 rows, is the price of one product per 128-deep tile over a group's sums being scaled apart in 32 bits, which would double
// the traffic of tensor memory.  It is as large as the rounding of the result to the same type.  As in the kernel for few rows, a masked nibble
// is a subnormal number: without zero points S (q - 8) is ONE packed multiply-add, S q - 8 S, with 8 S exact; with zero points S z
// need not be exact, so (q - z) comes first, exactly, and the scale second.
//
// Where tiles are too few to fill the GPU, the CTAs of a cluster split the inner dimension and add their sums in a fixed order over
// distributed shared memory.  Every wait has a limit, after which the CTA gives up, frees its tensor memory and raises a flag (wait_for).
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "llm.h"
#include "strassen_b200.h"

namespace cg = cooperative_groups;

namespace strassen {

namespace {

enum { XBF16 = 0, XF16 = 1, XE4M3 = 2 };

constexpr int TOKENS = 128;                 // most rows of x in a tile
constexpr int DEQUANT_WARPS = 8, LOAD_WARPS = 8, THREADS = 32 * (DEQUANT_WARPS + LOAD_WARPS + 2);
constexpr int MMA_WARP = 16, COPY_WARP = 17;
constexpr int MAX_STAGES = 8;
constexpr int A_COLUMN = 256;               // first tensor-memory column of the A buffers; D is below
constexpr int A_WIDTH = 64;                 // columns of 128 rows x 128 values of 16 bits
constexpr uint32_t kWaitLimit = 1u << 22;   // tries of a wait; each may sleep for a while

// Set by a CTA that gave up on a wait; read and cleared by strassen_device_status.
__device__ int g_gave_up;

struct Args {
    const uint8_t *packed, *zeros;
    const uint16_t *scales;
    const float *exponents;
    const void *x;
    const float *x_scale;
    void *out;
    int64_t n, k, m, ldx_bytes, ldo, depth_tiles, row_tiles;
    int group_words;
    int x_align;
    int tokens;              // rows of x in a tile, a multiple of 16
    int stages, stage_bytes, x_bytes;
    int out_type;
    bool scale_bf16, out_wide;
};

struct Shared {
    uint64_t full_w[MAX_STAGES], empty_w[MAX_STAGES], full_x[MAX_STAGES], empty_x[MAX_STAGES], full_a[4], empty_a[4], done;
    uint32_t tmem;
    int dead;
    int64_t row_at[TOKENS];          // byte offset of each row of x; -1: none
};

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void bar_init(uint64_t *b, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(b)), "r"(count)); }
__device__ __forceinline__ void bar_arrive(uint64_t *b) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(b)) : "memory"); }
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
// For whole warps: the same answer in every lane, so that a warp leaves its loop as one.
__device__ __forceinline__ bool wait_for(uint64_t *b, uint32_t parity, Shared *sh);
__device__ __forceinline__ bool warp_wait_for(uint64_t *b, uint32_t parity, Shared *sh) { return __all_sync(~0u, wait_for(b, parity, sh)); }
// Waits until phase `parity` of the barrier is over.  False: the limit was reached, here or elsewhere in the CTA, and the caller leaves
// its loop; nothing that comes later waits long, and the results of the call are not valid.
__device__ __forceinline__ bool wait_for(uint64_t *b, uint32_t parity, Shared *sh)
{
    for (uint32_t i = 0; i < kWaitLimit; ++i) {
        if (bar_try(b, parity)) return true;
        if ((i & 255) == 255 && *reinterpret_cast<volatile int *>(&sh->dead)) return false;
    }
    *reinterpret_cast<volatile int *>(&sh->dead) = 1;
    g_gave_up = 1;
    return false;
}
__device__ __forceinline__ void bulk_copy(void *dst, const void *src, uint32_t bytes, uint64_t *bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_addr(dst)), "l"(src), "r"(bytes), "r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void commit(uint64_t *bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void mma(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// Shared-memory descriptor of a K-major operand whose rows of 64 values (128 bytes) are swizzled in groups of 8 (1024 bytes).
__device__ __forceinline__ uint64_t operand(uint32_t addr)
{
    return uint64_t((addr & 0x3ffff) >> 4) | (uint64_t(1) << 16) | (uint64_t(1024 >> 4) << 32) | (uint64_t(1) << 46) | (uint64_t(2) << 61);
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

// What a 16-bit weight is made of: w = FMA(nibble pair, big or small, add) without zero points, FMA(FMA(pair, BIG or SMALL, -z), scale, 0) with them.
template <bool BF16> struct Num;
template <> struct Num<true> {
    // a masked nibble is q 2^-133; the scale arrives as S 2^-e < 2; one step of q becomes S 2^-e UNIT
    static constexpr float FACTOR = 8.507059173023462e37f /* 2^126 */, UNIT = 1.f / 128, BACK = 128.f;
    static constexpr uint32_t BIG = 0x7f007f00, SMALL = 0x7d007d00;       // 2^127, 2^123: steps of 2^-6
    static constexpr float STEP = 1.f / 64;
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
    static constexpr float FACTOR = 16384.f, UNIT = 1.f / 1024, BACK = 1024.f;
    static constexpr uint32_t BIG = 0x78007800, SMALL = 0x68006800;       // 2^15, 2^11: steps of 2^-9
    static constexpr float STEP = 1.f / 512;
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

// 8 values of a row of x from k on, as 16 bits each.
template <int XT> __device__ __forceinline__ uint4 load_x(const char *row, int64_t k, int64_t size, int align)
{
    uint32_t v[4] = {0, 0, 0, 0};
    if constexpr (XT == XE4M3) {
        const uint8_t *p = reinterpret_cast<const uint8_t *>(row) + k;
        uint32_t w[2] = {0, 0};
        if (align >= 8 && k + 8 <= size) {
            const uint2 u = *reinterpret_cast<const uint2 *>(p);
            w[0] = u.x;
            w[1] = u.y;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < size) w[i >> 2] |= uint32_t(p[i]) << (8 * (i & 3));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(w[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
            v[i] = uint32_t(h.x) | (uint32_t(h.y) << 16);
        }
    } else {
        const uint16_t *p = reinterpret_cast<const uint16_t *>(row) + k;
        if (align >= 16 && k + 8 <= size) return *reinterpret_cast<const uint4 *>(p);
        if (align >= 4 && k + 8 <= size) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = reinterpret_cast<const uint32_t *>(p)[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = k + 2 * i < size ? p[2 * i] : 0, hi = k + 2 * i + 1 < size ? p[2 * i + 1] : 0;
                v[i] = lo | (hi << 16);
            }
        }
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}

template <int XT, int HALVES, bool ZEROS> __global__ void __launch_bounds__(THREADS, 1) w4_tile_kernel(const Args p)
{
    using N = Num<XT == XBF16>;
    constexpr int A_BUFFERS = HALVES == 2 ? 2 : 4, ROWS = 128 * HALVES;
    extern __shared__ uint8_t raw[];
    __shared__ Shared sh;
    uint8_t *const ring = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);      // the swizzle's groups start at multiples of 1024
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t nt0 = int64_t(blockIdx.x) * HALVES, row0 = nt0 * kW4Rows, t0 = int64_t(blockIdx.z) * p.tokens;
    const int splits = int(gridDim.y);
    const int kb0 = int(p.depth_tiles * blockIdx.y / splits), tiles = int(p.depth_tiles * (blockIdx.y + 1) / splits) - kb0;
    const int per_tile = 4 / p.group_words;                                   // groups of a 128-deep tile

    if (threadIdx.x == 0) {
        for (int i = 0; i < p.stages; ++i) {
            bar_init(&sh.full_w[i], 1);
            bar_init(&sh.empty_w[i], HALVES == 2 ? 8 : 4);
            bar_init(&sh.full_x[i], LOAD_WARPS);
            bar_init(&sh.empty_x[i], 1);
        }
        for (int i = 0; i < A_BUFFERS; ++i) {
            bar_init(&sh.full_a[i], HALVES == 2 ? 8 : 4);
            bar_init(&sh.empty_a[i], 1);
        }
        bar_init(&sh.done, 1);
        sh.dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&sh.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    for (int i = threadIdx.x; i < p.tokens; i += THREADS) sh.row_at[i] = t0 + i < p.m ? (t0 + i) * p.ldx_bytes : -1;
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = sh.tmem;
    const int w_at = p.x_bytes, s_at = w_at + HALVES * kW4TileBytes, z_at = s_at + HALVES * 1024;    // sections of a stage

    if (warp < DEQUANT_WARPS) {
        // ---- weights to tensor memory --------------------------------------------------------------------------------
        const int group = warp >> 2, r = (warp & 3) * 32 + lane;
        const int half = HALVES == 2 ? group : 0;
        const float down = 1.f / p.exponents[(nt0 + half < p.row_tiles ? nt0 + half : p.row_tiles - 1) * kW4Rows + r];      // 2^-e
        const int place = W4Layout::row_place(r);
        for (int t = HALVES == 2 ? 0 : group; t < tiles; t += HALVES == 2 ? 1 : 2) {
            const int s = t % p.stages, a = t % A_BUFFERS;
            if (!warp_wait_for(&sh.full_w[s], (t / p.stages) & 1, &sh)) break;
            const uint8_t *stage = ring + s * p.stage_bytes;
            uint32_t w[4][4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint4 u = *reinterpret_cast<const uint4 *>(stage + w_at + half * kW4TileBytes + c * 2048 + r * 16);
                w[c][0] = u.x;
                w[c][1] = u.y;
                w[c][2] = u.z;
                w[c][3] = u.w;
            }
            uint16_t sc[4];
            uint8_t z[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = (i / p.group_words) * kW4Rows + place;
                sc[i] = *reinterpret_cast<const uint16_t *>(stage + s_at + half * 1024 + at * 2);
                if (ZEROS) z[i] = stage[z_at + half * 512 + at];
            }
            __syncwarp();
            if (lane == 0) bar_arrive(&sh.empty_w[s]);
            if (!warp_wait_for(&sh.empty_a[a], ((t / A_BUFFERS) & 1) ^ 1, &sh)) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t at = tmem + (uint32_t((warp & 3) * 32) << 16) + A_COLUMN + (a * HALVES + half) * A_WIDTH;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t v[32];                      // column 16 w + 4 c + pair
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int i = 2 * h + j;
                    const float sn = scale_value(sc[i], p.scale_bf16) * down;
                    if (ZEROS) {
                        const uint32_t minus = N::both(-N::STEP * float(z[i])), scale = N::both(sn * (N::UNIT / N::STEP));
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const uint32_t u = w[c][i], uu = u >> 8;
                            v[16 * j + 4 * c + 0] = N::mul(N::fma(u & 0x000f000f, N::BIG, minus), scale);
                            v[16 * j + 4 * c + 1] = N::mul(N::fma(u & 0x00f000f0, N::SMALL, minus), scale);
                            v[16 * j + 4 * c + 2] = N::mul(N::fma(uu & 0x000f000f, N::BIG, minus), scale);
                            v[16 * j + 4 * c + 3] = N::mul(N::fma(uu & 0x00f000f0, N::SMALL, minus), scale);
                        }
                    } else {
                        const uint32_t big = N::both(sn * N::FACTOR), small = N::both(sn * (N::FACTOR / 16)), minus = N::both(sn * (-8 * N::UNIT));
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const uint32_t u = w[c][i], uu = u >> 8;
                            v[16 * j + 4 * c + 0] = N::fma(u & 0x000f000f, big, minus);
                            v[16 * j + 4 * c + 1] = N::fma(u & 0x00f000f0, small, minus);
                            v[16 * j + 4 * c + 2] = N::fma(uu & 0x000f000f, big, minus);
                            v[16 * j + 4 * c + 3] = N::fma(uu & 0x00f000f0, small, minus);
                        }
                    }
                }
                st_tmem32(at + 32 * h, v);
            }
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) bar_arrive(&sh.full_a[a]);
        }
    } else if (warp < DEQUANT_WARPS + LOAD_WARPS) {
        // ---- rows of x to the swizzled operand: 16 lanes a row, 8 values a lane ---------------------------------------
        const int j = lane & 15, first = (warp - DEQUANT_WARPS) * 2 + (lane >> 4);
        const int swizzled = (j >> 3) * (p.tokens * 128);            // which 64 of the 128
        const char *x = static_cast<const char *>(p.x);
        constexpr int PASSES = TOKENS / (2 * LOAD_WARPS);
        uint4 v[PASSES];
        auto fetch = [&](int t) {
            const int64_t k = int64_t(kb0 + t) * kW4Depth + 8 * j;
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                const int row = first + i * 2 * LOAD_WARPS;
                const int64_t at = row < p.tokens ? sh.row_at[row] : -1;
                v[i] = at >= 0 ? load_x<XT>(x + at, k, p.k, p.x_align) : make_uint4(0, 0, 0, 0);
            }
        };
        if (tiles > 0) fetch(0);
        for (int t = 0; t < tiles; ++t) {
            const int s = t % p.stages;
            if (!warp_wait_for(&sh.empty_x[s], ((t / p.stages) & 1) ^ 1, &sh)) break;
            uint8_t *stage = ring + s * p.stage_bytes + swizzled;
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                const int row = first + i * 2 * LOAD_WARPS;
                if (row < p.tokens) *reinterpret_cast<uint4 *>(stage + row * 128 + (((j & 7) ^ (row & 7)) << 4)) = v[i];
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) bar_arrive(&sh.full_x[s]);
            if (t + 1 < tiles) fetch(t + 1);
        }
    } else if (warp == MMA_WARP) {
        // ---- products ---------------------------------------------------------------------------------------------------
        if (lane == 0) {
            const uint32_t format = XT == XBF16 ? 1 : 0;
            const uint32_t idesc = (1u << 4) | (format << 7) | (format << 10) | (uint32_t(p.tokens >> 3) << 17) | (uint32_t(128 >> 4) << 24);
            bool alive = true;
            for (int t = 0; t < tiles && alive; ++t) {
                const int s = t % p.stages, a = t % A_BUFFERS;
                alive = wait_for(&sh.full_x[s], (t / p.stages) & 1, &sh) && wait_for(&sh.full_a[a], (t / A_BUFFERS) & 1, &sh);
                if (!alive) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t x_addr = smem_addr(ring + s * p.stage_bytes);
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {
                    const uint64_t b = operand(x_addr + (kk >> 2) * (p.tokens * 128) + (kk & 3) * 32);
#pragma unroll
                    for (int h = 0; h < HALVES; ++h)
                        mma(tmem + h * TOKENS, tmem + A_COLUMN + (a * HALVES + h) * A_WIDTH + kk * 8, b, idesc, t > 0 || kk > 0);
                }
                commit(&sh.empty_x[s]);
                commit(&sh.empty_a[a]);
            }
            commit(&sh.done);
        }
    } else if (lane == 0) {
        // ---- weights to shared memory -----------------------------------------------------------------------------------
        const uint32_t scale_bytes = uint32_t(per_tile) * 256, zero_bytes = ZEROS ? uint32_t(per_tile) * 128 : 0;
        int issued = 0;
        for (; issued < tiles; ++issued) {
            const int s = issued % p.stages;
            if (!wait_for(&sh.empty_w[s], ((issued / p.stages) & 1) ^ 1, &sh)) break;
            bar_expect(&sh.full_w[s], HALVES * (kW4TileBytes + scale_bytes + zero_bytes));
            uint8_t *stage = ring + s * p.stage_bytes;
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
                const int64_t nt = nt0 + h < p.row_tiles ? nt0 + h : p.row_tiles - 1;      // past the last tile: the last one again, its results not written
                const int64_t tile = nt * p.depth_tiles + kb0 + issued;
                bulk_copy(stage + w_at + h * kW4TileBytes, p.packed + tile * kW4TileBytes, kW4TileBytes, &sh.full_w[s]);
                bulk_copy(stage + s_at + h * 1024, p.scales + tile * per_tile * kW4Rows, scale_bytes, &sh.full_w[s]);
                if (ZEROS) bulk_copy(stage + z_at + h * 512, p.zeros + tile * per_tile * kW4Rows, zero_bytes, &sh.full_w[s]);
            }
        }
        // no copy may be in flight when the ring is used for the results or the CTA ends
        for (int t = issued > p.stages ? issued - p.stages : 0; t < issued; ++t)
            for (uint32_t i = 0; i < kWaitLimit && !bar_try(&sh.full_w[t % p.stages], (t / p.stages) & 1); ++i) {}
    }
    __syncwarp();

    // ---- results ------------------------------------------------------------------------------------------------------------
    const bool finished = warp_wait_for(&sh.done, 0, &sh);
    __syncthreads();                 // every role is through with the ring
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const int group = warp >> 2, r = (warp & 3) * 32 + lane;
    if (splits == 1) {
        constexpr int PITCH = ROWS * 2 + 16;          // bytes of one row of x's results in shared memory
        if (warp < DEQUANT_WARPS && finished) {
            const int half = HALVES == 2 ? group : 0;
            const int64_t row = row0 + half * kW4Rows + r;
            const float back = row < p.row_tiles * kW4Rows ? N::BACK * p.exponents[row] : 0.f;
            for (int c = HALVES == 2 ? 0 : 16 * group; c < p.tokens; c += HALVES == 2 ? 16 : 32) {
                uint32_t v[16];
                ld_tmem16(v, tmem + (uint32_t((warp & 3) * 32) << 16) + half * TOKENS + c);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float y = __uint_as_float(v[i]) * back;
                    if (p.x_scale) y *= t0 + c + i < p.m ? p.x_scale[t0 + c + i] : 0.f;
                    uint16_t *to = reinterpret_cast<uint16_t *>(ring + (c + i) * PITCH) + half * kW4Rows + r;
                    *to = p.out_type == STRASSEN_BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(y)) : __half_as_ushort(__float2half_rn(y));
                }
            }
        }
        __syncthreads();
        const int tokens = int(p.m - t0 < p.tokens ? p.m - t0 : p.tokens);
        const int rows = int(p.n - row0 < ROWS ? p.n - row0 : ROWS);
        uint16_t *out = static_cast<uint16_t *>(p.out) + t0 * p.ldo + row0;
        if (p.out_wide) {
            for (int e = threadIdx.x; e < tokens * (ROWS / 8); e += THREADS) {
                const int i = e / (ROWS / 8), c = e % (ROWS / 8) * 8;
                const uint16_t *from = reinterpret_cast<const uint16_t *>(ring + i * PITCH) + c;
                if (c + 8 <= rows) *reinterpret_cast<uint4 *>(out + i * p.ldo + c) = *reinterpret_cast<const uint4 *>(from);
                else
                    for (int b = 0; c + b < rows; ++b) out[i * p.ldo + c + b] = from[b];
            }
        } else {
            for (int e = threadIdx.x; e < tokens * ROWS; e += THREADS) {
                const int i = e / ROWS, c = e % ROWS;
                if (c < rows) out[i * p.ldo + c] = reinterpret_cast<const uint16_t *>(ring + i * PITCH)[c];
            }
        }
    } else {
        // partial sums side by side in the cluster: [row of x][row of weights], 32 bits
        float *sums = reinterpret_cast<float *>(ring);
        if (warp < DEQUANT_WARPS && finished) {
            const int half = HALVES == 2 ? group : 0;
            for (int c = HALVES == 2 ? 0 : 16 * group; c < p.tokens; c += HALVES == 2 ? 16 : 32) {
                uint32_t v[16];
                ld_tmem16(v, tmem + (uint32_t((warp & 3) * 32) << 16) + half * TOKENS + c);
#pragma unroll
                for (int i = 0; i < 16; ++i) sums[(c + i) * ROWS + half * kW4Rows + r] = __uint_as_float(v[i]);
            }
        }
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        const int tokens = int(p.m - t0 < p.tokens ? p.m - t0 : p.tokens);
        for (int e = threadIdx.x + int(blockIdx.y) * THREADS; e < tokens * ROWS; e += THREADS * splits) {
            const int i = e / ROWS, c = e % ROWS;
            float y = 0.f;
            for (int b = 0; b < splits; ++b) y += cluster.map_shared_rank(sums, b)[e];
            if (row0 + c < p.n) {
                y *= N::BACK * p.exponents[row0 + c];
                if (p.x_scale) y *= p.x_scale[t0 + i];
                static_cast<uint16_t *>(p.out)[(t0 + i) * p.ldo + row0 + c] =
                    p.out_type == STRASSEN_BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(y)) : __half_as_ushort(__float2half_rn(y));
            }
        }
        cluster.sync();              // no CTA leaves while another reads its sums
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

constexpr int kDynamicLimit = 222 * 1024;         // of 227 KB: the rest holds Shared

template <int XT, int HALVES, bool ZEROS> cudaError_t launch_one(Args p, int splits, cudaStream_t stream)
{
    p.x_bytes = p.tokens * 256;
    p.stage_bytes = (p.x_bytes + HALVES * (kW4TileBytes + 1024 + 512) + 1023) / 1024 * 1024;
    int stages = (kDynamicLimit - 1024) / p.stage_bytes;
    p.stages = stages > MAX_STAGES ? MAX_STAGES : stages;
    int bytes = p.stages * p.stage_bytes;
    const int rows = 128 * HALVES, results = splits == 1 ? p.tokens * (rows * 2 + 16) : p.tokens * rows * 4;
    if (results > bytes) bytes = results;
    bytes += 1024;
    cudaError_t e = cudaFuncSetAttribute(w4_tile_kernel<XT, HALVES, ZEROS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kDynamicLimit);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned((p.row_tiles + HALVES - 1) / HALVES), unsigned(splits), unsigned((p.m + p.tokens - 1) / p.tokens));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = size_t(bytes);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 1;
    attr[0].val.clusterDim.y = unsigned(splits);
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, w4_tile_kernel<XT, HALVES, ZEROS>, p);
}

template <int XT> cudaError_t launch_type(const Args &p, bool zeros, int sm_count, cudaStream_t stream)
{
    const int64_t token_tiles = (p.m + p.tokens - 1) / p.tokens;
    // two row tiles share the rows of x that a CTA brings in: taken where that leaves enough CTAs
    if ((p.row_tiles + 1) / 2 * token_tiles >= sm_count) return zeros ? launch_one<XT, 2, true>(p, 1, stream) : launch_one<XT, 2, false>(p, 1, stream);
    int splits = 1;
    while (splits < 8 && p.row_tiles * token_tiles * (splits + 1) <= sm_count && p.depth_tiles >= 2 * (splits + 1)) ++splits;
    return zeros ? launch_one<XT, 1, true>(p, splits, stream) : launch_one<XT, 1, false>(p, splits, stream);
}

int alignment(uintptr_t bits)
{
    int a = 16;
    while (bits % a) a /= 2;
    return a;
}

}  // namespace

cudaError_t launch_w4_tiles(const W4Args &a, int sm_count, cudaStream_t stream)
{
    const int size = a.type == STRASSEN_E4M3 ? 1 : 2;
    constexpr int64_t most = int64_t(65535) * TOKENS;            // rows of x in one launch: the grid's z
    for (int64_t m0 = 0; m0 < a.m; m0 += most) {
        Args p = {};
        p.packed = a.packed;
        p.zeros = a.packed + a.lay.zero_off;
        p.scales = reinterpret_cast<const uint16_t *>(a.packed + a.lay.scale_off);
        p.exponents = reinterpret_cast<const float *>(a.packed + a.lay.exponent_off);
        p.x = static_cast<const char *>(a.x) + m0 * a.ldx * size;
        p.x_scale = a.x_scale ? a.x_scale + m0 : nullptr;
        p.out = static_cast<char *>(a.out) + m0 * a.ldo * 2;
        p.n = a.lay.n;
        p.k = a.lay.k;
        p.m = a.m - m0 < most ? a.m - m0 : most;
        p.ldx_bytes = a.ldx * size;
        p.ldo = a.ldo;
        p.depth_tiles = a.lay.depth_tiles;
        p.row_tiles = a.lay.row_tiles;
        p.group_words = a.lay.group / 32;
        p.x_align = alignment(reinterpret_cast<uintptr_t>(p.x) | uintptr_t(p.m > 1 ? p.ldx_bytes : 0));
        p.scale_bf16 = a.lay.scale_type == STRASSEN_BF16;
        p.out_type = a.out_type;
        p.out_wide = reinterpret_cast<uintptr_t>(p.out) % 16 == 0 && (p.m == 1 || p.ldo % 8 == 0);
        const int64_t tiles = (p.m + TOKENS - 1) / TOKENS;
        p.tokens = int(((p.m + tiles - 1) / tiles + 15) / 16 * 16);
        cudaError_t e;
        if (a.type == STRASSEN_BF16) e = launch_type<XBF16>(p, a.lay.has_zeros, sm_count, stream);
        else if (a.type == STRASSEN_F16) e = launch_type<XF16>(p, a.lay.has_zeros, sm_count, stream);
        else e = launch_type<XE4M3>(p, a.lay.has_zeros, sm_count, stream);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

cudaError_t read_gave_up(int *flag)
{
    cudaError_t e = cudaMemcpyFromSymbol(flag, g_gave_up, sizeof(int));
    if (e != cudaSuccess || !*flag) return e;
    const int zero = 0;
    return cudaMemcpyToSymbol(g_gave_up, &zero, sizeof(int));
}

}  // namespace strassen
