// Products of a few rows with a matrix of 4-bit weights:  y_mn = xs_m sum_k x_mk S_{n,g(k)} (Q_nk - Z_{n,g(k)}).
//
// The matrix is read once and dominates the bytes: bound by HBM (by latency for small matrices).  A warp multiplies
// 16 rows of weights x 128 positions by 8 rows of x with m16n8k16 tensor instructions; the weights are the 16-row operand, so one token
// pays for eight, which costs nothing while the weights arrive slower than they are multiplied.
//
// A nibble becomes an exact 16-bit float without a conversion instruction.  Masked out of its word, a pair of nibbles IS a pair of
// subnormal numbers q 2^-133 (bf16) or q 2^-24 (f16); one packed multiply-add takes it to (q - z) 2^-6 or (q - z) 2^-9, exactly.
// Nibbles in bits 4..7 are 16 q in the same unit and take a sixteenth of the factor, so two pairs need no shift: 9 instructions for 8 weights.
//
// Products are summed over one group in the 32-bit accumulators of the tensor instructions and only then multiplied by the group's
// scale, in 32 bits: no weight is ever rounded.  (Scales are held as S 2^-e; the row's power of two joins at the end: w4_pack.cu.)
//
// The warps of a CTA form WR groups of rows of weights; the WK warps of a group take the 128-deep tiles of the inner dimension in turn, U at a time, with the
// weights, scales and zero points of the next U on their way while these are multiplied.  The rows of x are staged in shared memory as 16-bit values, from
// any alignment.  The sums of a group's warps meet in shared memory and are added in a fixed order.  WK is as small as leaves work for every warp of
// the GPU: each warp's fixed costs are then spread over the most tiles.  Where the rows are too few even for WK = 8, the CTAs of a cluster split the inner
// dimension (or the ids of a token) further and add their sums over distributed shared memory, again in a fixed order: no atomics, the same bits every time.
//
// Bound by latency and by what a tile takes in instructions (some 160 a warp for 16 x 128 weights), not by HBM: 1 row, 4099 x 12345 f16 in 11.7 us, 7 rows 15.8 us
// (27.5 MB, 1.7 TB/s); 16384 x 4096, 1 row 12.6 us (2.8 TB/s); 4096 x 4096, 1 row 6.7 us.
#pragma once

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <atomic>

#include "llm.h"
#include "pieces.cuh"
#include "strassen_b200.h"

namespace cg = cooperative_groups;

namespace strassen {
namespace thin {

constexpr int WARPS = 8;

enum { XBF16 = 0, XF16 = 1, XE4M3 = 2 };

template <int XT> struct Num;
// BIG, SMALL: factors for nibbles in bits 0..3 and 4..7; BACK: the inverse of what one step of q is afterwards
template <> struct Num<XBF16> {
    static constexpr uint32_t BIG = 0x7f007f00, SMALL = 0x7d007d00;      // 2^127, 2^123
    static constexpr float BACK = 64.f;
    // -z 2^-6 twice, as (128 + z) (-2^-6) + 2: 128 + z is 0x4300 + z
    static __device__ __forceinline__ uint32_t minus(uint32_t z) { return fma(0x43004300u | z | (z << 16), 0xbc80bc80u, 0x40004000u); }
    static __device__ __forceinline__ uint32_t fma(uint32_t a, uint32_t b, uint32_t c)
    {
        uint32_t d;
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
        return d;
    }
    // first: d starts from zero
    static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, bool first)
    {
        const float c0 = first ? 0.f : d[0], c1 = first ? 0.f : d[1], c2 = first ? 0.f : d[2], c3 = first ? 0.f : d[3];
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
    }
};
template <> struct Num<XF16> {
    static constexpr uint32_t BIG = 0x78007800, SMALL = 0x68006800;      // 2^15, 2^11
    static constexpr float BACK = 512.f;
    // -z 2^-9 twice, as (1024 + z) (-2^-9) + 2: 1024 + z is 0x6400 + z
    static __device__ __forceinline__ uint32_t minus(uint32_t z) { return fma(0x64006400u | z | (z << 16), 0x98009800u, 0x40004000u); }
    static __device__ __forceinline__ uint32_t fma(uint32_t a, uint32_t b, uint32_t c)
    {
        uint32_t d;
        asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
        return d;
    }
    // first: d starts from zero
    static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, bool first)
    {
        const float c0 = first ? 0.f : d[0], c1 = first ? 0.f : d[1], c2 = first ? 0.f : d[2], c3 = first ? 0.f : d[3];
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
    }
};
template <> struct Num<XE4M3> : Num<XF16> {};       // every e4m3 value is an f16 value

// Eight values of a row of x from k on as 16 bits each; zeros past the inner size.
template <int XT> __device__ __forceinline__ uint4 load_x(const char *row, int64_t k, int64_t size, uintptr_t lo, uintptr_t hi)
{
    if constexpr (XT == XE4M3) {
        const uint2 u = load_bytes8(reinterpret_cast<const uint8_t *>(row), k, size, lo, hi);
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t((i < 2 ? u.x : u.y) >> (16 * (i & 1))), __NV_E4M3);
            v[i] = uint32_t(h.x) | (uint32_t(h.y) << 16);
        }
        return make_uint4(v[0], v[1], v[2], v[3]);
    } else {
        Words<__half> w;
        load(w, reinterpret_cast<const __half *>(row), k, size, lo, hi);
        return make_uint4(w.w[0], w.w[1], w.w[2], w.w[3]);
    }
}

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ float scale_value(uint32_t bits, bool bf16)
{
    return bf16 ? __uint_as_float(bits << 16) : __half2float(__ushort_as_half(uint16_t(bits)));
}

struct Ptrs {
    const uint8_t *packed;
    const float *exponents;
    const void *x;
    const float *x_scale;
    void *out;
    int64_t n, k, m, ldx_bytes, ldo, depth_tiles;
    uintptr_t x_end;         // of the memory of x
    int tile_bytes, zero_off;
    int x_align;             // of the rows of x, in bytes: 2 .. 16
    int wk_shift;            // WK = 1 << wk_shift
    int chunk;               // tiles of the inner dimension whose rows of x are staged at a time
    bool scale_bf16, out_bf16;
    // experts: m tokens with `top` ids each
    const int *ids;
    const float *weights;
    int64_t row_tiles;       // of one matrix
    int top, experts;
    bool each;
};

enum { ONE = 0, EACH_ID = 1, SUM_OF_IDS = 2 };

// The weights of U tiles of a warp, as they come from memory.
template <int RT, int U> struct Batch {
    uint4 w[U][RT][2];
    uint32_t scales[U][RT][4], zeros[U][RT][4];          // of each group
};

// RT pieces of 16 rows, TT pieces of 8 tokens, U tiles of a warp at a time.
// With experts a CTA has a single row of x at a time: MODE EACH_ID that of one id, its row of results; MODE SUM_OF_IDS those of all ids of
// a token one after another, their sums multiplied by the ids' weights on the way.
// A group is 1 << GS words of a row's 16 bytes.
template <int XT, int GS, int RT, int TT, int U, bool ZEROS, int MODE> __global__ void __launch_bounds__(WARPS * 32, RT == 1 ? 4 : 2) w4_thin_kernel(const Ptrs p)
{
    using N = Num<XT>;
    constexpr int ROWS = 16 * RT, TOKENS = 8 * TT, CELLS = ROWS * TOKENS;
    extern __shared__ __align__(16) uint8_t staged[];        // rows of x, at the end the warps' sums
    after_work_before();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const int wk_count = 1 << p.wk_shift, wk = warp & (wk_count - 1), wr = warp >> p.wk_shift, wr_count = WARPS >> p.wk_shift;
    const int64_t row0 = (int64_t(blockIdx.x) * wr_count + wr) * ROWS;
    const int64_t nt = row0 / kW4Rows < p.row_tiles ? row0 / kW4Rows : p.row_tiles - 1;      // past the last rows: those again, not written
    const int r_in = int(row0 % kW4Rows);
    const int64_t t0 = MODE == ONE ? int64_t(blockIdx.z) * TOKENS : int64_t(blockIdx.z);        // first row of x; with experts, of the result
    const int rows = MODE == ONE ? int(p.m - t0 < TOKENS ? p.m - t0 : TOKENS) : 1;
    const uintptr_t x_begin = reinterpret_cast<uintptr_t>(p.x);
    constexpr int in_group = (1 << GS) - 1;
    const int pitch = p.chunk * (kW4Depth * 2) + 64;        // + 64: two rows' 64 bytes, which 8 lanes read at a time, in different banks
    const int splits = int(gridDim.y);

    const int chunk = W4Layout::chunk_place(r_in + g, c);
    // where this lane's rows of x are; past the last row, that one again: a column of sums that is not written
    int mine[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) mine[t] = (8 * t + g < rows ? 8 * t + g : rows - 1) * pitch;

    float acc[RT][TT][4] = {};
    for (int choice = MODE == SUM_OF_IDS ? blockIdx.y : 0; choice < (MODE == SUM_OF_IDS ? p.top : 1); choice += MODE == SUM_OF_IDS ? splits : 1) {
        int64_t matrix_tile = nt, from = t0;
        float factor[RT][2];
        if (MODE != ONE) {
            const int64_t at = MODE == SUM_OF_IDS ? t0 * p.top + choice : t0;
            from = p.each ? at : at / p.top;
            const int id = p.ids[at];
            if (id < 0 || id >= p.experts) continue;         // no expert: adds nothing
            matrix_tile += id * p.row_tiles;
            const float f = (p.x_scale ? p.x_scale[from] : 1.f) * (MODE == SUM_OF_IDS ? p.weights[at] : 1.f);
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h) factor[r][h] = f * p.exponents[matrix_tile * kW4Rows + r_in + 16 * r + 8 * h + g];
        }
        const int first = MODE == SUM_OF_IDS ? 0 : int(p.depth_tiles * blockIdx.y / splits), end = MODE == SUM_OF_IDS ? int(p.depth_tiles) : int(p.depth_tiles * (blockIdx.y + 1) / splits);
        const uint8_t *const matrix = p.packed + matrix_tile * p.depth_tiles * p.tile_bytes;
        // tiles kb, kb + WK, .. kb + (U - 1) WK
        const auto fetch = [&](Batch<RT, U> &b, int kb, int stop) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (kb + u * wk_count < stop) {
                    const uint8_t *const packed = matrix + int64_t(kb + u * wk_count) * p.tile_bytes;
                    const uint8_t *const tile = packed + chunk;
#pragma unroll
                    for (int r = 0; r < RT; ++r)
#pragma unroll
                        for (int h = 0; h < 2; ++h) b.w[u][r][h] = __ldg(reinterpret_cast<const uint4 *>(tile + 1024 * r + 512 * h));
#pragma unroll
                    for (int gg = 0; gg < 4; ++gg)
                        if ((gg & in_group) == 0) {
                            const int at = (gg >> GS) * kW4Rows + r_in + 2 * g;
#pragma unroll
                            for (int r = 0; r < RT; ++r) {
                                b.scales[u][r][gg] = *reinterpret_cast<const uint32_t *>(packed + kW4NibbleBytes + 2 * (at + 16 * r));
                                b.zeros[u][r][gg] = ZEROS ? *reinterpret_cast<const uint16_t *>(packed + p.zero_off + at + 16 * r) : 0x0808;
                            }
                        }
                }
        };
        const auto multiply = [&](const Batch<RT, U> &b, int kb, int stop, int chunk0) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (kb + u * wk_count >= stop) break;
                const uint8_t *const xs = staged + (kb + u * wk_count - chunk0) * (kW4Depth * 2) + 16 * c;
                float part[RT][TT][4];
                float scale[RT][2];
                uint32_t minus[RT][2];
#pragma unroll
                for (int gg = 0; gg < 4; ++gg) {
                    if ((gg & in_group) == 0) {
#pragma unroll
                        for (int r = 0; r < RT; ++r) {
                            const uint32_t s = b.scales[u][r][gg], z = b.zeros[u][r][gg];
                            scale[r][0] = scale_value(s & 0xffff, p.scale_bf16) * (MODE == ONE ? 1.f : factor[r][0]);
                            scale[r][1] = scale_value(s >> 16, p.scale_bf16) * (MODE == ONE ? 1.f : factor[r][1]);
                            minus[r][0] = N::minus(z & 0x00ff);
                            minus[r][1] = N::minus(z >> 8);
                        }
                    }
                    uint4 xv[TT];
#pragma unroll
                    for (int t = 0; t < TT; ++t) {
                        xv[t] = *reinterpret_cast<const uint4 *>(xs + mine[t] + 64 * gg);
                    }
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
#pragma unroll
                        for (int r = 0; r < RT; ++r) {
                            uint32_t a[4];
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const uint32_t word = gg == 0 ? b.w[u][r][h].x : gg == 1 ? b.w[u][r][h].y : gg == 2 ? b.w[u][r][h].z : b.w[u][r][h].w, v = half ? word >> 8 : word;
                                a[h] = N::fma(v & 0x000f000f, N::BIG, minus[r][h]);
                                a[2 + h] = N::fma(v & 0x00f000f0, N::SMALL, minus[r][h]);
                            }
#pragma unroll
                            for (int t = 0; t < TT; ++t) N::mma(part[r][t], a, half ? xv[t].z : xv[t].x, half ? xv[t].w : xv[t].y, (gg & in_group) == 0 && half == 0);
                        }
                    }
                    if ((gg & in_group) == in_group) {
#pragma unroll
                        for (int r = 0; r < RT; ++r)
#pragma unroll
                            for (int t = 0; t < TT; ++t)
#pragma unroll
                                for (int i = 0; i < 4; ++i) acc[r][t][i] += scale[r][i >> 1] * part[r][t][i];
                    }
                }
            }
        };
        for (int chunk0 = first; chunk0 < end; chunk0 += p.chunk) {
            const int stop = end - chunk0 < p.chunk ? end : chunk0 + p.chunk, step = U * wk_count;
            Batch<RT, U> one, two;
            int kb = chunk0 + wk;
            fetch(one, kb, stop);
            if (chunk0 > first || choice >= splits) __syncthreads();         // the rows that were staged before have been read
            // the rows of x of these tiles
            const int64_t k0 = int64_t(chunk0) * kW4Depth;
            const int pieces = (stop - chunk0) * (kW4Depth / 8), all = rows * pieces;
            if (XT != XE4M3 && p.x_align >= 4) {
                // copies past the registers, as wide as the rows' alignment allows; zeros past the inner size
                for (int i = threadIdx.x; i < all; i += WARPS * 32) {
                    const int row = i / pieces, at = i - row * pieces;
                    const uint32_t to = smem_addr(staged + row * pitch + at * 16);
                    const int64_t k = k0 + at * 8;
                    const char *x = static_cast<const char *>(p.x) + (from + row) * p.ldx_bytes + 2 * k;
                    const int valid = k >= p.k ? 0 : p.k - k >= 8 ? 16 : int(p.k - k) * 2;
                    if (valid == 0) x = static_cast<const char *>(p.x);
                    if (p.x_align >= 16) {
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(x), "r"(valid) : "memory");
                    } else if (p.x_align == 8) {
#pragma unroll
                        for (int b = 0; b < 16; b += 8) {
                            const int v = valid - b < 0 ? 0 : valid - b > 8 ? 8 : valid - b;
                            asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(to + b), "l"(v > 0 ? x + b : x), "r"(v) : "memory");
                        }
                    } else {
#pragma unroll
                        for (int b = 0; b < 16; b += 4) {
                            const int v = valid - b < 0 ? 0 : valid - b > 4 ? 4 : valid - b;
                            asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + b), "l"(v > 0 ? x + b : x), "r"(v) : "memory");
                        }
                    }
                }
                asm volatile("cp.async.wait_all;" ::: "memory");
            } else {
#pragma unroll 4
                for (int i = threadIdx.x; i < all; i += WARPS * 32) {
                    const int row = i / pieces, at = i - row * pieces;
                    *reinterpret_cast<uint4 *>(staged + row * pitch + at * 16) = load_x<XT>(static_cast<const char *>(p.x) + (from + row) * p.ldx_bytes, k0 + at * 8, p.k, x_begin, p.x_end);
                }
            }
            __syncthreads();
            for (; kb < stop; kb += 2 * step) {
                fetch(two, kb + step, stop);
                multiply(one, kb, stop, chunk0);
                fetch(one, kb + 2 * step, stop);
                multiply(two, kb + step, stop, chunk0);
            }
        }
    }
    __syncthreads();
    // cell (row, token) at token * ROWS + row: accumulator i is row g + 8 (i / 2), token 2 c + i % 2
    float *const red = reinterpret_cast<float *>(staged);
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) red[warp * CELLS + (8 * t + 2 * c + (i & 1)) * ROWS + 16 * r + g + 8 * (i >> 1)] = acc[r][t][i];
    __syncthreads();
    cg::cluster_group cluster = cg::this_cluster();
    const int cells = wr_count * CELLS;                      // of the CTA; those of a group's WK warps lie one set after another
    if (splits > 1) {
        for (int e = threadIdx.x; e < cells; e += WARPS * 32) {
            const int at = (e / CELLS << p.wk_shift) * CELLS + e % CELLS;
            float s = red[at];
            for (int w = 1; w < wk_count; ++w) s += red[at + w * CELLS];
            red[at] = s;
        }
        cluster.sync();
    }
    // CTA y of the cluster writes every splits-th run of cells
    for (int e = blockIdx.y * (WARPS * 32) + threadIdx.x; e < cells; e += splits * (WARPS * 32)) {
        const int group = e / CELLS, cell = e - group * CELLS, at = (group << p.wk_shift) * CELLS + cell;
        const int64_t n = (int64_t(blockIdx.x) * wr_count + group) * ROWS + cell % ROWS, t = t0 + cell / ROWS;
        if (n >= p.n || (MODE == ONE ? t >= p.m : cell >= ROWS)) continue;
        float s = 0.f;
        if (splits > 1) {
            for (int y = 0; y < splits; ++y) s += cluster.map_shared_rank(red, y)[at];
        } else {
            for (int w = 0; w < wk_count; ++w) s += red[at + w * CELLS];
        }
        s *= N::BACK;
        if (MODE == ONE) s *= p.x_scale ? p.x_scale[t] * p.exponents[n] : p.exponents[n];
        if (p.out_bf16) static_cast<__nv_bfloat16 *>(p.out)[t * p.ldo + n] = __float2bfloat16_rn(s);
        else static_cast<__half *>(p.out)[t * p.ldo + n] = __float2half_rn(s);
    }
    if (splits > 1) cluster.sync();         // no CTA leaves while another reads its sums
}

template <int XT, int GS, int RT, int TT, int U, bool ZEROS, int MODE> cudaError_t launch_one(Ptrs p, int sm_count, cudaStream_t stream)
{
    constexpr int SUMS = WARPS * 16 * RT * 8 * TT * 4, MOST = 208 / (RT == 1 ? 4 : 2) * 1024;        // of shared memory, for the CTAs that an SM's registers hold
    static std::atomic<uint64_t> opted_in{0};                // devices that this kernel has been given its shared memory on
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (!(opted_in.load(std::memory_order_relaxed) >> dev & 1)) {
        e = cudaFuncSetAttribute(w4_thin_kernel<XT, GS, RT, TT, U, ZEROS, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST);
        if (e != cudaSuccess) return e;
        opted_in.fetch_or(uint64_t(1) << dev, std::memory_order_relaxed);
    }
    const int64_t rows = (p.n + 16 * RT - 1) / (16 * RT), tokens = MODE == ONE ? (p.m + 8 * TT - 1) / (8 * TT) : MODE == EACH_ID ? p.m * p.top : p.m;
    const int64_t room = int64_t(RT == 1 ? 4 : 2) * WARPS * sm_count;      // warps that the GPU holds
    const int64_t tiles = rows * tokens;                     // that need a warp at least
    // the ids of a token go to different CTAs of a cluster, the inner dimension to the warps of a CTA and then to CTAs
    int splits = 1;
    if (MODE == SUM_OF_IDS)
        while (splits < 8 && splits * 2 <= p.top && tiles * splits < room) splits *= 2;
    p.wk_shift = 0;
    while (p.wk_shift < 3 && tiles * splits * (2 << p.wk_shift) <= room && (int64_t(2) << p.wk_shift) <= p.depth_tiles) ++p.wk_shift;
    if (MODE != SUM_OF_IDS)
        while (splits < 8 && tiles * WARPS * splits * 2 <= room && p.depth_tiles >= int64_t(splits) * 2 * WARPS) splits *= 2;
    const int staged_rows = MODE == ONE ? int(p.m < 8 * TT ? p.m : 8 * TT) : 1;
    const int64_t depth = MODE == SUM_OF_IDS ? p.depth_tiles : (p.depth_tiles + splits - 1) / splits, fit = (MOST / staged_rows - 64) / (kW4Depth * 2);
    // as few and as even chunks as fit, each a multiple of WK: a warp's tiles, and with them the order of its sums, then do not depend on how many rows
    // are staged, and a row's result has the same bits alone and among others
    const int64_t whole = fit >> p.wk_shift << p.wk_shift, chunks = (depth + whole - 1) / whole, even = (depth + chunks - 1) / chunks, wk = int64_t(1) << p.wk_shift;
    p.chunk = int(chunks == 1 ? depth : (even + wk - 1) / wk * wk);
    int bytes = staged_rows * (p.chunk * kW4Depth * 2 + 64);
    if (bytes < SUMS) bytes = SUMS;
    const int64_t groups = WARPS >> p.wk_shift;
    return launch_after(w4_thin_kernel<XT, GS, RT, TT, U, ZEROS, MODE>, dim3(unsigned((rows + groups - 1) / groups), unsigned(splits), unsigned(tokens)), dim3(WARPS * 32), size_t(bytes), stream, dim3(1, unsigned(splits)), p);
}

template <int XT, int GS, bool ZEROS> cudaError_t launch_shape(const Ptrs &p, int sm_count, cudaStream_t stream)
{
    if (p.ids) return p.weights ? launch_one<XT, GS, 1, 1, 1, ZEROS, SUM_OF_IDS>(p, sm_count, stream) : launch_one<XT, GS, 1, 1, 1, ZEROS, EACH_ID>(p, sm_count, stream);
    // Two tiles of 16 rows of weights to a warp share the rows of x that it reads from shared memory: 1 row, 4096 x 16384, groups of 32: 13.2 us, 15.5 with
    // one; 8 rows: 20.9 and 28.7 (16384 x 4096, groups of 128: 12.9 and 13.1; 16.4 and 21.6).  Products of ids have a row each, and more warps with one.
    if (p.m <= 8) return launch_one<XT, GS, 2, 1, 1, ZEROS, ONE>(p, sm_count, stream);
    return launch_one<XT, GS, 2, 2, 1, ZEROS, ONE>(p, sm_count, stream);
}

template <int XT, int GS> cudaError_t launch_group(const Ptrs &p, bool zeros, int sm_count, cudaStream_t stream)
{
    return zeros ? launch_shape<XT, GS, true>(p, sm_count, stream) : launch_shape<XT, GS, false>(p, sm_count, stream);
}

// One for each type of x, in a source file of its own (w4_thin_bf16.cu and so on).
cudaError_t launch_bf16(const Ptrs &p, int group, bool zeros, int sm_count, cudaStream_t stream);
cudaError_t launch_f16(const Ptrs &p, int group, bool zeros, int sm_count, cudaStream_t stream);
cudaError_t launch_e4m3(const Ptrs &p, int group, bool zeros, int sm_count, cudaStream_t stream);

template <int XT> cudaError_t launch_type(const Ptrs &p, int group, bool zeros, int sm_count, cudaStream_t stream)
{
    if (group == 32) return launch_group<XT, 0>(p, zeros, sm_count, stream);
    return group == 64 ? launch_group<XT, 1>(p, zeros, sm_count, stream) : launch_group<XT, 2>(p, zeros, sm_count, stream);
}

}  // namespace thin
}  // namespace strassen
