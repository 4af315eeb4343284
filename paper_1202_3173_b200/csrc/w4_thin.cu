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
// The warps of a CTA hold the same rows of weights and take the 128-deep tiles of the inner dimension in turn, U at a time: the weights, scales
// and zero points of U tiles are under way before the rows of x are staged in shared memory (as 16-bit values, from any alignment) and any of them is used.
// The warps' sums meet in shared memory and are added in a fixed order.  Where the rows are too few to fill the GPU, the CTAs of a cluster split the inner
// dimension further and add their sums over distributed shared memory, again in a fixed order: no atomics, the same bits every time.
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

namespace {

constexpr int WARPS = 8;

enum { XBF16 = 0, XF16 = 1, XE4M3 = 2 };

template <int XT> struct Num;
// BIG, SMALL: factors for nibbles in bits 0..3 and 4..7; UNIT: what one step of q is afterwards; BACK: its inverse
template <> struct Num<XBF16> {
    static constexpr uint32_t BIG = 0x7f007f00, SMALL = 0x7d007d00;      // 2^127, 2^123
    static constexpr float UNIT = 1.f / 64, BACK = 64.f;
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
    static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
    {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};
template <> struct Num<XF16> {
    static constexpr uint32_t BIG = 0x78007800, SMALL = 0x68006800;      // 2^15, 2^11
    static constexpr float UNIT = 1.f / 512, BACK = 512.f;
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
    static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
    {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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
    int group_words;         // words of a row's 16 bytes in one group: 1, 2 or 4
    int tile_bytes, zero_off;
    int buffers;             // of a chunk of the rows of x
    bool scale_bf16, out_bf16;
    // experts: m tokens with `top` ids each
    const int *ids;
    const float *weights;
    int64_t row_tiles;       // of one matrix
    int top, experts;
    bool each;
};

enum { ONE = 0, EACH_ID = 1, SUM_OF_IDS = 2 };

// RT pieces of 16 rows, TT pieces of 8 tokens, U tiles of a warp at a time.
// With experts a CTA has a single row of x at a time: MODE EACH_ID that of one id, its row of results; MODE SUM_OF_IDS those of all ids of
// a token one after another, their sums multiplied by the ids' weights on the way.
template <int XT, int RT, int TT, int U, bool ZEROS, int MODE> __global__ void __launch_bounds__(WARPS * 32, 2) w4_thin_kernel(const Ptrs p)
{
    using N = Num<XT>;
    constexpr int ROWS = 16 * RT, TOKENS = 8 * TT, CELLS = ROWS * TOKENS;
    constexpr int CHUNK_TILES = WARPS * U, CHUNK = CHUNK_TILES * kW4Depth;
    constexpr int PITCH = CHUNK * 2 + 64;                    // bytes of a row of x: two rows' 64 bytes, which 8 lanes read at a time, in different banks
    extern __shared__ __align__(16) uint8_t staged[];        // chunks of rows of x, at the end the warps' sums
    after_work_before();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const int64_t row0 = int64_t(blockIdx.x) * ROWS, nt = row0 / kW4Rows;
    const int r_in = int(row0 % kW4Rows);
    const int64_t t0 = MODE == ONE ? int64_t(blockIdx.z) * TOKENS : int64_t(blockIdx.z);        // first row of x; with experts, of the result
    const int rows = MODE == ONE ? int(p.m - t0 < TOKENS ? p.m - t0 : TOKENS) : 1;
    const uintptr_t x_begin = reinterpret_cast<uintptr_t>(p.x);

    float acc[RT][TT][4] = {};
    int buffer = 0;
    const int choices = MODE == SUM_OF_IDS ? p.top : 1;
    for (int choice = 0; choice < choices; ++choice) {
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
        for (int64_t base = int64_t(blockIdx.y) * CHUNK_TILES; base < p.depth_tiles; base += int64_t(gridDim.y) * CHUNK_TILES) {
            uint4 w[U][RT][2];
            uint32_t scales[U][RT][4], zeros[U][RT][4];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t kb = base + u * WARPS + warp;
                if (kb < p.depth_tiles) {
                    const uint8_t *const packed = p.packed + (matrix_tile * p.depth_tiles + kb) * p.tile_bytes;
                    const uint4 *tile = reinterpret_cast<const uint4 *>(packed) + c * kW4Rows + r_in + g;
#pragma unroll
                    for (int r = 0; r < RT; ++r)
#pragma unroll
                        for (int h = 0; h < 2; ++h) w[u][r][h] = __ldg(tile + 16 * r + 8 * h);
#pragma unroll
                    for (int gg = 0; gg < 4; ++gg)
                        if (gg % p.group_words == 0) {
                            const int at = gg / p.group_words * kW4Rows + r_in + 2 * g;
#pragma unroll
                            for (int r = 0; r < RT; ++r) {
                                scales[u][r][gg] = *reinterpret_cast<const uint32_t *>(packed + kW4NibbleBytes + 2 * (at + 16 * r));
                                zeros[u][r][gg] = ZEROS ? *reinterpret_cast<const uint16_t *>(packed + p.zero_off + at + 16 * r) : 0x0808;
                            }
                        }
                }
            }
            // this chunk of the rows of x
            uint8_t *const xs = staged + buffer * (rows * PITCH);
            const int64_t k0 = base * kW4Depth;
            const int pieces = int(p.k - k0 < CHUNK ? (p.k - k0 + 127) / 128 * 16 : CHUNK / 8);          // of a row; whole tiles
            for (int row = 0; row < rows; ++row) {
                const char *const x = static_cast<const char *>(p.x) + (from + row) * p.ldx_bytes;
                for (int i = threadIdx.x; i < pieces; i += WARPS * 32)
                    *reinterpret_cast<uint4 *>(xs + row * PITCH + i * 16) = load_x<XT>(x, k0 + i * 8, p.k, x_begin, p.x_end);
            }
            __syncthreads();
            if (p.buffers > 1) buffer ^= 1;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (base + u * WARPS + warp >= p.depth_tiles) break;
                float part[RT][TT][4] = {};
                float scale[RT][2];
                uint32_t minus[RT][2];
#pragma unroll
                for (int gg = 0; gg < 4; ++gg) {
                    if (gg % p.group_words == 0) {
#pragma unroll
                        for (int r = 0; r < RT; ++r) {
                            const uint32_t s = scales[u][r][gg], z = zeros[u][r][gg];
                            scale[r][0] = scale_value(s & 0xffff, p.scale_bf16) * (MODE == ONE ? 1.f : factor[r][0]);
                            scale[r][1] = scale_value(s >> 16, p.scale_bf16) * (MODE == ONE ? 1.f : factor[r][1]);
                            minus[r][0] = N::both(-N::UNIT * float(z & 0xff));
                            minus[r][1] = N::both(-N::UNIT * float(z >> 8));
                        }
                    }
                    uint4 xv[TT];
#pragma unroll
                    for (int t = 0; t < TT; ++t) {
                        xv[t] = make_uint4(0, 0, 0, 0);
                        if (8 * t + g < rows) xv[t] = *reinterpret_cast<const uint4 *>(xs + (8 * t + g) * PITCH + ((u * WARPS + warp) * kW4Depth + 32 * gg + 8 * c) * 2);
                    }
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
#pragma unroll
                        for (int r = 0; r < RT; ++r) {
                            uint32_t a[4];
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const uint32_t word = gg == 0 ? w[u][r][h].x : gg == 1 ? w[u][r][h].y : gg == 2 ? w[u][r][h].z : w[u][r][h].w, v = half ? word >> 8 : word;
                                a[h] = N::fma(v & 0x000f000f, N::BIG, minus[r][h]);
                                a[2 + h] = N::fma(v & 0x00f000f0, N::SMALL, minus[r][h]);
                            }
#pragma unroll
                            for (int t = 0; t < TT; ++t) N::mma(part[r][t], a, half ? xv[t].z : xv[t].x, half ? xv[t].w : xv[t].y);
                        }
                    }
                    if ((gg + 1) % p.group_words == 0) {
#pragma unroll
                        for (int r = 0; r < RT; ++r)
#pragma unroll
                            for (int t = 0; t < TT; ++t)
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    acc[r][t][i] += scale[r][i >> 1] * part[r][t][i];
                                    part[r][t][i] = 0.f;
                                }
                    }
                }
            }
            if (p.buffers == 1) __syncthreads();             // before the only buffer is written again
        }
    }
    __syncthreads();
    float *const red = reinterpret_cast<float *>(staged);
    // cell (row, token) at token * ROWS + row: accumulator i is row g + 8 (i / 2), token 2 c + i % 2
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) red[warp * CELLS + (8 * t + 2 * c + (i & 1)) * ROWS + 16 * r + g + 8 * (i >> 1)] = acc[r][t][i];
    __syncthreads();
    cg::cluster_group cluster = cg::this_cluster();
    const int splits = int(gridDim.y);
    if (splits > 1) {
        for (int e = threadIdx.x; e < CELLS; e += WARPS * 32) {
            float s = red[e];
#pragma unroll
            for (int w = 1; w < WARPS; ++w) s += red[w * CELLS + e];
            red[e] = s;
        }
        cluster.sync();
    }
    // CTA y of the cluster writes every splits-th run of cells
    for (int e = blockIdx.y * (WARPS * 32) + threadIdx.x; e < CELLS; e += splits * (WARPS * 32)) {
        float s = 0.f;
        if (splits > 1) {
            for (int y = 0; y < splits; ++y) s += cluster.map_shared_rank(red, y)[e];
        } else {
#pragma unroll
            for (int w = 0; w < WARPS; ++w) s += red[w * CELLS + e];
        }
        const int64_t n = row0 + e % ROWS, t = t0 + e / ROWS;
        if (n < p.n && (MODE == ONE ? t < p.m : e < ROWS)) {
            s *= N::BACK;
            if (MODE == ONE) s *= p.x_scale ? p.x_scale[t] * p.exponents[n] : p.exponents[n];
            if (p.out_bf16) static_cast<__nv_bfloat16 *>(p.out)[t * p.ldo + n] = __float2bfloat16_rn(s);
            else static_cast<__half *>(p.out)[t * p.ldo + n] = __float2half_rn(s);
        }
    }
    if (splits > 1) cluster.sync();         // no CTA leaves while another reads its sums
}

template <int XT, int RT, int TT, int U, bool ZEROS, int MODE> cudaError_t launch_one(Ptrs p, int sm_count, cudaStream_t stream)
{
    constexpr int PITCH = WARPS * U * kW4Depth * 2 + 64, SUMS = WARPS * 16 * RT * 8 * TT * 4, MOST = 2 * 8 * TT * PITCH > SUMS ? 2 * 8 * TT * PITCH : SUMS;
    static std::atomic<uint64_t> opted_in{0};                // devices that this kernel has been given its shared memory on
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (MOST > 48 * 1024 && !(opted_in.load(std::memory_order_relaxed) >> dev & 1)) {
        e = cudaFuncSetAttribute(w4_thin_kernel<XT, RT, TT, U, ZEROS, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST);
        if (e != cudaSuccess) return e;
        opted_in.fetch_or(uint64_t(1) << dev, std::memory_order_relaxed);
    }
    const int64_t rows = (p.n + 16 * RT - 1) / (16 * RT), tokens = MODE == ONE ? (p.m + 8 * TT - 1) / (8 * TT) : MODE == EACH_ID ? p.m * p.top : p.m;
    const int64_t chunks = (p.depth_tiles + WARPS * U - 1) / (WARPS * U);
    int splits = 1;
    while (splits < 8 && splits * 2 <= chunks && rows * tokens * splits * 2 <= 2 * sm_count) splits *= 2;
    p.buffers = chunks > splits || (MODE == SUM_OF_IDS && p.top > 1) ? 2 : 1;
    const int staged_rows = MODE == ONE ? int(p.m < 8 * TT ? p.m : 8 * TT) : 1;
    int bytes = p.buffers * staged_rows * PITCH;
    if (bytes < SUMS) bytes = SUMS;
    return launch_after(w4_thin_kernel<XT, RT, TT, U, ZEROS, MODE>, dim3(unsigned(rows), unsigned(splits), unsigned(tokens)), dim3(WARPS * 32), size_t(bytes), stream, dim3(1, unsigned(splits)), p);
}

template <int XT, bool ZEROS> cudaError_t launch_shape(const Ptrs &p, int sm_count, cudaStream_t stream)
{
    if (p.ids) return p.weights ? launch_one<XT, 1, 1, 4, ZEROS, SUM_OF_IDS>(p, sm_count, stream) : launch_one<XT, 1, 1, 4, ZEROS, EACH_ID>(p, sm_count, stream);
    if (p.m <= 2) return launch_one<XT, 1, 1, 4, ZEROS, ONE>(p, sm_count, stream);
    if (p.m <= 8) return launch_one<XT, 2, 1, 2, ZEROS, ONE>(p, sm_count, stream);
    return launch_one<XT, 4, 2, 1, ZEROS, ONE>(p, sm_count, stream);
}

template <int XT> cudaError_t launch_type(const Ptrs &p, bool zeros, int sm_count, cudaStream_t stream)
{
    return zeros ? launch_shape<XT, true>(p, sm_count, stream) : launch_shape<XT, false>(p, sm_count, stream);
}

}  // namespace

cudaError_t launch_w4_thin(const W4Args &a, int sm_count, cudaStream_t stream)
{
    const int size = a.type == STRASSEN_E4M3 ? 1 : 2;
    constexpr int64_t most = int64_t(65535) * 8;                 // rows of x in one launch: the grid's z
    for (int64_t m0 = 0; m0 < a.m; m0 += most) {
        Ptrs p;
        p.packed = a.packed;
        p.exponents = reinterpret_cast<const float *>(a.packed + a.lay.exponent_off);
        p.tile_bytes = a.lay.tile_bytes;
        p.zero_off = a.lay.zero_off();
        p.x = static_cast<const char *>(a.x) + m0 * a.ldx * size;
        p.x_scale = a.x_scale ? a.x_scale + m0 : nullptr;
        p.out = static_cast<char *>(a.out) + m0 * a.ldo * 2;
        p.n = a.lay.n;
        p.k = a.lay.k;
        p.m = a.m - m0 < most ? a.m - m0 : most;
        p.ldx_bytes = a.ldx * size;
        p.ldo = a.ldo;
        p.depth_tiles = a.lay.depth_tiles;
        p.group_words = a.lay.group / 32;
        const int64_t x_rows = a.ids && a.each ? a.m * a.top : p.m;
        p.x_end = reinterpret_cast<uintptr_t>(p.x) + uintptr_t((x_rows - 1) * p.ldx_bytes + p.k * size);
        p.scale_bf16 = a.lay.scale_type == STRASSEN_BF16;
        p.out_bf16 = a.out_type == STRASSEN_BF16;
        p.ids = a.ids;
        p.weights = a.weights;
        p.row_tiles = a.lay.row_tiles;
        p.top = int(a.top);
        p.experts = int(a.lay.experts);
        p.each = a.each;
        cudaError_t e;
        if (a.type == STRASSEN_BF16) e = launch_type<XBF16>(p, a.lay.has_zeros, sm_count, stream);
        else if (a.type == STRASSEN_F16) e = launch_type<XF16>(p, a.lay.has_zeros, sm_count, stream);
        else e = launch_type<XE4M3>(p, a.lay.has_zeros, sm_count, stream);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace strassen
