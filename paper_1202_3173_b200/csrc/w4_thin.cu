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
// The warps of a CTA hold the same rows of weights and take the 128-deep tiles of the inner dimension in turn; their sums meet in
// shared memory and are added in a fixed order.  Where the rows are too few to fill the GPU, the CTAs of a cluster split the inner
// dimension further and add their sums over distributed shared memory, again in a fixed order: no atomics, the same bits every time.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "llm.h"
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
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
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
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};
template <> struct Num<XE4M3> : Num<XF16> {};       // every e4m3 value is an f16 value

// Eight consecutive values of a row of x from k on, as four packed pairs; zeros past the inner size.
template <int XT> __device__ __forceinline__ void load_x(uint32_t (&v)[4], const void *row, int64_t k, int64_t size, int align)
{
    if constexpr (XT == XE4M3) {
        const uint8_t *p = static_cast<const uint8_t *>(row) + k;
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
        const uint16_t *p = static_cast<const uint16_t *>(row) + k;
        if (align >= 16 && k + 8 <= size) {
            const uint4 u = *reinterpret_cast<const uint4 *>(p);
            v[0] = u.x;
            v[1] = u.y;
            v[2] = u.z;
            v[3] = u.w;
        } else if (align >= 4 && k + 8 <= size) {
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
    int group_words;         // words of a row's 16 bytes in one group: 1, 2 or 4
    int tile_bytes, zero_off;
    int x_align;
    bool scale_bf16, out_bf16;
    // experts: m tokens with `top` ids each
    const int *ids;
    const float *weights;
    int64_t row_tiles;       // of one matrix
    int top, experts;
    bool each;
};

enum { ONE = 0, EACH_ID = 1, SUM_OF_IDS = 2 };

// RT pieces of 16 rows, TT pieces of 8 tokens.
// With experts a CTA has a single row of x at a time: MODE EACH_ID that of one id, its row of results; MODE SUM_OF_IDS those of all ids of
// a token one after another, their sums multiplied by the ids' weights on the way.
template <int XT, int RT, int TT, bool ZEROS, int MODE> __global__ void __launch_bounds__(WARPS * 32) w4_thin_kernel(const Ptrs p)
{
    using N = Num<XT>;
    constexpr int ROWS = 16 * RT, TOKENS = 8 * TT, CELLS = ROWS * TOKENS;
    __shared__ float red[WARPS][CELLS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const int64_t row0 = int64_t(blockIdx.x) * ROWS, nt = row0 / kW4Rows;
    const int r_in = int(row0 % kW4Rows);
    const int64_t t0 = MODE == ONE ? int64_t(blockIdx.z) * TOKENS : int64_t(blockIdx.z);        // first row of x; with experts, of the result

    float acc[RT][TT][4] = {};
    const void *xrow[TT];
    const int choices = MODE == SUM_OF_IDS ? p.top : 1;
    for (int choice = 0; choice < choices; ++choice) {
    int64_t matrix_tile = nt;
    float factor[RT][2];
    if (MODE == ONE) {
#pragma unroll
        for (int t = 0; t < TT; ++t) xrow[t] = t0 + 8 * t + g < p.m ? static_cast<const char *>(p.x) + (t0 + 8 * t + g) * p.ldx_bytes : nullptr;
    } else {
        const int64_t at = MODE == SUM_OF_IDS ? t0 * p.top + choice : t0, from = p.each ? at : at / p.top;
        const int id = p.ids[at];
        if (id < 0 || id >= p.experts) continue;         // no expert: adds nothing
        matrix_tile += id * p.row_tiles;
        xrow[0] = g == 0 ? static_cast<const char *>(p.x) + from * p.ldx_bytes : nullptr;
        const float f = (p.x_scale ? p.x_scale[from] : 1.f) * (MODE == SUM_OF_IDS ? p.weights[at] : 1.f);
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h) factor[r][h] = f * p.exponents[matrix_tile * kW4Rows + r_in + 16 * r + 8 * h + g];
    }

    for (int64_t kb = blockIdx.y * WARPS + warp; kb < p.depth_tiles; kb += int64_t(gridDim.y) * WARPS) {
        const uint8_t *const packed = p.packed + (matrix_tile * p.depth_tiles + kb) * p.tile_bytes;
        const uint4 *tile = reinterpret_cast<const uint4 *>(packed) + c * kW4Rows + r_in + g;
        uint32_t w[RT][2][4];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 u = __ldg(tile + 16 * r + 8 * h);
                w[r][h][0] = u.x;
                w[r][h][1] = u.y;
                w[r][h][2] = u.z;
                w[r][h][3] = u.w;
            }
        float part[RT][TT][4] = {};
        float scale[RT][2];
        uint32_t minus[RT][2];
#pragma unroll
        for (int gg = 0; gg < 4; ++gg) {
            if (gg % p.group_words == 0) {
                const int at = gg / p.group_words * kW4Rows + r_in + 2 * g;
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const uint32_t s = *reinterpret_cast<const uint32_t *>(packed + kW4NibbleBytes + 2 * (at + 16 * r));
                    scale[r][0] = scale_value(s & 0xffff, p.scale_bf16) * (MODE == ONE ? 1.f : factor[r][0]);
                    scale[r][1] = scale_value(s >> 16, p.scale_bf16) * (MODE == ONE ? 1.f : factor[r][1]);
                    uint32_t z = 0x0808;
                    if (ZEROS) z = *reinterpret_cast<const uint16_t *>(packed + p.zero_off + at + 16 * r);
                    minus[r][0] = N::both(-N::UNIT * float(z & 0xff));
                    minus[r][1] = N::both(-N::UNIT * float(z >> 8));
                }
            }
            uint32_t xv[TT][4];
#pragma unroll
            for (int t = 0; t < TT; ++t) {
#pragma unroll
                for (int i = 0; i < 4; ++i) xv[t][i] = 0;
                if (xrow[t]) load_x<XT>(xv[t], xrow[t], kb * kW4Depth + 32 * gg + 8 * c, p.k, p.x_align);
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    uint32_t a[4];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t u = half ? w[r][h][gg] >> 8 : w[r][h][gg];
                        a[h] = N::fma(u & 0x000f000f, N::BIG, minus[r][h]);
                        a[2 + h] = N::fma(u & 0x00f000f0, N::SMALL, minus[r][h]);
                    }
#pragma unroll
                    for (int t = 0; t < TT; ++t) N::mma(part[r][t], a, xv[t][2 * half], xv[t][2 * half + 1]);
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
    }
    // cell (row, token) at token * ROWS + row: accumulator i is row g + 8 (i / 2), token 2 c + i % 2
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) red[warp][(8 * t + 2 * c + (i & 1)) * ROWS + 16 * r + g + 8 * (i >> 1)] = acc[r][t][i];
    __syncthreads();
    cg::cluster_group cluster = cg::this_cluster();
    const int splits = int(gridDim.y);
    if (splits > 1) {
        for (int e = threadIdx.x; e < CELLS; e += WARPS * 32) {
            float s = red[0][e];
#pragma unroll
            for (int w = 1; w < WARPS; ++w) s += red[w][e];
            red[0][e] = s;
        }
        cluster.sync();
    }
    // CTA y of the cluster writes every splits-th run of cells
    for (int e = blockIdx.y * (WARPS * 32) + threadIdx.x; e < CELLS; e += splits * (WARPS * 32)) {
        float s = 0.f;
        if (splits > 1) {
            for (int y = 0; y < splits; ++y) s += cluster.map_shared_rank(&red[0][0], y)[e];
        } else {
#pragma unroll
            for (int w = 0; w < WARPS; ++w) s += red[w][e];
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

template <int XT, int RT, int TT, bool ZEROS, int MODE> cudaError_t launch_one(const Ptrs &p, int sm_count, cudaStream_t stream)
{
    const int64_t rows = (p.n + 16 * RT - 1) / (16 * RT), tokens = MODE == ONE ? (p.m + 8 * TT - 1) / (8 * TT) : MODE == EACH_ID ? p.m * p.top : p.m;
    int splits = 1;
    while (splits < 8 && rows * tokens * splits * 2 <= 2 * sm_count && p.depth_tiles >= int64_t(splits) * 2 * WARPS) splits *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(rows), unsigned(splits), unsigned(tokens));
    cfg.blockDim = dim3(WARPS * 32);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 1;
    attr[0].val.clusterDim.y = unsigned(splits);
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, w4_thin_kernel<XT, RT, TT, ZEROS, MODE>, p);
}

template <int XT, bool ZEROS> cudaError_t launch_shape(const Ptrs &p, int sm_count, cudaStream_t stream)
{
    if (p.ids) return p.weights ? launch_one<XT, 1, 1, ZEROS, SUM_OF_IDS>(p, sm_count, stream) : launch_one<XT, 1, 1, ZEROS, EACH_ID>(p, sm_count, stream);
    if (p.m <= 2) return launch_one<XT, 1, 1, ZEROS, ONE>(p, sm_count, stream);
    if (p.m <= 8) return launch_one<XT, 2, 1, ZEROS, ONE>(p, sm_count, stream);
    return launch_one<XT, 4, 2, ZEROS, ONE>(p, sm_count, stream);
}

template <int XT> cudaError_t launch_type(const Ptrs &p, bool zeros, int sm_count, cudaStream_t stream)
{
    return zeros ? launch_shape<XT, true>(p, sm_count, stream) : launch_shape<XT, false>(p, sm_count, stream);
}

int alignment(uintptr_t bits)
{
    int a = 16;
    while (bits % a) a /= 2;
    return a;
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
        p.x_align = alignment(reinterpret_cast<uintptr_t>(p.x) | uintptr_t(p.m > 1 || a.each ? p.ldx_bytes : 0));
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
