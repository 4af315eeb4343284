// Feed-forward operators: what the host entry points (llm_api.cu) and the kernels share.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "strassen_b200.h"

namespace strassen {

// Programmatic dependent launch: the kernels below may be placed on the GPU while the one before them in the stream drains, and let the one
// behind them do the same; every CTA waits here, before its first access to memory, until the work before it is done and visible.
__device__ __forceinline__ void after_work_before()
{
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Launches `kernel` so; cluster: CTAs of a cluster along x and y.
template <class... Parameters, class... Arguments>
cudaError_t launch_after(void (*kernel)(Parameters...), dim3 grid, dim3 block, size_t bytes, cudaStream_t stream, dim3 cluster, const Arguments &...arguments)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster.x;
    attr[1].val.clusterDim.y = cluster.y;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster.x * cluster.y > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, arguments...);
}

constexpr float kE4M3Max = 448.f;                    // largest finite e4m3
constexpr float kMinRowScale = 5.421010862427522e-20f;   // 2^-64: scale of a row of zeros; its reciprocal is finite

// ---- passes over rows (rows8.cu) ----------------------------------------------------------------------------------
struct RowArgs {
    int64_t m, k;
    int type;                    // STRASSEN_BF16 / F16 / F32
    const void *a, *b;           // norm: x and the residual (or NULL); gate: gate and up
    int64_t lda, ldb;            // elements between rows
    const void *weight;          // norm only
    float eps;
    void *sum;                   // norm with a residual: x + residual
    int64_t lds;
    uint8_t *q;                  // e4m3
    int64_t ldq;
    float *scale;
};
cudaError_t launch_rms_norm_quant(const RowArgs &a, int sm_count, cudaStream_t stream);
cudaError_t launch_silu_mul_quant(const RowArgs &a, int sm_count, cudaStream_t stream);
cudaError_t rows8_gave_up(int *flag);        // reads and clears the flag of a copy that did not come

// ---- routing (route.cu) -------------------------------------------------------------------------------------------
struct RouteArgs {
    int64_t tokens;
    int experts, type;
    const void *logits;
    int64_t ld;
    const float *bias;
    int softmax, groups, top_groups, top, renormalize;
    float factor;
    int *ids;
    float *weights;
    uint32_t size_magic;
};
constexpr int kMostExperts = 1024, kMostTop = 32, kMostGroups = 32;
cudaError_t launch_route(RouteArgs p, cudaStream_t stream);

// ---- 4-bit weights (w4_pack.cu, w4_thin.cu, w4_tiles.cu) -----------------------------------------------------------
// Laid-out weights: tiles of 128 rows x 128 inner positions, one after another along the inner dimension, then along the
// rows.  A tile is eight pieces of 16 rows, 1 KB each, in which the 64 bytes of rows g = 0..7 come first and those of rows g + 8 second.  The four
// 16-byte chunks c of a row hold k = 32 w + 8 c + (0..7), w = 0..3 their 32-bit words, in the nibble order 0, 2, 4, 6, 1, 3, 5, 7 from the lowest nibble up,
// so that (word & 0x000f000f) is the pair k = 0, 1, ((word >> 4) & 0x000f000f) the pair 2, 3, and so on.  A piece is then the operand of eight
// m16n8k16 products with two 16-byte loads of a lane, 512 neighbouring bytes of the warp each; and the rows of 32 lanes of tensor memory are in pieces
// too: chunk c of row r is in place c ^ (r / 2 & 3), so that neighbouring rows' are in different banks.
// The nibbles are followed by the tile's scales (128 of 16 bits for each group) and its zero points (128 bytes for each group), so that a tile is
// one piece of memory.
constexpr int kW4Rows = 128, kW4Depth = 128, kW4NibbleBytes = kW4Rows * kW4Depth / 2;

struct W4Layout {
    int64_t n, k;
    int64_t experts;             // matrices of this size, one after another
    int group;                   // 32, 64 or 128
    int scale_type;              // STRASSEN_BF16 / F16
    int has_zeros;
    int64_t row_tiles, depth_tiles;      // of one matrix
    int tile_bytes;
    // byte offset of the rows' exponents (w4_pack.cu) in the packed memory, and its size
    size_t exponent_off, bytes;

    __host__ __device__ int zero_off() const { return kW4NibbleBytes + kW4Depth / group * kW4Rows * 2; }     // within a tile
    // byte of chunk c of row r (0..127) of a tile
    __host__ __device__ static int chunk_place(int r, int c) { return (r >> 3) * 512 + (r & 7) * 64 + (c ^ (r >> 1 & 3)) * 16; }
    // position of row r (0..127) of a tile in the scale and zero sections: rows g and g + 8 of a 16-row piece are neighbours
    __host__ __device__ static int row_place(int r) { return (r & ~15) | ((r & 7) << 1) | ((r >> 3) & 1); }
};

struct W4Args {
    W4Layout lay;
    const uint8_t *packed;
    int64_t m;
    int type;                    // STRASSEN_BF16 / F16 / E4M3
    const void *x;
    int64_t ldx;
    const float *x_scale;
    int out_type;                // STRASSEN_BF16 / F16
    void *out;
    int64_t ldo;
    void *workspace;
    // products of experts: m tokens, `top` rows of ids each; x has a row for each token, or with `each` for each of its ids
    const int *ids;
    int64_t top;
    bool each;
    const float *weights;        // NULL: a row of results for each id
};

struct W4PackArgs {
    W4Layout lay;
    const uint8_t *q;
    int64_t ldq;
    const void *scales;
    int64_t lds;
    const uint8_t *zeros;
    int64_t ldz;
    uint8_t *packed;
};
cudaError_t launch_w4_pack(const W4PackArgs &a, cudaStream_t stream);
// Most rows of x that the kernel for few rows (w4_thin.cu) takes; beyond that the tiles of w4_tiles.cu.  Few rows against tiles: 4096 x 4096 bf16, 8 rows
// 7.7 and 7.8 us, 16 rows 9.8 and 7.8, 17 to 32 rows 14.7 and 8.0; 16384 x 4096 e4m3 with zero points, 8 rows 16.4 and 15.6, 16 rows 25.2 and 15.8.  Time
// alone would change over at 8; up to 16 it is the promise that no weight is rounded for a batch that small.
constexpr int64_t kThinRows = STRASSEN_W4_THIN_ROWS;
// A run of rows of x that one matrix multiplies: rows first .. first + count - 1 of the rows in order.
struct W4Tile {
    int expert, first, count, unused;
};
int64_t w4_tiles_workspace(const W4Args &a);        // bytes; 0: none is needed
cudaError_t launch_w4_tiles(const W4Args &a, int sm_count, cudaStream_t stream);
cudaError_t read_gave_up(int *flag);        // reads and clears the flag of w4_tiles.cu
// Most ids for which every id's matrix is read by itself (w4_thin.cu); beyond that the rows are put in order of their experts.  64 experts of 2048 x 2048,
// by itself against in order: 16 ids 13 and 25 us, 32 ids 22 and 32, 64 ids 41 and 44, 128 ids 74 and 53.  Fewer experts share more (8 of 4096 x 4096,
// 40 ids: 87 and 36 us); up to 32 ids, as up to 16 rows, no weight is rounded.
constexpr int64_t kThinIds = STRASSEN_W4_THIN_IDS;
int64_t w4_experts_workspace(const W4Args &a);
cudaError_t launch_w4_experts_tiles(const W4Args &a, int sm_count, cudaStream_t stream);
cudaError_t launch_w4_thin(const W4Args &a, int sm_count, cudaStream_t stream);

}  // namespace strassen
