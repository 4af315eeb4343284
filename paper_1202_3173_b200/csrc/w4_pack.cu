// Laying out 4-bit weights, once for a matrix: from rows of packed nibbles to the tiles that the products read (llm.h).
//
// Positions past the inner size hold their group's zero point (their value is 0), or past the last group 8 with a scale of 0, as rows past the matrix do.
// Scales are held as S 2^-e with e such that 2^15 <= max_g |S_g| 2^-e < 2^16 in each row (the upper end of f16), and 2^e (32 bits) apart, in the exponent
// section; the products multiply their 32-bit sums by 2^e.  Both steps are exact: f16 scales only ever move up.  (Of bf16 scales only those below 2^-141 of
// their row's largest lose bits.)  A thread writes one 16-byte piece: once for a matrix, at the rate of scattered reads of nibbles; nothing that a
// product waits for.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "llm.h"
#include "strassen_b200.h"

namespace strassen {

namespace {

__device__ __forceinline__ float scale_value(uint16_t bits, int type)
{
    return type == STRASSEN_BF16 ? __uint_as_float(uint32_t(bits) << 16) : __half2float(__ushort_as_half(bits));
}

// One thread per row and chunk of a tile: 32 nibbles, 16 bytes out.
__global__ void __launch_bounds__(512) pack_weights_kernel(const W4PackArgs p)
{
    const int64_t tile = blockIdx.x;
    const int64_t nt = tile / p.lay.depth_tiles, kb = tile % p.lay.depth_tiles;
    const int c = threadIdx.x >> 7, r = threadIdx.x & 127;
    const int64_t matrix = nt / p.lay.row_tiles, in = (nt - matrix * p.lay.row_tiles) * kW4Rows + r, row = matrix * p.lay.n + in;
    const bool real = in < p.lay.n;
    const uint8_t *src = p.q + row * p.ldq;
    uint32_t out[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int64_t k0 = kb * kW4Depth + 32 * w + 8 * c;
        uint32_t pad = 8;
        // a group that is cut short has its zero point to its end
        if (p.lay.has_zeros && real && k0 / p.lay.group < (p.lay.k + p.lay.group - 1) / p.lay.group) pad = p.zeros[row * p.ldz + k0 / p.lay.group] & 15;
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t k = k0 + i;
            uint32_t v = pad;
            if (real && k < p.lay.k) v = (src[k >> 1] >> (4 * (i & 1))) & 15;
            word |= v << (4 * (i >> 1) + 16 * (i & 1));
        }
        out[w] = word;
    }
    *reinterpret_cast<uint4 *>(p.packed + tile * p.lay.tile_bytes + W4Layout::chunk_place(r, c)) = make_uint4(out[0], out[1], out[2], out[3]);
}

// One warp per row: its exponent, and its scales and zero points to their places.
__global__ void __launch_bounds__(128) pack_scales_kernel(const W4PackArgs p)
{
    const int64_t slot = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 5);         // row among the padded rows of all matrices
    const int lane = threadIdx.x & 31;
    const int64_t nt = slot / kW4Rows, matrix = nt / p.lay.row_tiles, in = slot - matrix * p.lay.row_tiles * kW4Rows;
    const int place = W4Layout::row_place(int(slot % kW4Rows));
    const int64_t groups = (p.lay.k + p.lay.group - 1) / p.lay.group;
    const int per_tile = kW4Depth / p.lay.group;
    const bool real = in < p.lay.n;
    const int64_t row = real ? matrix * p.lay.n + in : 0;
    const uint16_t *scales = static_cast<const uint16_t *>(p.scales) + row * p.lds;
    float mx = 0.f;
    for (int64_t g = lane; g < groups && real; g += 32) {
        const float v = fabsf(scale_value(scales[g], p.lay.scale_type));
        if (isfinite(v)) mx = fmaxf(mx, v);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, o));
    int e = mx > 0.f ? ilogbf(mx) - 15 : 0;
    e = e < -126 ? -126 : e;
    if (lane == 0) reinterpret_cast<float *>(p.packed + p.lay.exponent_off)[slot] = ldexpf(1.f, e);
    for (int64_t g = lane; g < p.lay.depth_tiles * per_tile; g += 32) {
        const bool on = real && g < groups;
        uint8_t *tile = p.packed + (nt * p.lay.depth_tiles + g / per_tile) * p.lay.tile_bytes;
        const int at = int(g % per_tile) * kW4Rows + place;
        const float v = on ? ldexpf(scale_value(scales[g], p.lay.scale_type), -e) : 0.f;
        reinterpret_cast<uint16_t *>(tile + kW4NibbleBytes)[at] =
            p.lay.scale_type == STRASSEN_BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(v)) : __half_as_ushort(__float2half_rn(v));
        if (p.lay.has_zeros) tile[p.lay.zero_off() + at] = on ? uint8_t(p.zeros[row * p.ldz + g] & 15) : uint8_t(8);
    }
}

}  // namespace

cudaError_t launch_w4_pack(const W4PackArgs &p, cudaStream_t stream)
{
    pack_weights_kernel<<<unsigned(p.lay.experts * p.lay.row_tiles * p.lay.depth_tiles), 512, 0, stream>>>(p);
    pack_scales_kernel<<<unsigned(p.lay.experts * p.lay.row_tiles * kW4Rows / 4), 128, 0, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace strassen
