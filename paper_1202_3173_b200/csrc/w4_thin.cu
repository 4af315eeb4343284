// Products of a few rows with a matrix of 4-bit weights: arguments of the kernels in w4_thin.cuh.
#include "w4_thin.cuh"

namespace strassen {

cudaError_t launch_w4_thin(const W4Args &a, int sm_count, cudaStream_t stream)
{
    const int size = a.type == STRASSEN_E4M3 ? 1 : 2;
    constexpr int64_t most = int64_t(65535) * 8;                 // rows of x in one launch: the grid's z
    for (int64_t m0 = 0; m0 < a.m; m0 += most) {
        thin::Ptrs p;
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
        const int64_t x_rows = a.ids && a.each ? a.m * a.top : p.m;
        const uintptr_t bits = reinterpret_cast<uintptr_t>(p.x) | uintptr_t(x_rows > 1 ? p.ldx_bytes : 0);
        p.x_align = bits % 16 == 0 ? 16 : bits % 8 == 0 ? 8 : bits % 4 == 0 ? 4 : 2;
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
        if (a.type == STRASSEN_BF16) e = thin::launch_bf16(p, a.lay.group, a.lay.has_zeros, sm_count, stream);
        else if (a.type == STRASSEN_F16) e = thin::launch_f16(p, a.lay.group, a.lay.has_zeros, sm_count, stream);
        else e = thin::launch_e4m3(p, a.lay.group, a.lay.has_zeros, sm_count, stream);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace strassen
