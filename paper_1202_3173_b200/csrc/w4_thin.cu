// Products of a few rows with a matrix of 4-bit weights: arguments of the kernels in w4_thin.cuh.
#include "w4_thin.cuh"

namespace strassen {

cudaError_t launch_w4_thin(const W4Args &a, int sm_count, cudaStream_t stream)
{
    const int size = a.type == STRASSEN_E4M3 ? 1 : 2;
    thin::Ptrs p;
    p.packed = a.packed;
    p.exponents = reinterpret_cast<const float *>(a.packed + a.lay.exponent_off);
    p.tile_bytes = a.lay.tile_bytes;
    p.zero_off = a.lay.zero_off();
    p.x = static_cast<const char *>(a.x);
    p.x_scale = a.x_scale;
    p.out = static_cast<char *>(a.out);
    p.n = a.lay.n;
    p.k = a.lay.k;
    p.m = a.m;
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
    if (a.type == STRASSEN_BF16) return thin::launch_bf16(p, a.lay.group, a.lay.has_zeros, sm_count, stream);
    if (a.type == STRASSEN_F16) return thin::launch_f16(p, a.lay.group, a.lay.has_zeros, sm_count, stream);
    return thin::launch_e4m3(p, a.lay.group, a.lay.has_zeros, sm_count, stream);
}

}  // namespace strassen
