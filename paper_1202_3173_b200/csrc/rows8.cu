// Rows to 8 bits: the root-mean-square norm with the residual's addition, and the gated activation, each with an e4m3
// output and one scale per row.
//
//   norm   h = x + r,  inv = 1 / sqrt(mean_k h_k^2 + eps),  v_k = h_k w_k inv
//   gate   v_k = g_k / (1 + exp(-g_k)) u_k
//   both   s = max(max_k |v_k| / 448, 2^-64),  q_k = e4m3(v_k / s)
//
// inv > 0 is the same for the whole row, so max_k |v_k| = inv max_k |h_k w_k|: the sum of squares and the maximum come out of ONE
// reduction, and a row that fits the registers of its CTA is read once.  Sums, the maximum and v are held in 32 bits; the
// only roundings are h to its own type (the residual stream) and q.  A NaN, or an infinity in a norm's row, makes the
// row's scale and outputs NaN (the maximum propagates NaN), as the formulas say.
//
// Bound by HBM for many rows, by launch and memory latency for few.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "llm.h"
#include "strassen_b200.h"

namespace strassen {

namespace {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// VEC consecutive elements: 16-byte accesses for VEC = 8 (two of them for f32), single elements for VEC = 1.
template <class T, int VEC> struct Piece {
    T v[VEC];
    __device__ __forceinline__ void load(const T *p)
    {
        if constexpr (VEC == 1) {
            v[0] = *p;
        } else {
            constexpr int N16 = VEC * int(sizeof(T)) / 16;
            uint4 w[N16];
#pragma unroll
            for (int i = 0; i < N16; ++i) w[i] = reinterpret_cast<const uint4 *>(p)[i];
            memcpy(v, w, sizeof(v));
        }
    }
    __device__ __forceinline__ void store(T *p) const
    {
        if constexpr (VEC == 1) {
            *p = v[0];
        } else {
            constexpr int N16 = VEC * int(sizeof(T)) / 16;
            uint4 w[N16];
            memcpy(w, v, sizeof(v));
#pragma unroll
            for (int i = 0; i < N16; ++i) reinterpret_cast<uint4 *>(p)[i] = w[i];
        }
    }
};

template <int VEC> __device__ __forceinline__ void store_e4m3(uint8_t *p, const float (&v)[VEC])
{
    if constexpr (VEC == 1) {
        *p = __nv_cvt_float_to_fp8(v[0], __NV_SATFINITE, __NV_E4M3);
    } else {
        uint32_t w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i], v[4 * i + 1]), __NV_SATFINITE, __NV_E4M3);
            const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i + 2], v[4 * i + 3]), __NV_SATFINITE, __NV_E4M3);
            w[i] = lo | (hi << 16);
        }
        *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
    }
}

// Sum and maximum over the CTA, the same bits in every thread (each adds the warps' values in the same order).
__device__ __forceinline__ void reduce_row(float &sum, float &mx, float (*part)[32])
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        sum += __shfl_xor_sync(~0u, sum, o);
        mx = max_nan(mx, __shfl_xor_sync(~0u, mx, o));
    }
    const int warps = blockDim.x >> 5;
    if (warps == 1) return;
    if ((threadIdx.x & 31) == 0) {
        part[0][threadIdx.x >> 5] = sum;
        part[1][threadIdx.x >> 5] = mx;
    }
    __syncthreads();
    const int lane = threadIdx.x & 31;
    sum = lane < warps ? part[0][lane] : 0.f;
    mx = lane < warps ? part[1][lane] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        sum += __shfl_xor_sync(~0u, sum, o);
        mx = max_nan(mx, __shfl_xor_sync(~0u, mx, o));
    }
}

enum { GATE = 0, NORM = 1, NORM_RESIDUAL = 2 };

template <class T, int VEC, int MODE> struct Row {
    const T *a, *b, *w;
    T *sum;
    uint8_t *q;

    // The VEC values at k before the row's factor: h w for the norm, silu(g) u for the gate.
    __device__ __forceinline__ void values(int k, float (&v)[VEC], float (&h)[VEC], float &sq, float &mx) const
    {
        Piece<T, VEC> pa, pb;
        pa.load(a + k);
        if (MODE != NORM) pb.load(b + k);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float x = to_f32(pa.v[i]);
            if (MODE == GATE) v[i] = x / (1.f + expf(-x)) * to_f32(pb.v[i]);
            else h[i] = MODE == NORM_RESIDUAL ? x + to_f32(pb.v[i]) : x;
        }
        if (MODE != GATE) {
            Piece<T, VEC> pw;
            pw.load(w + k);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                sq += h[i] * h[i];
                v[i] = h[i] * to_f32(pw.v[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) mx = max_nan(mx, fabsf(v[i]));
    }
    __device__ __forceinline__ void finish(int k, const float (&v)[VEC], const float (&h)[VEC], float factor) const
    {
        float y[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) y[i] = v[i] * factor;
        store_e4m3<VEC>(q + k, y);
        if (MODE == NORM_RESIDUAL) {
            Piece<T, VEC> ps;
#pragma unroll
            for (int i = 0; i < VEC; ++i) ps.v[i] = from_f32<T>(h[i]);
            ps.store(sum + k);
        }
    }
};

// The row's scale, and the factor that takes a value before the row's factor to the e4m3 range.
template <int MODE> __device__ __forceinline__ float row_factor(float sq, float mx, int k, float eps, float &scale)
{
    const float inv = MODE == GATE ? 1.f : 1.f / sqrtf(sq / float(k) + eps);
    const float s = mx * inv / kE4M3Max;
    scale = s <= kMinRowScale ? kMinRowScale : s;        // NaN stays NaN
    return inv / scale;
}

// One CTA per row, the row in registers: ITEMS pieces of VEC values a thread.
template <class T, int VEC, int MODE, int ITEMS, int THREADS>
__global__ void __launch_bounds__(THREADS) row_kernel(const RowArgs p)
{
    __shared__ float part[2][32];
    const int64_t r = blockIdx.x;
    const int k = int(p.k);
    const Row<T, VEC, MODE> row = {static_cast<const T *>(p.a) + r * p.lda, static_cast<const T *>(p.b) + r * p.ldb, static_cast<const T *>(p.weight),
                                   static_cast<T *>(p.sum) + r * p.lds, p.q + r * p.ldq};
    float v[ITEMS][VEC], h[ITEMS][VEC];
    float sq = 0.f, mx = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int c = (i * int(blockDim.x) + int(threadIdx.x)) * VEC;
        if (c < k) row.values(c, v[i], h[i], sq, mx);
    }
    reduce_row(sq, mx, part);
    float scale;
    const float factor = row_factor<MODE>(sq, mx, k, p.eps, scale);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int c = (i * int(blockDim.x) + int(threadIdx.x)) * VEC;
        if (c < k) row.finish(c, v[i], h[i], factor);
    }
    if (threadIdx.x == 0) p.scale[r] = scale;
}

// Rows longer than the registers of a CTA: read twice, the second time for the most part from L2.  A thread reads an
// element again before it writes the sum there, so the sum may take the residual's place here too.
template <class T, int VEC, int MODE> __global__ void __launch_bounds__(1024) long_row_kernel(const RowArgs p)
{
    __shared__ float part[2][32];
    const int64_t r = blockIdx.x;
    const Row<T, VEC, MODE> row = {static_cast<const T *>(p.a) + r * p.lda, static_cast<const T *>(p.b) + r * p.ldb, static_cast<const T *>(p.weight),
                                   static_cast<T *>(p.sum) + r * p.lds, p.q + r * p.ldq};
    float v[VEC], h[VEC];
    float sq = 0.f, mx = 0.f;
    for (int64_t c = int64_t(threadIdx.x) * VEC; c < p.k; c += int64_t(blockDim.x) * VEC) row.values(int(c), v, h, sq, mx);
    reduce_row(sq, mx, part);
    float scale;
    const float factor = row_factor<MODE>(sq, mx, int(p.k), p.eps, scale);
    float none_sq = 0.f, none_mx = 0.f;
    for (int64_t c = int64_t(threadIdx.x) * VEC; c < p.k; c += int64_t(blockDim.x) * VEC) {
        row.values(int(c), v, h, none_sq, none_mx);
        row.finish(int(c), v, h, factor);
    }
    if (threadIdx.x == 0) p.scale[r] = scale;
}

int threads_for(int64_t pieces) { return int((pieces + 31) / 32 * 32); }

template <class T, int VEC, int MODE> void launch_rows(const RowArgs &p, cudaStream_t stream)
{
    const int64_t pieces = (p.k + VEC - 1) / VEC;
    const unsigned grid = unsigned(p.m);
    constexpr int BIG = VEC == 1 ? 16 : 2;      // pieces per thread of the larger register form
    if (pieces <= 1024) row_kernel<T, VEC, MODE, 1, 1024><<<grid, threads_for(pieces), 0, stream>>>(p);
    else if (pieces <= 1024 * BIG) row_kernel<T, VEC, MODE, BIG, 1024><<<grid, threads_for((pieces + BIG - 1) / BIG), 0, stream>>>(p);
    else long_row_kernel<T, VEC, MODE><<<grid, 1024, 0, stream>>>(p);
}

bool aligned(const void *p, int64_t ld, int size, int bytes)
{
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && (ld * size) % bytes == 0;
}

template <class T, int MODE> cudaError_t launch_type(const RowArgs &p, cudaStream_t stream)
{
    const int t = int(sizeof(T));
    bool vec = p.k % 8 == 0 && aligned(p.a, p.lda, t, 16) && aligned(p.q, p.ldq, 1, 8);
    if (MODE != NORM) vec = vec && aligned(p.b, p.ldb, t, 16);
    if (MODE != GATE) vec = vec && aligned(p.weight, 0, t, 16);
    if (MODE == NORM_RESIDUAL) vec = vec && aligned(p.sum, p.lds, t, 16);
    if (vec) launch_rows<T, 8, MODE>(p, stream);
    else launch_rows<T, 1, MODE>(p, stream);
    return cudaGetLastError();
}

template <int MODE> cudaError_t launch_mode(const RowArgs &p, cudaStream_t stream)
{
    if (p.m == 0) return cudaSuccess;
    switch (p.type) {
    case STRASSEN_BF16: return launch_type<__nv_bfloat16, MODE>(p, stream);
    case STRASSEN_F16: return launch_type<__half, MODE>(p, stream);
    case STRASSEN_F32: return launch_type<float, MODE>(p, stream);
    }
    return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_rms_norm_quant(const RowArgs &p, cudaStream_t stream)
{
    return p.b ? launch_mode<NORM_RESIDUAL>(p, stream) : launch_mode<NORM>(p, stream);
}

cudaError_t launch_silu_mul_quant(const RowArgs &p, cudaStream_t stream) { return launch_mode<GATE>(p, stream); }

}  // namespace strassen
