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
// A thread has pieces of 8 neighbouring elements.  Rows that do not start at a multiple of 16 bytes (odd lengths, halves of odd rows) are read and
// written in the same 16-byte accesses: two aligned words around a piece are shifted into place, and on the way out neighbouring lanes pass
// each other the bytes that belong to the other's word.  Bound by HBM for many rows, by launch and memory latency for few.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "llm.h"
#include "strassen_b200.h"

namespace strassen {

namespace {

__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// A piece of 8 elements in 32-bit words, as they lie in memory.
template <class T> struct Words {
    static constexpr int N = 8 * int(sizeof(T)) / 4;
    uint32_t w[N];
};

__device__ __forceinline__ void unpack(const Words<float> &p, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(p.w[i]);
}
__device__ __forceinline__ void unpack(const Words<__nv_bfloat16> &p, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(p.w[i] << 16);
        v[2 * i + 1] = __uint_as_float(p.w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const Words<__half> &p, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(__half2(__ushort_as_half(uint16_t(p.w[i])), __ushort_as_half(uint16_t(p.w[i] >> 16))));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ void pack(Words<float> &p, const float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) p.w[i] = __float_as_uint(v[i]);
}
__device__ __forceinline__ void pack(Words<__nv_bfloat16> &p, const float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p.w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
}
__device__ __forceinline__ void pack(Words<__half> &p, const float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(p.w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
}

template <int N> __device__ __forceinline__ void load_words(uint32_t (&w)[N], const void *at)
{
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const uint4 u = static_cast<const uint4 *>(at)[i];
        w[4 * i] = u.x;
        w[4 * i + 1] = u.y;
        w[4 * i + 2] = u.z;
        w[4 * i + 3] = u.w;
    }
}

// Elements k .. k + 7 of a row of `size`; zeros past its end.  lo, hi: the memory of the whole matrix, which wider accesses do not leave.
template <class T> __device__ __forceinline__ void load(Words<T> &p, const T *row, int64_t k, int64_t size, uintptr_t lo, uintptr_t hi)
{
    constexpr int N = Words<T>::N;
    const uintptr_t at = reinterpret_cast<uintptr_t>(row + k), off = at & 15, from = at - off;
    if (k + 8 <= size && off == 0) {
        load_words<N>(p.w, reinterpret_cast<const void *>(at));
    } else if (k + 8 <= size && from >= lo && from + 4 * N + 16 <= hi) {
        // the aligned words around the piece, moved down by `off` bytes
        uint32_t a[N + 4];
        load_words<N + 4>(a, reinterpret_cast<const void *>(from));
        if (off & 8) {
#pragma unroll
            for (int i = 0; i < N + 2; ++i) a[i] = a[i + 2];
        }
        if (off & 4) {
#pragma unroll
            for (int i = 0; i < N + 1; ++i) a[i] = a[i + 1];
        }
#pragma unroll
        for (int i = 0; i < N; ++i) p.w[i] = __funnelshift_r(a[i], a[i + 1], 8 * (off & 3));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) p.w[i] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < size) {
                if (sizeof(T) == 4) p.w[i] = reinterpret_cast<const uint32_t *>(row)[k + i];
                else p.w[i / 2] |= uint32_t(reinterpret_cast<const uint16_t *>(row)[k + i]) << (16 * (i & 1));
            }
    }
}

// The same way out.  The lanes of a warp have neighbouring pieces, lane 0 the first; all of them come here, with k >= size where there is none.
template <class T> __device__ __forceinline__ void store(const Words<T> &p, T *row, int64_t k, int64_t size)
{
    constexpr int N = Words<T>::N;
    const int lane = threadIdx.x & 31;
    const uintptr_t at = reinterpret_cast<uintptr_t>(row + k), off = at & 15;        // the same in all lanes
    if (off == 0 && k + 8 <= size) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) reinterpret_cast<uint4 *>(at)[i] = make_uint4(p.w[4 * i], p.w[4 * i + 1], p.w[4 * i + 2], p.w[4 * i + 3]);
        return;
    }
    const bool full = k + 8 <= size;
    int first = 0, last = k >= size ? 0 : full ? 8 : int(size - k);                 // what is left to write element by element
    if (off != 0) {
        // aligned words that end with this piece's: `off` bytes of the lane below, then this lane's own
        uint32_t a[N + 4];
#pragma unroll
        for (int i = 0; i < N; ++i) a[i + 4] = p.w[i];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = __shfl_up_sync(~0u, p.w[N - 4 + i], 1);
        const bool above = __shfl_down_sync(~0u, int(full), 1) && lane < 31;        // the lane above writes this one's last bytes
        if (full && lane > 0) {
            const uintptr_t up = 16 - off;                                          // how far the piece moves up from an aligned place
            uint32_t b[N + 4];
#pragma unroll
            for (int i = 0; i < N + 4; ++i) b[i] = a[i];
            if (up & 8) {
#pragma unroll
                for (int i = 0; i < N + 2; ++i) b[i] = b[i + 2];
            }
            if (up & 4) {
#pragma unroll
                for (int i = 0; i < N + 1; ++i) b[i] = b[i + 1];
            }
            uint32_t out[N];
#pragma unroll
            for (int i = 0; i < N; ++i) out[i] = __funnelshift_r(b[i], b[i + 1], 8 * (up & 3));
#pragma unroll
            for (int i = 0; i < N / 4; ++i) reinterpret_cast<uint4 *>(at - off)[i] = make_uint4(out[4 * i], out[4 * i + 1], out[4 * i + 2], out[4 * i + 3]);
            first = above ? 8 : 8 - int(off / sizeof(T));
        } else if (above) {
            last = 8 - int(off / sizeof(T));
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i >= first && i < last) {
            if (sizeof(T) == 4) reinterpret_cast<uint32_t *>(row)[k + i] = p.w[i * N / 8];
            else reinterpret_cast<uint16_t *>(row)[k + i] = uint16_t(p.w[i / 2 * (N / 4)] >> (16 * (i & 1)));
        }
}

__device__ __forceinline__ void store_e4m3(uint8_t *row, int64_t k, int64_t size, const float (&v)[8])
{
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i], v[4 * i + 1]), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i + 2], v[4 * i + 3]), __NV_SATFINITE, __NV_E4M3);
        w[i] = lo | (hi << 16);
    }
    if (reinterpret_cast<uintptr_t>(row) % 8 == 0 && k + 8 <= size) {
        *reinterpret_cast<uint2 *>(row + k) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < size) row[k + i] = uint8_t(w[i / 4] >> (8 * (i & 3)));
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

template <class T> struct Range {
    uintptr_t lo, hi;
    __device__ Range(const void *p, int64_t m, int64_t k, int64_t ld) : lo(reinterpret_cast<uintptr_t>(p)), hi(lo + uintptr_t((m - 1) * ld + k) * sizeof(T)) {}
};

// The values of a piece before the row's factor: h w for the norm, silu(g) u for the gate, and what they add to the row's sum and maximum.
// exp and the quotient are the fast forms: some 2^-21 of a value, against 2^-5 of its rounding to e4m3.
template <int MODE> __device__ __forceinline__ void values(float (&x)[8], const float (&y)[8], const float (&w)[8], float (&v)[8], float &sq, float &mx)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (MODE == GATE) {
            v[i] = __fdividef(x[i], 1.f + __expf(-x[i])) * y[i];
        } else {
            if (MODE == NORM_RESIDUAL) x[i] += y[i];
            sq += x[i] * x[i];
            v[i] = x[i] * w[i];
        }
        mx = max_nan(mx, fabsf(v[i]));
    }
}

// The row's scale, and the factor that takes a value before the row's factor to the e4m3 range.
template <int MODE> __device__ __forceinline__ float row_factor(float sq, float mx, int64_t k, float eps, float &scale)
{
    const float inv = MODE == GATE ? 1.f : 1.f / sqrtf(sq / float(k) + eps);
    const float s = mx * inv / kE4M3Max;
    scale = s <= kMinRowScale ? kMinRowScale : s;        // NaN stays NaN
    return inv / scale;
}

// One CTA per row, the row in registers: ITEMS pieces a thread, their loads all under way before the first is used.
template <class T, int MODE, int ITEMS, int THREADS> __global__ void __launch_bounds__(THREADS) row_kernel(const RowArgs p)
{
    __shared__ float part[2][32];
    after_work_before();
    const int64_t r = blockIdx.x;
    const T *const a = static_cast<const T *>(p.a) + r * p.lda, *const b = static_cast<const T *>(p.b) + r * p.ldb, *const w = static_cast<const T *>(p.weight);
    const Range<T> range_a(p.a, p.m, p.k, p.lda), range_b(p.b, p.m, p.k, p.ldb), range_w(p.weight, 1, p.k, p.k);
    Words<T> pa[ITEMS], pb[ITEMS], pw[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int64_t c = (i * int64_t(blockDim.x) + threadIdx.x) * 8;
        if (c < p.k) {
            load(pa[i], a, c, p.k, range_a.lo, range_a.hi);
            if (MODE != NORM) load(pb[i], b, c, p.k, range_b.lo, range_b.hi);
            if (MODE != GATE) load(pw[i], w, c, p.k, range_w.lo, range_w.hi);
        } else {
#pragma unroll
            for (int j = 0; j < Words<T>::N; ++j) pa[i].w[j] = pb[i].w[j] = pw[i].w[j] = 0;
        }
    }
    // kept until the row's factor is known: h of a norm, v of a gate (the norm's weights stay as they came)
    float kept[ITEMS][8];
    float sq = 0.f, mx = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        float y[8], f[8], v[8];
        unpack(pa[i], kept[i]);
        if (MODE != NORM) unpack(pb[i], y);
        if (MODE != GATE) unpack(pw[i], f);
        values<MODE>(kept[i], y, f, v, sq, mx);
        if (MODE == GATE) memcpy(kept[i], v, sizeof(v));
    }
    reduce_row(sq, mx, part);
    float scale;
    const float factor = row_factor<MODE>(sq, mx, p.k, p.eps, scale);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int64_t c = (i * int64_t(blockDim.x) + threadIdx.x) * 8;
        if (MODE == NORM_RESIDUAL) {
            Words<T> ps;
            pack(ps, kept[i]);
            store(ps, static_cast<T *>(p.sum) + r * p.lds, c, p.k);
        }
        float f[8], v[8];
        if (MODE != GATE) unpack(pw[i], f);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = kept[i][j] * (MODE == GATE ? factor : f[j] * factor);
        if (c < p.k) store_e4m3(p.q + r * p.ldq, c, p.k, v);
    }
    if (threadIdx.x == 0) p.scale[r] = scale;
}

// Rows longer than the registers of a CTA: read twice, the second time for the most part from L2.  A thread reads a piece again before it or the lane
// beside it writes the sum there, so the sum may take the residual's place here too.
template <class T, int MODE> __global__ void __launch_bounds__(1024) long_row_kernel(const RowArgs p)
{
    __shared__ float part[2][32];
    after_work_before();
    const int64_t r = blockIdx.x;
    const T *const a = static_cast<const T *>(p.a) + r * p.lda, *const b = static_cast<const T *>(p.b) + r * p.ldb, *const w = static_cast<const T *>(p.weight);
    const Range<T> range_a(p.a, p.m, p.k, p.lda), range_b(p.b, p.m, p.k, p.ldb), range_w(p.weight, 1, p.k, p.k);
    float sq = 0.f, mx = 0.f, scale = 0.f, factor = 0.f;
    for (int pass = 0; pass < 2; ++pass) {
        for (int64_t c0 = 0; c0 < p.k; c0 += int64_t(blockDim.x) * 8) {
            const int64_t c = c0 + int64_t(threadIdx.x) * 8;
            float x[8] = {}, y[8] = {}, f[8] = {}, v[8];
            if (c < p.k) {
                Words<T> t;
                load(t, a, c, p.k, range_a.lo, range_a.hi);
                unpack(t, x);
                if (MODE != NORM) {
                    load(t, b, c, p.k, range_b.lo, range_b.hi);
                    unpack(t, y);
                }
                if (MODE != GATE) {
                    load(t, w, c, p.k, range_w.lo, range_w.hi);
                    unpack(t, f);
                }
            }
            values<MODE>(x, y, f, v, sq, mx);
            if (pass == 0) continue;
            if (MODE == NORM_RESIDUAL) {
                // a piece of a misaligned row is read with its neighbours' bytes: all reads of these pieces come before the writes
                __syncthreads();
                Words<T> t;
                pack(t, x);
                store(t, static_cast<T *>(p.sum) + r * p.lds, c, p.k);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= factor;
            if (c < p.k) store_e4m3(p.q + r * p.ldq, c, p.k, v);
        }
        if (pass == 0) {
            reduce_row(sq, mx, part);
            factor = row_factor<MODE>(sq, mx, p.k, p.eps, scale);
        }
    }
    if (threadIdx.x == 0) p.scale[r] = scale;
}

template <class T, int MODE> cudaError_t launch_type(const RowArgs &p, cudaStream_t stream)
{
    const int64_t pieces = (p.k + 7) / 8;
    const dim3 grid(unsigned(p.m));
    const auto threads = [&](int items) { return dim3(unsigned((pieces + 32 * items - 1) / (32 * items) * 32)); };
    // two pieces a thread for rows that then still make a CTA of 128 threads or more: more of the row under way for each of its registers
    if (pieces <= 256) return launch_after(row_kernel<T, MODE, 1, 256>, grid, threads(1), 0, stream, dim3(1, 1), p);
    if (pieces <= 1024) return launch_after(row_kernel<T, MODE, 2, 512>, grid, threads(2), 0, stream, dim3(1, 1), p);
    if (pieces <= 2048) return launch_after(row_kernel<T, MODE, 2, 1024>, grid, threads(2), 0, stream, dim3(1, 1), p);
    return launch_after(long_row_kernel<T, MODE>, grid, dim3(1024), 0, stream, dim3(1, 1), p);
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
