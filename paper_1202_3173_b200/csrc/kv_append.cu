// Rotary embedding of queries and keys, and keys and values stored into a paged cache.
//
// A row of a head (up to 128 values) is 16 lanes' work, 8 values each: a row's pairs (x, y) turn by the angle p f,
//     (x, y) -> (x cos - y sin, x sin + y cos),
// and an 8-bit row's largest value is found among the 16.  Where pairs are a half of the turned values apart, a lane reads its partners' 8 values too
// (they are in the first cache): it needs both to write its own.  A CTA takes a token; its angles, the same for all heads, are found once:
// p f / 2 pi in 64 bits, of which the fraction is an angle in 32 bits with an error of 2^-24 of a turn's size wherever p is.
//
// Bound by the bytes, read once and written once.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "attention.h"
#include "llm.h"

namespace strassen {

namespace {

constexpr int THREADS = 256, ROWS = THREADS / 16;

template <bool BF16> __device__ __forceinline__ float2 two_floats(uint32_t w)
{
    if (BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}
template <bool BF16> __device__ __forceinline__ uint32_t two_16_bits(float lo, float hi)
{
    uint32_t d;
    if (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}

// The sequence that row t of q belongs to, -1 if none.
__device__ __forceinline__ int sequence_of(const SequenceArgs &s, int64_t t)
{
    if (!s.offsets) return int(t);
    int lo = 0, hi = s.batch - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s.offsets[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    const NewTokens n = new_tokens(s, lo);
    return t >= n.first && t < n.end ? lo : -1;
}

template <bool BF16, bool WIDE> __device__ __forceinline__ void load8(float (&x)[8], const uint16_t *row, int at)
{
    if (WIDE) {
        const uint4 u = *reinterpret_cast<const uint4 *>(row + at);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = two_floats<BF16>(w[i]);
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = two_floats<BF16>(row[at + i]).x;
    }
}

template <bool BF16, bool E4M3, bool WIDE> __global__ void __launch_bounds__(THREADS) append_kernel(const AppendArgs p)
{
    __shared__ float angles[2][kMostHeadSize];       // cos and sin for each value of a row; 1 and 0 for those that do not turn
    after_work_before();
    const int64_t t = blockIdx.x;
    const int d = p.cache.d, half = p.rotary / 2, lane = threadIdx.x & 15, first = 8 * lane;
    const int b = sequence_of(p.seq, t);
    if (b < 0) return;
    const NewTokens n = new_tokens(p.seq, b);
    const int64_t position = n.length - (n.end - t);
    if (position < 0) return;
    for (int i = threadIdx.x; i < kMostHeadSize; i += THREADS) {
        float c = 1.f, s = 0.f;
        if (i < p.rotary) {
            // 1 / 2 pi
            const double turns = double(position) * double(p.frequencies[p.interleaved ? i / 2 : i < half ? i : i - half]) * 0.15915494309189535;
            sincospif(float(2 * (turns - rint(turns))), &s, &c);
            if (p.interleaved ? !(i & 1) : i < half) s = -s;
        }
        angles[0][i] = c;
        angles[1][i] = s;
    }
    __syncthreads();
    const int page = page_of(p.cache, p.seq, b, position);
    const int64_t slot = position & ((1 << p.cache.page_shift) - 1);
    const int rows = p.heads + 2 * p.cache.kv_heads;
    for (int r = blockIdx.y * ROWS + (threadIdx.x >> 4); r < (rows + ROWS - 1) / ROWS * ROWS; r += gridDim.y * ROWS) {
        const bool is_q = r < p.heads, is_v = r >= p.heads + p.cache.kv_heads;
        const int h = is_q ? r : is_v ? r - p.heads - p.cache.kv_heads : r - p.heads;
        const Heads &from = is_q ? p.q : is_v ? p.v : p.k;
        const uint16_t *row = static_cast<const uint16_t *>(from.p) + t * from.row + h * from.head;
        const bool mine = r < rows && first < d;
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0.f;
        if (mine) {
            load8<BF16, WIDE>(x, row, first);
            if (!is_v && first < p.rotary) {
                float y[8];
                if (p.interleaved) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = x[i ^ 1];
                } else if (WIDE && half % 8 == 0) {
                    load8<BF16, WIDE>(y, row, first < half ? first + half : first - half);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int at = first + i;
                        y[i] = at < half ? two_floats<BF16>(row[at + half]).x : at < p.rotary ? two_floats<BF16>(row[at - half]).x : 0.f;
                    }
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (first + i < p.rotary) x[i] = x[i] * angles[0][first + i] + y[i] * angles[1][first + i];
            }
        }
        __syncwarp();                    // in place: a row is read by all before it is written
        if (is_q) {
            if (!mine) continue;
            uint16_t *to = static_cast<uint16_t *>(p.out) + t * p.out_row + h * p.out_head + first;
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = two_16_bits<BF16>(x[2 * i], x[2 * i + 1]);
            if (WIDE) {
                *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) to[i] = uint16_t(w[i / 2] >> (16 * (i & 1)));
            }
            continue;
        }
        uint8_t *const to = (is_v ? p.cache.v : p.cache.k) + page * p.cache.page_stride + h * p.cache.head_stride + slot * p.cache.row_stride + first * (E4M3 ? 1 : 2);
        if (E4M3) {
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(x[i]));
#pragma unroll
            for (int i = 0; i < 8; ++i) most = x[i] == x[i] ? most : x[i];      // NaN stays
            for (int i = 8; i > 0; i >>= 1) {
                const float other = __shfl_xor_sync(0xffffu << (threadIdx.x & 16), most, i);       // the other half of the warp may have a row of q
                most = most == most ? (other == other ? fmaxf(most, other) : other) : most;
            }
            const float scale = most == most ? fmaxf(most / kE4M3Max, kMinRowScale) : most;
            if (!mine || page < 0) continue;
            uint32_t w[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float *v = x + 4 * i;
                const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[0] / scale, v[1] / scale), __NV_SATFINITE, __NV_E4M3);
                const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[2] / scale, v[3] / scale), __NV_SATFINITE, __NV_E4M3);
                w[i] = lo | hi << 16;
            }
            *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
            if (lane == 0) (is_v ? p.cache.v_scale : p.cache.k_scale)[((int64_t(page) * p.cache.kv_heads + h) << p.cache.page_shift) + slot] = scale;
        } else if (mine && page >= 0) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = two_16_bits<BF16>(x[2 * i], x[2 * i + 1]);
            *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

}  // namespace

cudaError_t launch_append(const AppendArgs &a, int sm_count, cudaStream_t stream)
{
    const int rows = a.heads + 2 * a.cache.kv_heads, parts = (rows + ROWS - 1) / ROWS;
    // one CTA a token and all of its rows, where there are tokens enough to fill the GPU
    const dim3 grid(unsigned(a.seq.tokens), unsigned(a.seq.tokens >= sm_count ? 1 : parts), 1);
    const bool e = a.cache.type == STRASSEN_E4M3;
    void (*kernel)(AppendArgs) = a.type == STRASSEN_BF16 ? (e ? (a.wide ? append_kernel<true, true, true> : append_kernel<true, true, false>) : (a.wide ? append_kernel<true, false, true> : append_kernel<true, false, false>))
                                                         : (e ? (a.wide ? append_kernel<false, true, true> : append_kernel<false, true, false>) : (a.wide ? append_kernel<false, false, true> : append_kernel<false, false, false>));
    void (*const k)(const AppendArgs) = kernel;
    return launch_after(k, grid, dim3(THREADS), 0, stream, dim3(1, 1), a);
}

}  // namespace strassen
