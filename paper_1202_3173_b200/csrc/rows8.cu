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

#include <atomic>

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

// The 32 bits that start `bytes` (0..3 of them into w[0]) into two words.
__device__ __forceinline__ uint32_t bytes_from(uint32_t w0, uint32_t w1, uint32_t bytes) { return __funnelshift_r(w0, w1, 8 * bytes); }

// The same way out.  W neighbouring lanes have neighbouring pieces of a row, the first of them the first; all of them come here, with
// k >= size where there is none.
template <class T, int W> __device__ __forceinline__ void store(const Words<T> &p, T *row, int64_t k, int64_t size)
{
    constexpr int N = Words<T>::N;
    const int lane = threadIdx.x & (W - 1);
    const uintptr_t at = reinterpret_cast<uintptr_t>(row + k), off = at & 15;        // off: the same in all lanes
    const bool full = k + 8 <= size;
    bool whole = !full;                                                             // to be written element by element
    if (off == 0) {
        if (full) {
#pragma unroll
            for (int i = 0; i < N / 4; ++i) reinterpret_cast<uint4 *>(at)[i] = make_uint4(p.w[4 * i], p.w[4 * i + 1], p.w[4 * i + 2], p.w[4 * i + 3]);
        }
    } else {
        // aligned words that end within this piece: the last `off` bytes of the lane below's, then this lane's own
        uint32_t b[N + 4];
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = __shfl_up_sync(~0u, p.w[N - 4 + i], 1, W);
#pragma unroll
        for (int i = 0; i < N; ++i) b[i + 4] = p.w[i];
        const bool above = __shfl_down_sync(~0u, int(full), 1, W) && lane < W - 1;   // the lane above writes this one's last bytes
        const uint32_t up = 16 - uint32_t(off);                                     // how far the piece moves up from an aligned place
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
        for (int i = 0; i < N; ++i) out[i] = bytes_from(b[i], b[i + 1], up & 3);
        if (full && lane > 0) {
#pragma unroll
            for (int i = 0; i < N / 4; ++i) reinterpret_cast<uint4 *>(at - off)[i] = make_uint4(out[4 * i], out[4 * i + 1], out[4 * i + 2], out[4 * i + 3]);
        } else if (full) {
            // the first lane: all of its aligned words but the one that begins before the piece, of which it has the upper part
#pragma unroll
            for (int i = 1; i < N / 4; ++i) reinterpret_cast<uint4 *>(at - off)[i] = make_uint4(out[4 * i], out[4 * i + 1], out[4 * i + 2], out[4 * i + 3]);
            uint16_t *const o = reinterpret_cast<uint16_t *>(at - off);
            if (sizeof(T) == 2 && (off & 2)) o[off / 2] = uint16_t(p.w[0]);
            const uint32_t two = uint32_t(off + 2) & ~3u;                            // first word of the upper part
            if (two & 4) reinterpret_cast<uint32_t *>(o)[two / 4] = two == 4 ? out[1] : out[3];
            if (off <= 8) *reinterpret_cast<uint2 *>(o + 4) = make_uint2(out[2], out[3]);
        }
        if (full && !above) {
            // the lane above writes nothing: this one's last `off` bytes begin an aligned word
            uint32_t t[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) t[i] = p.w[N - 4 + i];
            uint32_t c[5] = {t[0], t[1], t[2], t[3], 0};
            if (up & 8) {
#pragma unroll
                for (int i = 0; i < 3; ++i) c[i] = c[i + 2];
            }
            if (up & 4) {
#pragma unroll
                for (int i = 0; i < 4; ++i) c[i] = c[i + 1];
            }
            uint32_t *const o = reinterpret_cast<uint32_t *>(at - off + 4 * N);
            const uint32_t c0 = bytes_from(c[0], c[1], up & 3), c1 = bytes_from(c[1], c[2], up & 3), c2 = bytes_from(c[2], c[3], up & 3), c3 = bytes_from(c[3], 0, up & 3);
            if (off >= 8) *reinterpret_cast<uint2 *>(o) = make_uint2(c0, c1);
            if (off & 4) o[off & 8 ? 2 : 0] = off & 8 ? c2 : c0;
            if (sizeof(T) == 2 && (off & 2)) {
                const int w = int(off) / 4;
                reinterpret_cast<uint16_t *>(o)[2 * w] = uint16_t(w == 0 ? c0 : w == 1 ? c1 : w == 2 ? c2 : c3);
            }
        }
    }
    if (whole && k < size) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < size) {
                if (sizeof(T) == 4) reinterpret_cast<uint32_t *>(row)[k + i] = p.w[i * N / 8];
                else reinterpret_cast<uint16_t *>(row)[k + i] = uint16_t(p.w[i / 2 * (N / 4)] >> (16 * (i & 1)));
            }
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
            store<T, 32>(ps, static_cast<T *>(p.sum) + r * p.lds, c, p.k);
        }
        float f[8], v[8];
        if (MODE != GATE) unpack(pw[i], f);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = kept[i][j] * (MODE == GATE ? factor : f[j] * factor);
        if (c < p.k) store_e4m3(p.q + r * p.ldq, c, p.k, v);
    }
    if (threadIdx.x == 0) p.scale[r] = scale;
}

// Many rows: CTAs that stay and take every gridDim.x-th row, the thread that is through first keeping the copies of the rows to come under way
// (cp.async.bulk into a ring of shared memory), so that reading never pauses for the reduction, the arithmetic or the writes of a row.
// A row goes from shared memory to registers at once and its place is free for the next.  A copy takes the 16-byte words that the row lies in;
// the first and last row of a matrix, where those may reach past it, are read by the threads themselves.
constexpr int MOST_SLOTS = 4;
constexpr int64_t kWaitLimit = int64_t(1) << 31;             // clocks of a wait, about a second
__device__ int g_gave_up;                                    // a copy that did not come: read and cleared by strassen_device_status

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ bool wait_for(uint64_t *b, uint32_t parity)
{
    for (const int64_t start = clock64(); clock64() - start < kWaitLimit;) {
        uint32_t ok;
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(smem_addr(b)), "r"(parity) : "memory");
        if (ok) return true;
    }
    g_gave_up = 1;
    return false;
}

// The 16-byte words that a row lies in, and whether they are all memory of the matrix.
template <class T> struct Window {
    uintptr_t from;
    uint32_t bytes, off;
    bool inside;
    __device__ __forceinline__ Window(const T *row, int64_t k, const Range<T> &range)
    {
        const uintptr_t at = reinterpret_cast<uintptr_t>(row), end = (at + uintptr_t(k) * sizeof(T) + 15) & ~uintptr_t(15);
        off = uint32_t(at & 15);
        from = at - off;
        bytes = uint32_t(end - from);
        inside = from >= range.lo && end <= range.hi;
    }
};

template <class T, int MODE, int ITEMS, int THREADS> __global__ void __launch_bounds__(THREADS, 1024 / THREADS) stream_kernel(const RowArgs p, int slots, int slot_bytes)
{
    extern __shared__ __align__(16) uint8_t memory[];            // the weights of a norm, then the ring
    uint8_t *const ring = memory + (MODE == GATE ? 0 : int(blockDim.x) * ITEMS * 8 * int(sizeof(T)));
    __shared__ float part[2][32];
    __shared__ uint64_t full[MOST_SLOTS];
    if (threadIdx.x == 0) {
        for (int i = 0; i < slots; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_addr(&full[i])));
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    after_work_before();
    __syncthreads();
    const int k = int(p.k);
    const Range<T> range_a(p.a, p.m, p.k, p.lda), range_b(p.b, p.m, p.k, p.ldb), range_w(p.weight, 1, p.k, p.k);
    const auto row_a = [&](int64_t r) { return static_cast<const T *>(p.a) + r * p.lda; };
    const auto row_b = [&](int64_t r) { return static_cast<const T *>(p.b) + r * p.ldb; };
    const auto copied = [&](int64_t r) { return Window<T>(row_a(r), k, range_a).inside && (MODE == NORM || Window<T>(row_b(r), k, range_b).inside); };
    const int half = MODE == NORM ? slot_bytes : slot_bytes / 2;
    const auto fetch = [&](int64_t r, int slot) {                // by thread 0
        if (r >= p.m || !copied(r)) return;
        const Window<T> a(row_a(r), k, range_a);
        const uint32_t bar = smem_addr(&full[slot]), to = smem_addr(ring + slot * slot_bytes);
        uint32_t bytes = a.bytes;
        if (MODE != NORM) bytes += Window<T>(row_b(r), k, range_b).bytes;
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(a.from), "r"(a.bytes), "r"(bar) : "memory");
        if (MODE != NORM) {
            const Window<T> b(row_b(r), k, range_b);
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to + half), "l"(b.from), "r"(b.bytes), "r"(bar) : "memory");
        }
    };
    if (threadIdx.x == 0)
        for (int i = 0; i < slots; ++i) fetch(blockIdx.x + int64_t(i) * gridDim.x, i);
    // weights: each thread's own pieces, 16 bytes of all threads side by side
    constexpr int N16 = Words<T>::N / 4;
    uint4 *const weights = reinterpret_cast<uint4 *>(memory);
    const auto weight = [&](int i, float (&f)[8]) {
        Words<T> w;
#pragma unroll
        for (int j = 0; j < N16; ++j) {
            const uint4 u = weights[(i * N16 + j) * int(blockDim.x) + int(threadIdx.x)];
            w.w[4 * j] = u.x;
            w.w[4 * j + 1] = u.y;
            w.w[4 * j + 2] = u.z;
            w.w[4 * j + 3] = u.w;
        }
        unpack(w, f);
    };
    if (MODE != GATE) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = (i * int(blockDim.x) + int(threadIdx.x)) * 8;
            Words<T> w;
            memset(&w, 0, sizeof(w));
            if (c < k) load(w, static_cast<const T *>(p.weight), c, k, range_w.lo, range_w.hi);
#pragma unroll
            for (int j = 0; j < N16; ++j) weights[(i * N16 + j) * int(blockDim.x) + int(threadIdx.x)] = make_uint4(w.w[4 * j], w.w[4 * j + 1], w.w[4 * j + 2], w.w[4 * j + 3]);
        }
    }
    int slot = 0;
    uint32_t phases = 0;                                         // of each slot's barrier
    bool alive = true;
    for (int64_t r = blockIdx.x; r < p.m && alive; r += gridDim.x) {
        Words<T> pa[ITEMS], pb[ITEMS];
        const T *a = row_a(r), *b = row_b(r);
        uintptr_t lo_a = range_a.lo, hi_a = range_a.hi, lo_b = range_b.lo, hi_b = range_b.hi;
        if (copied(r)) {
            alive = wait_for(&full[slot], phases >> slot & 1);
            phases ^= 1u << slot;
            // the row's place in the ring, in which wider accesses stay inside what was copied and its margin
            uint8_t *const at = ring + slot * slot_bytes;
            a = reinterpret_cast<const T *>(at + (reinterpret_cast<uintptr_t>(a) & 15));
            lo_a = reinterpret_cast<uintptr_t>(at);
            hi_a = lo_a + half;
            b = reinterpret_cast<const T *>(at + half + (reinterpret_cast<uintptr_t>(b) & 15));
            lo_b = lo_a + half;
            hi_b = lo_b + half;
        }
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = (i * int(blockDim.x) + int(threadIdx.x)) * 8;
            if (c < k) {
                load(pa[i], a, c, k, lo_a, hi_a);
                if (MODE != NORM) load(pb[i], b, c, k, lo_b, hi_b);
            } else {
                memset(&pa[i], 0, sizeof(pa[i]));
                memset(&pb[i], 0, sizeof(pb[i]));
            }
        }
        alive = __syncthreads_and(alive);
        if (!alive) break;
        if (threadIdx.x == 0) fetch(r + int64_t(slots) * gridDim.x, slot);
        slot = slot + 1 == slots ? 0 : slot + 1;
        float kept[ITEMS][8];
        float sq = 0.f, mx = 0.f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            float y[8], f[8], v[8];
            unpack(pa[i], kept[i]);
            if (MODE != NORM) unpack(pb[i], y);
            if (MODE != GATE) weight(i, f);
            values<MODE>(kept[i], y, f, v, sq, mx);
            if (MODE == GATE) memcpy(kept[i], v, sizeof(v));
        }
        reduce_row(sq, mx, part);
        float scale;
        const float factor = row_factor<MODE>(sq, mx, p.k, p.eps, scale);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = (i * int(blockDim.x) + int(threadIdx.x)) * 8;
            if (MODE == NORM_RESIDUAL) {
                Words<T> ps;
                pack(ps, kept[i]);
                store<T, 32>(ps, static_cast<T *>(p.sum) + r * p.lds, c, k);
            }
            float f[8], v[8];
            if (MODE != GATE) weight(i, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = kept[i][j] * (MODE == GATE ? factor : f[j] * factor);
            if (c < k) store_e4m3(p.q + r * p.ldq, c, k, v);
        }
        if (threadIdx.x == 0) p.scale[r] = scale;
    }
    // given up: the copies that are under way end before the CTA does
    if (!alive)
        for (int i = 0; i < 10000; ++i) __nanosleep(100);
}

template <class T, int MODE, int ITEMS, int THREADS> cudaError_t launch_stream(const RowArgs &p, int sm_count, cudaStream_t stream)
{
    static std::atomic<uint64_t> opted_in{0};                // devices that this kernel has been given its shared memory on
    constexpr int most = 216 * 1024 / (1024 / THREADS);      // of an SM's 227 KB, with as many CTAs as its registers hold
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (!(opted_in.load(std::memory_order_relaxed) >> dev & 1)) {
        e = cudaFuncSetAttribute(stream_kernel<T, MODE, ITEMS, THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
        if (e != cudaSuccess) return e;
        opted_in.fetch_or(uint64_t(1) << dev, std::memory_order_relaxed);
    }
    const int threads = int((p.k + 256 * ITEMS - 1) / (256 * ITEMS) * 32), weights = MODE == GATE ? 0 : threads * ITEMS * 8 * int(sizeof(T));
    const int half = int((p.k * int64_t(sizeof(T)) + 15) / 16 * 16 + 48);        // the words it lies in, and what a piece's window may read beyond
    const int slot_bytes = MODE == NORM ? half : 2 * half;
    int slots = (most - weights) / slot_bytes;
    if (slots > MOST_SLOTS) slots = MOST_SLOTS;
    const int ctas = 1024 / THREADS * sm_count;
    return launch_after(stream_kernel<T, MODE, ITEMS, THREADS>, dim3(unsigned(p.m < ctas ? p.m : ctas)), dim3(unsigned(threads)), size_t(weights + slots * slot_bytes), stream, dim3(1, 1), p, slots, slot_bytes);
}

// Short rows: W lanes of a warp for each, which nothing has to meet with, ITEMS pieces a lane.
template <class T, int MODE, int W, int ITEMS> __global__ void __launch_bounds__(256) short_row_kernel(const RowArgs p)
{
    after_work_before();
    const int lane = threadIdx.x & (W - 1);
    const int64_t at = (int64_t(blockIdx.x) * 256 + threadIdx.x) / W;
    const bool on = at < p.m;
    const int64_t r = on ? at : p.m - 1, size = on ? p.k : 0;         // lanes without a row read and write nothing, but take part in the shuffles
    const T *const a = static_cast<const T *>(p.a) + r * p.lda, *const b = static_cast<const T *>(p.b) + r * p.ldb, *const w = static_cast<const T *>(p.weight);
    const Range<T> range_a(p.a, p.m, p.k, p.lda), range_b(p.b, p.m, p.k, p.ldb), range_w(p.weight, 1, p.k, p.k);
    Words<T> pa[ITEMS], pb[ITEMS], pw[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int64_t c = (i * W + lane) * 8;
        if (c < size) {
            load(pa[i], a, c, size, range_a.lo, range_a.hi);
            if (MODE != NORM) load(pb[i], b, c, size, range_b.lo, range_b.hi);
            if (MODE != GATE) load(pw[i], w, c, size, range_w.lo, range_w.hi);
        } else {
#pragma unroll
            for (int j = 0; j < Words<T>::N; ++j) pa[i].w[j] = pb[i].w[j] = pw[i].w[j] = 0;
        }
    }
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
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) {
        sq += __shfl_xor_sync(~0u, sq, o);
        mx = max_nan(mx, __shfl_xor_sync(~0u, mx, o));
    }
    float scale;
    const float factor = row_factor<MODE>(sq, mx, p.k, p.eps, scale);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int64_t c = (i * W + lane) * 8;
        if (MODE == NORM_RESIDUAL) {
            Words<T> ps;
            pack(ps, kept[i]);
            store<T, W>(ps, static_cast<T *>(p.sum) + r * p.lds, c, size);
        }
        float f[8], v[8];
        if (MODE != GATE) unpack(pw[i], f);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = kept[i][j] * (MODE == GATE ? factor : f[j] * factor);
        if (c < size) store_e4m3(p.q + r * p.ldq, c, size, v);
    }
    if (lane == 0 && on) p.scale[r] = scale;
}

template <class T, int MODE, int W, int ITEMS> cudaError_t launch_short(const RowArgs &p, cudaStream_t stream)
{
    return launch_after(short_row_kernel<T, MODE, W, ITEMS>, dim3(unsigned((p.m + 256 / W - 1) / (256 / W))), dim3(256), 0, stream, dim3(1, 1), p);
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
                store<T, 32>(t, static_cast<T *>(p.sum) + r * p.lds, c, p.k);
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

template <class T, int MODE> cudaError_t launch_type(const RowArgs &p, int sm_count, cudaStream_t stream)
{
    const int64_t pieces = (p.k + 7) / 8;
    // Short rows, where there are enough of them for the lanes to be all in use; a CTA for each row would spend its time on its launch and its
    // reduction (128 bf16 values: 310 us for 300000 rows).
    if (pieces <= 128 && p.m >= 2 * sm_count) {
        if (pieces <= 8) return launch_short<T, MODE, 8, 1>(p, stream);
        if (pieces <= 16) return launch_short<T, MODE, 16, 1>(p, stream);
        if (pieces <= 32) return launch_short<T, MODE, 32, 1>(p, stream);
        if (pieces <= 64) return launch_short<T, MODE, 32, 2>(p, stream);
        return launch_short<T, MODE, 32, 4>(p, stream);
    }
    // Rows enough for CTAs that stay.  Two pieces a thread, so that an SM has several rows at a time in different steps, four where a row would
    // need more than half of its threads.
    if (p.m >= 4 * sm_count && pieces > 128 && pieces <= 2048 && p.k * int64_t(sizeof(T)) <= 32 * 1024) {
        if (pieces <= 512) return launch_stream<T, MODE, 2, 256>(p, sm_count, stream);
        if (pieces <= 1024) return launch_stream<T, MODE, 2, 512>(p, sm_count, stream);
        return launch_stream<T, MODE, 4, 512>(p, sm_count, stream);
    }
    const dim3 grid(unsigned(p.m));
    const auto threads = [&](int items) { return dim3(unsigned((pieces + 32 * items - 1) / (32 * items) * 32)); };
    // two pieces a thread for rows that then still make a CTA of 128 threads or more: more of the row under way for each of its registers
    if (pieces <= 256) return launch_after(row_kernel<T, MODE, 1, 256>, grid, threads(1), 0, stream, dim3(1, 1), p);
    if (pieces <= 1024) return launch_after(row_kernel<T, MODE, 2, 512>, grid, threads(2), 0, stream, dim3(1, 1), p);
    if (pieces <= 2048) return launch_after(row_kernel<T, MODE, 2, 1024>, grid, threads(2), 0, stream, dim3(1, 1), p);
    return launch_after(long_row_kernel<T, MODE>, grid, dim3(1024), 0, stream, dim3(1, 1), p);
}

template <int MODE> cudaError_t launch_mode(const RowArgs &p, int sm_count, cudaStream_t stream)
{
    if (p.m == 0) return cudaSuccess;
    switch (p.type) {
    case STRASSEN_BF16: return launch_type<__nv_bfloat16, MODE>(p, sm_count, stream);
    case STRASSEN_F16: return launch_type<__half, MODE>(p, sm_count, stream);
    case STRASSEN_F32: return launch_type<float, MODE>(p, sm_count, stream);
    }
    return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_rms_norm_quant(const RowArgs &p, int sm_count, cudaStream_t stream)
{
    return p.b ? launch_mode<NORM_RESIDUAL>(p, sm_count, stream) : launch_mode<NORM>(p, sm_count, stream);
}

cudaError_t launch_silu_mul_quant(const RowArgs &p, int sm_count, cudaStream_t stream) { return launch_mode<GATE>(p, sm_count, stream); }

cudaError_t rows8_gave_up(int *flag)
{
    cudaError_t e = cudaMemcpyFromSymbol(flag, g_gave_up, sizeof(int));
    if (e != cudaSuccess || !*flag) return e;
    const int zero = 0;
    return cudaMemcpyToSymbol(g_gave_up, &zero, sizeof(int));
}

}  // namespace strassen
