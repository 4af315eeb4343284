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
// row's scale and outputs NaN (the maximum propagates NaN), as the formulas say; so does a row whose squares do not fit 32 bits.
//
// A thread has pieces of 8 neighbouring elements.  Rows that do not start at a multiple of 16 bytes (odd lengths, halves of odd rows) are read and
// written in the same 16-byte accesses: two aligned words around a piece are shifted into place, and on the way out neighbouring lanes pass
// each other the bytes that belong to the other's word.  Many rows come near HBM: 9600 x 8192 bf16, inputs changing, norm with residual 89 us (6.2 TB/s), without 50 us
// (4.7 TB/s), gate 58 us (6.7 TB/s, four bytes read for each one written; a copy, which writes as many as it reads, has 6.5).  Misaligned rows pay for shifting and
// staging (4099 x 12345 f16: 80 us, 4.4 TB/s), few rows for launch and latency.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <atomic>

#include "llm.h"
#include "pieces.cuh"
#include "strassen_b200.h"

namespace strassen {

namespace {

__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

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

// The 32 bits that start `bytes` (0..3 of them into w[0]) into two words.
__device__ __forceinline__ uint32_t bytes_from(uint32_t w0, uint32_t w1, uint32_t bytes) { return __funnelshift_r(w0, w1, 8 * bytes); }

// The same way out.  W neighbouring lanes have neighbouring pieces of a row, the first of them the first; all of them come here, with
// k >= size where there is none.
template <class T, int W> __device__ __forceinline__ void store(const Words<T> &p, T *row, int64_t k, int64_t size)
{
    constexpr int N = Words<T>::N;
    const int lane = threadIdx.x & (W - 1);
    const uint32_t row_lanes = W == 32 ? ~0u : ((1u << (W & 31)) - 1) << (threadIdx.x & 31 & ~(W - 1));     // other rows of the warp may take another way
    const uintptr_t at = reinterpret_cast<uintptr_t>(row + k), off = at & 15;        // off: the same in all lanes of the row
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
        for (int i = 0; i < 4; ++i) b[i] = __shfl_up_sync(row_lanes, p.w[N - 4 + i], 1, W);
#pragma unroll
        for (int i = 0; i < N; ++i) b[i + 4] = p.w[i];
        const bool above = lane < W - 1 && k + 16 <= size;                          // the lane above writes this one's last bytes
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

enum { GATE = 0, NORM = 1, NORM_RESIDUAL = 2 };

// Sum (of a norm) and maximum over a warp.  The maximum is of absolute values, so its bits have the order of unsigned numbers, NaN (0x7fffffff) above
// infinity: one reduction instruction.
template <int MODE> __device__ __forceinline__ void reduce_warp(float &sum, float &mx)
{
    if (MODE != GATE) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    }
    mx = __uint_as_float(__reduce_max_sync(~0u, __float_as_uint(mx)));
}
// ... of the warps' values in `part` (sum, maximum), the same bits in every thread: each adds them in the same order.
template <int MODE> __device__ __forceinline__ void reduce_warps(float &sum, float &mx, const float2 *part, int warps)
{
    const int lane = threadIdx.x & 31;
    const float2 v = lane < warps ? part[lane] : make_float2(0.f, 0.f);
    sum = v.x;
    mx = v.y;
    reduce_warp<MODE>(sum, mx);
}
// ... over the CTA.
template <int MODE> __device__ __forceinline__ void reduce_row(float &sum, float &mx, float2 *part)
{
    reduce_warp<MODE>(sum, mx);
    const int warps = blockDim.x >> 5;
    if (warps == 1) return;
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = make_float2(sum, mx);
    __syncthreads();
    reduce_warps<MODE>(sum, mx, part, warps);
}

// Two f32 in a register pair: Blackwell adds and multiplies them in one instruction.
struct Pair {
    uint64_t v;
    __device__ __forceinline__ Pair() {}
    __device__ __forceinline__ Pair(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ void get(float &a, float &b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
};
__device__ __forceinline__ Pair operator+(Pair a, Pair b)
{
    Pair d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
    return d;
}
__device__ __forceinline__ Pair operator*(Pair a, Pair b)
{
    Pair d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
    return d;
}
__device__ __forceinline__ Pair fma(Pair a, Pair b, Pair c)
{
    Pair d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return d;
}
__device__ __forceinline__ float max_abs(float m, Pair v)
{
    float a, b, d;
    v.get(a, b);
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(m), "f"(a), "f"(b));
    return d;
}

// A piece's values before the row's factor, v = h w for the norm, silu(g) u for the gate; what they add to the row's sum of squares and maximum; and
// for a norm with a residual h itself, in its type.  exp and the reciprocal are the approximate instructions: some 2^-21 of a value for gates of a few units,
// and, since g log2(e) is rounded once, 2^-24 |g| for large negative ones (2^-17 at -80, where silu is below 2^-109); beyond -87 the reciprocal is flushed to 0.
// All of it is far below the 2^-4 of the rounding to e4m3.
template <class T, int MODE> __device__ __forceinline__ void values(const Words<T> &pa, const Words<T> &pb, const Words<T> &pw, Pair (&v)[4], Words<T> &sum, Pair &sq, float &mx)
{
    float x[8], y[8], w[8];
    unpack(pa, x);
    if (MODE != NORM) unpack(pb, y);
    if (MODE != GATE) unpack(pw, w);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        Pair h(x[2 * i], x[2 * i + 1]);
        if (MODE == GATE) {
            // one by one: the two special-function instructions of each decide, and pairs would have to be taken apart for them
            float t[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float e, over;
                asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x[2 * i + j] * -1.4426950408889634f));
                asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(over) : "f"(1.f + e));
                t[j] = x[2 * i + j] * over * y[2 * i + j];
            }
            v[i] = Pair(t[0], t[1]);
        } else {
            if (MODE == NORM_RESIDUAL) {
                h = h + Pair(y[2 * i], y[2 * i + 1]);
                h.get(x[2 * i], x[2 * i + 1]);
            }
            sq = fma(h, h, sq);
            v[i] = h * Pair(w[2 * i], w[2 * i + 1]);
        }
        mx = max_abs(mx, v[i]);
    }
    if (MODE == NORM_RESIDUAL) pack(sum, x);
}
__device__ __forceinline__ float both(Pair v)
{
    float a, b;
    v.get(a, b);
    return a + b;
}

// The row's scale, and the factor that takes a value before the row's factor to the e4m3 range.  The quotients of two values and the root are the
// approximate instructions here too, within two units of the last place.
template <int MODE> __device__ __forceinline__ float row_factor(float sq, float mx, float over_k, float eps, float &scale)
{
    // squares that pass the range of 32 bits make NaN of their row; the root's reciprocal, 0, would make zeros
    const float inv = MODE == GATE ? 1.f : sq < INFINITY ? rsqrtf(sq * over_k + eps) : NAN;
    const float s = mx * inv * (1.f / kE4M3Max);
    scale = s <= kMinRowScale ? kMinRowScale : s;        // NaN stays NaN
    return __fdividef(inv, scale);
}

// v factor as e4m3; `wide`: rows of q start at multiples of 8 bytes.
__device__ __forceinline__ void store_e4m3(uint8_t *row, int64_t k, int64_t size, const Pair (&v)[4], float factor, bool wide)
{
    uint32_t w[2];
    const Pair f(factor, factor);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float a, b, c, d;
        (v[2 * i] * f).get(a, b);
        (v[2 * i + 1] * f).get(c, d);
        uint16_t lo, hi;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
        asm("mov.b32 %0, {%1, %2};" : "=r"(w[i]) : "h"(lo), "h"(hi));
    }
    if (wide && k + 8 <= size) {
        *reinterpret_cast<uint2 *>(row + k) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < size) row[k + i] = uint8_t(w[i / 4] >> (8 * (i & 3)));
    }
}

// One CTA per row, the row in registers: ITEMS pieces a thread, their loads all under way before the first is used.
template <class T, int MODE, int ITEMS, int THREADS> __global__ void __launch_bounds__(THREADS) row_kernel(const RowArgs p)
{
    __shared__ float2 part[32];
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
    // v is kept until the row's factor is known; the sum goes out at once: what a thread, or the lane beside it, writes over has been read
    Pair v[ITEMS][4], squares(0.f, 0.f);
    float mx = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        Words<T> sum;
        values<T, MODE>(pa[i], pb[i], pw[i], v[i], sum, squares, mx);
        if (MODE == NORM_RESIDUAL) store<T, 32>(sum, static_cast<T *>(p.sum) + r * p.lds, (i * int64_t(blockDim.x) + threadIdx.x) * 8, p.k);
    }
    float sq = both(squares);
    reduce_row<MODE>(sq, mx, part);
    float scale;
    const float factor = row_factor<MODE>(sq, mx, 1.f / float(p.k), p.eps, scale);
    uint8_t *const q = p.q + r * p.ldq;
    const bool wide = reinterpret_cast<uintptr_t>(q) % 8 == 0;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int64_t c = (i * int64_t(blockDim.x) + threadIdx.x) * 8;
        if (c < p.k) store_e4m3(q, c, p.k, v[i], factor, wide);
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

// 8 elements at `at` in shared memory, `off` bytes past a multiple of 16 (the same for all pieces of a row); what lies around them may be read.
template <class T> __device__ __forceinline__ void load_shared(Words<T> &p, const uint8_t *at, uint32_t off)
{
    constexpr int N = Words<T>::N;
    if (off == 0) {
        load_words<N>(p.w, at);
    } else {
        uint32_t a[N + 4];
        load_words<N + 4>(a, at - off);
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
    }
}
// Zeros in the place of the elements from `count` on.
template <class T> __device__ __forceinline__ void cut(Words<T> &p, int count)
{
    constexpr int N = Words<T>::N, PER = 8 / N;              // elements of a word
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i * PER >= count) p.w[i] = 0;
        else if (PER == 2 && i * PER + 1 == count) p.w[i] &= 0xffffu;
    }
}

template <class T, int MODE, int ITEMS, int THREADS> __global__ void __launch_bounds__(THREADS, 1024 / THREADS) stream_kernel(const RowArgs p, int slots, int slot_bytes, int stage_at)
{
    static_assert(MODE != GATE, "norms only");
    extern __shared__ __align__(16) uint8_t memory[];            // the norm's weights, then the ring
    constexpr bool TWO = MODE == NORM_RESIDUAL;                  // two inputs
    uint8_t *const ring = memory + int(blockDim.x) * ITEMS * 8 * int(sizeof(T));
    __shared__ float2 part[2][THREADS / 32];
    __shared__ uint64_t full[MOST_SLOTS];
    __shared__ int dead[2];              // a wait gave up; of even and odd turns, so that none is set while it is still being read for the turn before
    if (threadIdx.x == 0) {
        for (int i = 0; i < slots; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_addr(&full[i])));
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        dead[0] = dead[1] = 0;
    }
    after_work_before();
    __syncthreads();
    const int k = int(p.k), rows = int(p.m), step = int(gridDim.x);
    const uint32_t row_bytes = uint32_t(k) * uint32_t(sizeof(T));
    const uintptr_t base_a = reinterpret_cast<uintptr_t>(p.a), base_b = reinterpret_cast<uintptr_t>(p.b);
    const uintptr_t ld_a = uintptr_t(p.lda) * sizeof(T), ld_b = uintptr_t(p.ldb) * sizeof(T);
    const int half = TWO ? slot_bytes / 2 : slot_bytes;
    // the 16-byte words of a row: those of the first row may begin before the matrix, those of the last end after it
    const auto copied = [&](int r) {
        bool in = r > 0 || (((base_a | (TWO ? base_b : 0)) & 15) == 0);
        if (r == rows - 1) in = in && ((base_a + r * ld_a + row_bytes) & 15) == 0 && (!TWO || ((base_b + r * ld_b + row_bytes) & 15) == 0);
        return in;
    };
    const auto fetch = [&](int r, int slot) {                    // by one thread
        if (r >= rows || !copied(r)) return;
        const uint32_t bar = smem_addr(&full[slot]), to = smem_addr(ring + slot * slot_bytes);
        const uintptr_t a = base_a + r * ld_a, b = base_b + r * ld_b;
        const uint32_t bytes_a = (uint32_t(a & 15) + row_bytes + 15) & ~15u, bytes_b = TWO ? (uint32_t(b & 15) + row_bytes + 15) & ~15u : 0;
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes_a + bytes_b) : "memory");
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(a & ~uintptr_t(15)), "r"(bytes_a), "r"(bar) : "memory");
        if (TWO)
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to + half), "l"(b & ~uintptr_t(15)), "r"(bytes_b), "r"(bar) : "memory");
    };
    if (threadIdx.x == 0)
        for (int i = 0; i < slots; ++i) fetch(int(blockIdx.x) + i * step, i);
    // weights: each thread's own pieces, 16 bytes of all threads side by side
    constexpr int N16 = Words<T>::N / 4;
    uint4 *const weights = reinterpret_cast<uint4 *>(memory) + threadIdx.x;
    const auto weight = [&](int i, Words<T> &w) {
#pragma unroll
        for (int j = 0; j < N16; ++j) {
            const uint4 u = weights[(i * N16 + j) * int(blockDim.x)];
            w.w[4 * j] = u.x;
            w.w[4 * j + 1] = u.y;
            w.w[4 * j + 2] = u.z;
            w.w[4 * j + 3] = u.w;
        }
    };
    const Range<T> range_w(p.weight, 1, p.k, p.k);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int c = (i * int(blockDim.x) + int(threadIdx.x)) * 8;
        Words<T> w;
        memset(&w, 0, sizeof(w));
        if (c < k) load(w, static_cast<const T *>(p.weight), c, k, range_w.lo, range_w.hi);
#pragma unroll
        for (int j = 0; j < N16; ++j) weights[(i * N16 + j) * int(blockDim.x)] = make_uint4(w.w[4 * j], w.w[4 * j + 1], w.w[4 * j + 2], w.w[4 * j + 3]);
    }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const float over_k = 1.f / float(k);
    int slot = 0, turn = 0;
    uint32_t phases = 0;                                         // of each slot's barrier
    for (int r = blockIdx.x; r < rows; r += step) {
        Words<T> pa[ITEMS], pb[ITEMS];
        if (copied(r)) {
            if (!wait_for(&full[slot], phases >> slot & 1)) dead[turn] = 1;
            phases ^= 1u << slot;
            const uint32_t off_a = uint32_t(base_a + r * ld_a) & 15, off_b = uint32_t(base_b + r * ld_b) & 15;
            const uint8_t *const at = ring + slot * slot_bytes;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const int c = (i * int(blockDim.x) + int(threadIdx.x)) * 8;
                if (c < k) {
                    load_shared(pa[i], at + off_a + c * int(sizeof(T)), off_a);
                    if (TWO) load_shared(pb[i], at + half + off_b + c * int(sizeof(T)), off_b);
                    if (c + 8 > k) {
                        cut(pa[i], k - c);
                        if (TWO) cut(pb[i], k - c);
                    }
                } else {
                    memset(&pa[i], 0, sizeof(pa[i]));
                    memset(&pb[i], 0, sizeof(pb[i]));
                }
            }
        } else {
            const Range<T> range_a(p.a, p.m, p.k, p.lda), range_b(p.b, p.m, p.k, p.ldb);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const int c = (i * int(blockDim.x) + int(threadIdx.x)) * 8;
                memset(&pa[i], 0, sizeof(pa[i]));
                memset(&pb[i], 0, sizeof(pb[i]));
                if (c < k) {
                    load(pa[i], reinterpret_cast<const T *>(base_a + r * ld_a), c, k, range_a.lo, range_a.hi);
                    if (TWO) load(pb[i], reinterpret_cast<const T *>(base_b + r * ld_b), c, k, range_b.lo, range_b.hi);
                }
            }
        }
        // the sum goes out at once: its row is in shared memory, or in the registers of the threads beside it, whatever it is written over
        Pair v[ITEMS][4], squares(0.f, 0.f);
        float mx = 0.f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            Words<T> w, sum;
            weight(i, w);
            values<T, MODE>(pa[i], pb[i], w, v[i], sum, squares, mx);
            if (MODE == NORM_RESIDUAL) {
                const int c = (i * int(blockDim.x) + int(threadIdx.x)) * 8;
                if (stage_at == 0) {
                    store<T, 32>(sum, static_cast<T *>(p.sum) + r * p.lds, c, k);
                } else if (c < k) {
#pragma unroll
                    for (int j = 0; j < N16; ++j)
                        reinterpret_cast<uint4 *>(memory + stage_at + c * int(sizeof(T)))[j] = make_uint4(sum.w[4 * j], sum.w[4 * j + 1], sum.w[4 * j + 2], sum.w[4 * j + 3]);
                }
            }
        }
        float sq = both(squares);
        reduce_warp<MODE>(sq, mx);
        if (lane == 0) part[turn][warp] = make_float2(sq, mx);
        __syncthreads();
        // every thread has its part of the row: its place is free
        if (dead[turn]) break;
        if (threadIdx.x == 0) fetch(r + slots * step, slot);
        slot = slot + 1 == slots ? 0 : slot + 1;
        reduce_warps<MODE>(sq, mx, part[turn], warps);
        turn ^= 1;
        float scale;
        const float factor = row_factor<MODE>(sq, mx, over_k, p.eps, scale);
        uint8_t *const q = p.q + r * p.ldq;
        const bool wide = reinterpret_cast<uintptr_t>(q) % 8 == 0;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = (i * int(blockDim.x) + int(threadIdx.x)) * 8;
            if (c < k) store_e4m3(q, c, k, v[i], factor, wide);
        }
        if (threadIdx.x == 0) p.scale[r] = scale;
        if (MODE == NORM_RESIDUAL && stage_at) {
            // aligned words of a sum whose row is not: taken from where they lie in the staged row
            uint8_t *const row = reinterpret_cast<uint8_t *>(static_cast<T *>(p.sum) + r * p.lds);
            const uint8_t *const stage = memory + stage_at;
            const int off = int(reinterpret_cast<uintptr_t>(row) & 15), words = (off + int(row_bytes) + 15) / 16;
            for (int j = threadIdx.x; j < words; j += blockDim.x) {
                const int at = 16 * j - off;
                if (at >= 0 && at + 16 <= int(row_bytes)) {
                    Words<__half> t;
                    load_shared(t, stage + at, uint32_t(16 - off) & 15);
                    *reinterpret_cast<uint4 *>(row + at) = make_uint4(t.w[0], t.w[1], t.w[2], t.w[3]);
                } else {
                    for (int b = at < 0 ? 0 : at; b < at + 16 && b < int(row_bytes); b += 2) *reinterpret_cast<uint16_t *>(row + b) = *reinterpret_cast<const uint16_t *>(stage + b);
                }
            }
            __syncthreads();             // before the next row is staged
        }
    }
    // given up: the copies that are under way end before the CTA does
    if (dead[0] | dead[1])
        for (int i = 0; i < 10000; ++i) __nanosleep(100);
}

// cudaErrorNotSupported, with nothing launched, where not one row fits the CTA's shared memory.
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
    const int threads = int((p.k + 256 * ITEMS - 1) / (256 * ITEMS) * 32), weights = threads * ITEMS * 8 * int(sizeof(T));
    const int half = int((p.k * int64_t(sizeof(T)) + 15) / 16 * 16 + 48);        // the words it lies in, and what a piece's window may read beyond
    const int slot_bytes = MODE == NORM ? half : 2 * half;
    int slots = (most - weights) / slot_bytes;
    if (slots < 1) return cudaErrorNotSupported;
    // A sum whose rows do not start at multiples of 16 bytes goes through shared memory where a row of it fits: 4099 x 12345 f16 in 78 us, against 113 us
    // by exchanges between the lanes.
    int stage_at = 0;
    const int stage_bytes = int((p.k * int64_t(sizeof(T)) + 15) / 16 * 16 + 32);
    if (MODE == NORM_RESIDUAL && (reinterpret_cast<uintptr_t>(p.sum) | uintptr_t(p.lds * int64_t(sizeof(T)))) % 16 != 0 && weights + slot_bytes + stage_bytes <= most) {
        slots = (most - weights - stage_bytes) / slot_bytes;
        stage_at = -1;
    }
    if (slots > MOST_SLOTS) slots = MOST_SLOTS;
    if (stage_at) stage_at = weights + slots * slot_bytes;
    const int ctas = 1024 / THREADS * sm_count;
    return launch_after(stream_kernel<T, MODE, ITEMS, THREADS>, dim3(unsigned(p.m < ctas ? p.m : ctas)), dim3(unsigned(threads)), size_t(weights + slots * slot_bytes + (stage_at ? stage_bytes : 0)), stream, dim3(1, 1), p, slots, slot_bytes, stage_at);
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
    Pair v[ITEMS][4], squares(0.f, 0.f);
    float mx = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        Words<T> sum;
        values<T, MODE>(pa[i], pb[i], pw[i], v[i], sum, squares, mx);
        if (MODE == NORM_RESIDUAL) store<T, W>(sum, static_cast<T *>(p.sum) + r * p.lds, (i * W + lane) * 8, size);
    }
    float sq = both(squares);
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) {
        if (MODE != GATE) sq += __shfl_xor_sync(~0u, sq, o);
        mx = max_nan(mx, __shfl_xor_sync(~0u, mx, o));
    }
    float scale;
    const float factor = row_factor<MODE>(sq, mx, 1.f / float(p.k), p.eps, scale);
    uint8_t *const q = p.q + r * p.ldq;
    const bool wide = reinterpret_cast<uintptr_t>(q) % 8 == 0;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int64_t c = (i * W + lane) * 8;
        if (c < size) store_e4m3(q, c, size, v[i], factor, wide);
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
    __shared__ float2 part[32];
    after_work_before();
    const int64_t r = blockIdx.x;
    const T *const a = static_cast<const T *>(p.a) + r * p.lda, *const b = static_cast<const T *>(p.b) + r * p.ldb, *const w = static_cast<const T *>(p.weight);
    const Range<T> range_a(p.a, p.m, p.k, p.lda), range_b(p.b, p.m, p.k, p.ldb), range_w(p.weight, 1, p.k, p.k);
    float sq = 0.f, mx = 0.f, scale = 0.f, factor = 0.f;
    uint8_t *const q = p.q + r * p.ldq;
    const bool wide = reinterpret_cast<uintptr_t>(q) % 8 == 0;
    for (int pass = 0; pass < 2; ++pass) {
        Pair squares(0.f, 0.f);
        for (int64_t c0 = 0; c0 < p.k; c0 += int64_t(blockDim.x) * 8) {
            const int64_t c = c0 + int64_t(threadIdx.x) * 8;
            Words<T> pa, pb, pw, sum;
            memset(&pa, 0, sizeof(pa));
            memset(&pb, 0, sizeof(pb));
            memset(&pw, 0, sizeof(pw));
            if (c < p.k) {
                load(pa, a, c, p.k, range_a.lo, range_a.hi);
                if (MODE != NORM) load(pb, b, c, p.k, range_b.lo, range_b.hi);
                if (MODE != GATE) load(pw, w, c, p.k, range_w.lo, range_w.hi);
            }
            Pair v[4];
            values<T, MODE>(pa, pb, pw, v, sum, squares, mx);
            if (pass == 0) continue;
            if (MODE == NORM_RESIDUAL) store<T, 32>(sum, static_cast<T *>(p.sum) + r * p.lds, c, p.k);
            if (c < p.k) store_e4m3(q, c, p.k, v, factor, wide);
        }
        if (pass == 0) {
            sq = both(squares);
            reduce_row<MODE>(sq, mx, part);
            factor = row_factor<MODE>(sq, mx, 1.f / float(p.k), p.eps, scale);
        }
    }
    if (threadIdx.x == 0) p.scale[r] = scale;
}

template <class T, int MODE> cudaError_t launch_type(const RowArgs &p, int sm_count, cudaStream_t stream)
{
    const int64_t pieces = (p.k + 7) / 8;
    // Short rows, where there are enough of them for the lanes to be all in use; a CTA for each row would spend its time on its launch and its
    // reduction.  30000 rows of 512 bf16 values: 11.6 us, 32 with a CTA for each (gate: 13.8 and 32); 1000 rows of 256: 1.9 and 2.0.  Longer ones only without a
    // sum to write, and where they are very many: gate 30000 x 1024 25 and 33 us, but 1000 x 1024 3.7 and 2.6; with the sum 42 and 39 us.
    if (p.m >= 2 * sm_count && (pieces <= 64 || (MODE != NORM_RESIDUAL && pieces <= 128 && p.m >= 32 * sm_count))) {
        if (pieces <= 8) return launch_short<T, MODE, 8, 1>(p, stream);
        if (pieces <= 16) return launch_short<T, MODE, 16, 1>(p, stream);
        if (pieces <= 32) return launch_short<T, MODE, 32, 1>(p, stream);
        if (pieces <= 64) return launch_short<T, MODE, 32, 2>(p, stream);
        if constexpr (MODE != NORM_RESIDUAL) return launch_short<T, MODE, 32, 4>(p, stream);
    }
    // CTAs that stay, for norms with enough to do.  With a residual: half a megabyte of x an SM (1200 x 8192 bf16 16.1 us with them and 14.5 without, 9600 x 8192 90 and
    // 97, 4800 x 16384 96 and 108, 19200 x 2048 50 and 55, but f32 16384 x 2048 77 and 64), an eighth of a megabyte where the sum is misaligned and staged (8192 x 2047: 34 and 39 us, 4099 x 12345 f16 78 and 113).  Without
    // one: in 32 bits (4096 x 8192: 28 and 41) and for the longest rows (4800 x 16384 bf16: 47 and 56, but 19200 x 4096: 58 and 50).  Never for gates,
    // whose arithmetic wants more warps than that leaves (4800 x 16384 bf16: 78 and 67 us, 9600 x 8192: 85 and 59).  Two pieces a thread, so that
    // an SM has several rows at a time in different steps, four where a row would need more than half of its threads.
    if constexpr (MODE != GATE) {
        const bool staged = MODE == NORM_RESIDUAL && (reinterpret_cast<uintptr_t>(p.sum) | uintptr_t(p.lds * int64_t(sizeof(T)))) % 16 != 0;
        if (p.m * p.k * int64_t(sizeof(T)) >= int64_t(sm_count) << (staged ? 17 : 19) && pieces > 128 && pieces <= 2048) {
            cudaError_t e = cudaErrorNotSupported;
            if constexpr (MODE == NORM_RESIDUAL || sizeof(T) == 4) {
                if (pieces <= 256) {
                    if (MODE == NORM || staged || sizeof(T) == 2) e = launch_stream<T, MODE, 2, 128>(p, sm_count, stream);
                } else if (pieces <= 512) e = launch_stream<T, MODE, 2, 256>(p, sm_count, stream);
                else if (pieces <= 1024) e = launch_stream<T, MODE, 2, 512>(p, sm_count, stream);
                else e = launch_stream<T, MODE, 4, 512>(p, sm_count, stream);
            } else if (pieces > 1536) {
                e = launch_stream<T, MODE, 4, 512>(p, sm_count, stream);
            }
            if (e != cudaErrorNotSupported) return e;
        }
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
