// Rotary embedding of queries and keys, and keys and values stored into a paged cache.
//
//     (x, y) -> (x cos - y sin, x sin + y cos),   the angle of pair f at position p: p f,
// for the pairs of a row of a head, and an 8-bit row's scale from its largest value.  A CTA has up to 8 tokens, of few heads up to 64.  Their angles, the same for all heads,
// are found first: p f / 2 pi in 64 bits, of which the fraction is an angle in 32 bits with an error of 2^-24 of a turn's size wherever p is.  Then it goes through
// their rows; the first ones are on their way before offsets, lengths and angles are looked at, which take longer than a row.
//
// A lane has two chunks of 8 values of a row, both partners of its pairs, as many lanes a row as it has such pairs of chunks and as many rows a warp as that leaves
// room for: a cosine and a sine for two values, and addresses for sixteen (pairs_kernel).  Rows that do not come apart so, or are not aligned, are taken by 16
// lanes with a chunk each, partners' values from theirs (any_kernel).
//
// Bound by the bytes, read once and written once, and nearly as much by instructions: 16384 tokens of 32 + 2 x 8 heads of 128, 370 MB with an 8-bit cache, in
// 70 us, 5.3 TB/s (400 MB, 71 us, with one in bf16); with a chunk a lane 99, with a token a CTA and its angles first 139.  One sequence of 402 MB each, whose bytes take 62 us: 49152
// tokens of 16 + 2 x 8 heads of 64 70 us (106 with 8 lanes a row, half of them idle); 39320 of 80 values 79 (93); 262144 of one head over one of 128 117 (200 with 8 tokens a CTA),
// 524288 of 64 values 155 (395): there the angles and where a token goes are most of the work.  With an 8-bit cache heads of 64 and of 80 take 79 and 90 where the bytes take 54: a
// row's largest value, scale and address are as many instructions for half the bytes.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "attention.h"
#include "llm.h"

namespace strassen {

namespace {

constexpr int THREADS = 256, MOST_TOKENS = 64, ROWS = 384, MOST_PAIRS = kMostHeadSize / 2, CTAS_AN_SM = 3;

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

// (a b + c) for two numbers at once
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{\n .reg .b64 x, y, z;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mov.b64 z, {%6, %7};\n fma.rn.f32x2 z, x, y, z;\n mov.b64 {%0, %1}, z;\n}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
// v / scale in 8 bits, of two values; inv: 1 / scale, back: -scale, or 0 if that is infinite (finite values are 0 then).  v inv is not always the quotient's nearest number in
// 32 bits, and next to a border between two e4m3 values that gives the wrong one of them (for one value in 2000 of rows in bf16).  So what is left of v is found, exactly, and its own
// quotient added (Markstein, IBM J. Res. Dev. 34 (1990): the result is the rounded quotient).  Two numbers an instruction: 79.0 us where v inv alone takes 77.4 (49152 tokens of
// 16 + 2 x 8 heads of 64, 8-bit cache), a division 96.8; 16384 of 32 + 2 x 8 of 128: 70.3, 70.1 and 76.6.
__device__ __forceinline__ uint32_t two_of_8_bits(float2 v, float inv, float back)
{
    const float2 by = make_float2(inv, inv), y = make_float2(v.x * inv, v.y * inv), quotient = fma2(fma2(make_float2(back, back), y, v), by, y);
    return __nv_cvt_float2_to_fp8x2(quotient, __NV_SATFINITE, __NV_E4M3);
}

__device__ __forceinline__ float largest(float a, float b)       // NaN if one is
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
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

// 8 values in 16 bits.
template <bool WIDE> __device__ __forceinline__ uint4 load8(const uint16_t *at)
{
    if (WIDE) return *reinterpret_cast<const uint4 *>(at);
    return make_uint4(at[0] | uint32_t(at[1]) << 16, at[2] | uint32_t(at[3]) << 16, at[4] | uint32_t(at[5]) << 16, at[6] | uint32_t(at[7]) << 16);
}
template <bool BF16> __device__ __forceinline__ void floats(float (&x)[8], uint4 u)
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = two_floats<BF16>(w[i]);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}

// Where the CTA's tokens are, and their angles by pair.
struct Tokens {
    float cos[MOST_TOKENS][MOST_PAIRS], sin[MOST_TOKENS][MOST_PAIRS];
    int page[MOST_TOKENS], position[MOST_TOKENS];            // position -1: of no sequence, or before its first row
};
__device__ __forceinline__ void look(const AppendArgs &p, int64_t t0, int tokens, Tokens &sh)
{
    if (threadIdx.x < tokens) {
        const int64_t t = t0 + threadIdx.x;
        const int b = sequence_of(p.seq, t);
        int64_t position = -1;
        if (b >= 0) {
            const NewTokens n = new_tokens(p.seq, b);
            position = n.length - (n.end - t);
        }
        sh.position[threadIdx.x] = position < 0 ? -1 : int(position);
        sh.page[threadIdx.x] = position < 0 ? -1 : page_of(p.cache, p.seq, b, position);
    }
    __syncthreads();
    const int shift = 32 - __clz(max(p.rotary / 2 - 1, 0));             // pairs, rounded up to a power of two
    for (int i = threadIdx.x; i < tokens << shift; i += THREADS) {
        const int token = i >> shift, f = i & ((1 << shift) - 1);
        if (f >= p.rotary / 2) continue;
        // 1 / 2 pi
        const double turn = double(sh.position[token]) * double(p.frequencies[f]) * 0.15915494309189535;
        sincospif(float(2 * (turn - rint(turn))), &sh.sin[token][f], &sh.cos[token][f]);
    }
    __syncthreads();
}

// Row n of the CTA's: a token's queries, keys, values, then the next token's.
struct Row {
    int token, r;
    __device__ __forceinline__ void next(int n, int rows)
    {
        r += n;
        while (r >= rows) {
            r -= rows;
            ++token;
        }
    }
};
// Which of q, k and v the row is of, and its head there.
struct Which {
    bool is_q, is_v;
    int head;
    __device__ __forceinline__ Which(const AppendArgs &p, int r) : is_q(r < p.heads), is_v(r >= p.heads + p.cache.kv_heads), head(is_q ? r : is_v ? r - p.heads - p.cache.kv_heads : r - p.heads) {}
};

// `lanes` neighbouring lanes, up to 16, have a row's values v, lane `lane` of them chunks of 8 at places first[0], first[1]; chunks from head_size on are not there.
template <bool BF16, bool E4M3, bool WIDE, int CHUNKS> __device__ __forceinline__ void store(int lane, int lanes, const AppendArgs &p, const Tokens &sh, int64_t t0, int token, Which of, float (&v)[CHUNKS][8], const int (&first)[CHUNKS])
{
    const int d = p.cache.d;
    if (of.is_q) {
        uint16_t *const row = static_cast<uint16_t *>(p.out) + (t0 + token) * p.out_row + of.head * p.out_head;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            if (first[k] >= d) continue;
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = two_16_bits<BF16>(v[k][2 * i], v[k][2 * i + 1]);
            if (WIDE) {
                *reinterpret_cast<uint4 *>(row + first[k]) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) row[first[k] + i] = uint16_t(w[i / 2] >> (16 * (i & 1)));
            }
        }
        return;
    }
    const int page = sh.page[token], slot = sh.position[token] & ((1 << p.cache.page_shift) - 1);
    uint8_t *const row = (of.is_v ? p.cache.v : p.cache.k) + page * p.cache.page_stride + of.head * p.cache.head_stride + slot * p.cache.row_stride;
    if (E4M3) {
        float most = 0.f;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) most = largest(most, fabsf(v[k][i]));
        const int begin = (threadIdx.x & 31) - lane;
        const uint32_t mine = ((1u << lanes) - 1) << begin;
        // each lane's with that of the next, of the next but one, ..: all of them, however many there are, since some twice do no harm
        for (int i = 1; i < lanes; i <<= 1) most = largest(most, __shfl_sync(mine, most, begin + (lane + i < lanes ? lane + i : lane + i - lanes)));
        // a row with NaN has NaN for its scale, and throughout
        const float scale = largest(most / kE4M3Max, kMinRowScale), inv = 1.f / scale, back = scale < INFINITY ? -scale : 0.f;
        if (page < 0) return;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            if (first[k] >= d) continue;
            uint32_t w[2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                w[i] = two_of_8_bits(make_float2(v[k][4 * i], v[k][4 * i + 1]), inv, back) | two_of_8_bits(make_float2(v[k][4 * i + 2], v[k][4 * i + 3]), inv, back) << 16;
            *reinterpret_cast<uint2 *>(row + first[k]) = make_uint2(w[0], w[1]);
        }
        if (lane == 0) (of.is_v ? p.cache.v_scale : p.cache.k_scale)[((int64_t(page) * p.cache.kv_heads + of.head) << p.cache.page_shift) + slot] = scale;
    } else if (page >= 0) {
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k)
            if (first[k] < d)
                *reinterpret_cast<uint4 *>(row + 2 * first[k]) = make_uint4(two_16_bits<BF16>(v[k][0], v[k][1]), two_16_bits<BF16>(v[k][2], v[k][3]), two_16_bits<BF16>(v[k][4], v[k][5]), two_16_bits<BF16>(v[k][6], v[k][7]));
    }
}

// LANES: of a row, 0 for `given`.
template <bool BF16, bool E4M3, int LANES> __global__ void __launch_bounds__(THREADS, CTAS_AN_SM) pairs_kernel(const AppendArgs p, int per, int given)
{
    const int lanes = LANES ? LANES : given;
    constexpr int AT_ONCE = 2;                              // rows of a lane under way at once
    __shared__ Tokens sh;
    after_work_before();
    // a warp has as many rows as fit; lanes left over have none
    const int in_warp = 32 / lanes, group = (threadIdx.x & 31) / lanes, lane = (threadIdx.x & 31) - group * lanes, slots = THREADS / 32 * in_warp;
    const int d = p.cache.d, half = p.rotary / 2, rows = p.heads + 2 * p.cache.kv_heads, stride = slots * gridDim.y;
    const int64_t t0 = int64_t(blockIdx.x) * per;
    const int tokens = int(p.seq.tokens - t0 < per ? p.seq.tokens - t0 : per);
    // the lane's chunks: partners where pairs are half of the turned values apart, else neighbours
    const bool apart = !p.interleaved && 8 * lane < half;
    const int first[2] = {16 * lane >= d ? d : apart ? 8 * lane : 16 * lane, 16 * lane >= d ? d : apart ? 8 * lane + half : 16 * lane + 8};
    const bool there = 16 * lane < d && group < in_warp;
    Row at = {0, 0};
    if (group < in_warp) at.next(blockIdx.y * slots + threadIdx.x / 32 * in_warp + group, rows);
    else at.token = tokens;
    uint4 x[AT_ONCE][2];
    const auto load = [&] {
        Row w = at;
#pragma unroll
        for (int n = 0; n < AT_ONCE; ++n) {
            x[n][0] = x[n][1] = make_uint4(0, 0, 0, 0);
            if (w.token < tokens && there) {
                const Which of(p, w.r);
                const Heads &from = of.is_q ? p.q : of.is_v ? p.v : p.k;
                const uint16_t *const row = static_cast<const uint16_t *>(from.p) + (t0 + w.token) * from.row + of.head * from.head;
                x[n][0] = *reinterpret_cast<const uint4 *>(row + first[0]);
                x[n][1] = *reinterpret_cast<const uint4 *>(row + first[1]);
            }
            w.next(stride, rows);
        }
    };
    load();
    look(p, t0, tokens, sh);
    while (at.token < tokens) {
        Row w = at;
#pragma unroll
        for (int n = 0; n < AT_ONCE; ++n, w.next(stride, rows)) {
            if (w.token >= tokens) break;
            if (sh.position[w.token] < 0) continue;
            const Which of(p, w.r);
            float v[2][8];
            floats<BF16>(v[0], x[n][0]);
            floats<BF16>(v[1], x[n][1]);
            if (!of.is_v && apart) {
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    const float4 c = *reinterpret_cast<const float4 *>(&sh.cos[w.token][8 * lane + i]), s = *reinterpret_cast<const float4 *>(&sh.sin[w.token][8 * lane + i]);
                    const float cs[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float a = v[0][i + e], b = v[1][i + e];
                        v[0][i + e] = a * cs[e] - b * ss[e];
                        v[1][i + e] = a * ss[e] + b * cs[e];
                    }
                }
            } else if (!of.is_v && p.interleaved) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (first[k] >= p.rotary) continue;
                    const float4 c = *reinterpret_cast<const float4 *>(&sh.cos[w.token][first[k] / 2]), s = *reinterpret_cast<const float4 *>(&sh.sin[w.token][first[k] / 2]);
                    const float cs[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float a = v[k][2 * e], b = v[k][2 * e + 1];
                        v[k][2 * e] = a * cs[e] - b * ss[e];
                        v[k][2 * e + 1] = a * ss[e] + b * cs[e];
                    }
                }
            }
            store<BF16, E4M3, true, 2>(lane, lanes, p, sh, t0, w.token, of, v, first);
        }
        at.next(AT_ONCE * stride, rows);
        load();
    }
}

template <bool BF16, bool E4M3, bool WIDE> __global__ void __launch_bounds__(THREADS) any_kernel(const AppendArgs p, int per)
{
    constexpr int SLOTS = THREADS / 16;
    __shared__ Tokens sh;
    after_work_before();
    const int lane = threadIdx.x & 15, first[1] = {8 * lane}, d = p.cache.d, half = p.rotary / 2, rows = p.heads + 2 * p.cache.kv_heads, stride = SLOTS * gridDim.y;
    const int64_t t0 = int64_t(blockIdx.x) * per;
    const int tokens = int(p.seq.tokens - t0 < per ? p.seq.tokens - t0 : per);
    look(p, t0, tokens, sh);
    Row w = {0, 0};
    for (w.next(blockIdx.y * SLOTS + threadIdx.x / 16, rows); w.token < tokens; w.next(stride, rows)) {
        if (sh.position[w.token] < 0) continue;
        const Which of(p, w.r);
        const Heads &from = of.is_q ? p.q : of.is_v ? p.v : p.k;
        const uint16_t *const row = static_cast<const uint16_t *>(from.p) + (t0 + w.token) * from.row + of.head * from.head;
        float v[1][8];
        floats<BF16>(v[0], first[0] < d ? load8<WIDE>(row + first[0]) : make_uint4(0, 0, 0, 0));
        if (!of.is_v) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int e = first[0] + i;
                if (e >= p.rotary) continue;             // those that do not turn stay what they are, whatever they are
                const bool second = p.interleaved ? e & 1 : e >= half;
                const int f = p.interleaved ? e / 2 : second ? e - half : e;
                const float other = two_floats<BF16>(row[p.interleaved ? e ^ 1 : second ? e - half : e + half]).x, c = sh.cos[w.token][f], s = sh.sin[w.token][f];
                v[0][i] = second ? other * s + v[0][i] * c : v[0][i] * c - other * s;
            }
        }
        __syncwarp(0xffffu << (threadIdx.x & 16));           // in place: a row is read by all of its lanes before it is written
        store<BF16, E4M3, WIDE, 1>(lane, 16, p, sh, t0, w.token, of, v, first);
    }
}

template <bool BF16, bool E4M3> cudaError_t launch(const AppendArgs &a, int sm_count, cudaStream_t stream)
{
    const bool pairs = a.wide && a.cache.d % 16 == 0 && a.rotary % (a.interleaved ? 8 : 16) == 0;
    const int rows = a.heads + 2 * a.cache.kv_heads, lanes = pairs ? (a.cache.d + 15) / 16 : 16;
    // as many tokens a CTA as leave each SM its CTAs, up to 8, or of few heads 64, about ROWS rows: then a CTA has more to do than to look up where its
    // tokens are; where there are few tokens, a token's rows in several
    const int64_t tokens = a.seq.tokens / (CTAS_AN_SM * sm_count), most = rows * 8 >= ROWS ? 8 : ROWS / rows < MOST_TOKENS ? ROWS / rows : MOST_TOKENS,
                  per = tokens < 1 ? 1 : tokens < most ? tokens : most, ctas = (a.seq.tokens + per - 1) / per;
    const int slots = THREADS / 32 * (32 / lanes), steps = (rows + slots - 1) / slots;
    const dim3 grid(unsigned(ctas), unsigned(ctas >= sm_count ? 1 : steps < 16 ? steps : 16));
    // with the number of lanes known to the compiler 66 us where it is 71 (24576 tokens of 16 + 2 x 8 heads of 128, 8-bit cache), so the larger heads have it
    const auto with = [&](auto kernel) { return launch_after(kernel, grid, dim3(THREADS), 0, stream, dim3(1, 1), a, int(per), lanes); };
    if (pairs) {
        switch (lanes) {
        case 8: return with(pairs_kernel<BF16, E4M3, 8>);
        case 7: return with(pairs_kernel<BF16, E4M3, 7>);
        case 6: return with(pairs_kernel<BF16, E4M3, 6>);
        case 5: return with(pairs_kernel<BF16, E4M3, 5>);
        case 4: return with(pairs_kernel<BF16, E4M3, 4>);
        default: return with(pairs_kernel<BF16, E4M3, 0>);
        }
    }
    return a.wide ? launch_after(any_kernel<BF16, E4M3, true>, grid, dim3(THREADS), 0, stream, dim3(1, 1), a, int(per))
                  : launch_after(any_kernel<BF16, E4M3, false>, grid, dim3(THREADS), 0, stream, dim3(1, 1), a, int(per));
}

}  // namespace

cudaError_t launch_append(const AppendArgs &a, int sm_count, cudaStream_t stream)
{
    const bool e = a.cache.type == STRASSEN_E4M3;
    if (a.type == STRASSEN_BF16) return e ? launch<true, true>(a, sm_count, stream) : launch<true, false>(a, sm_count, stream);
    return e ? launch<false, true>(a, sm_count, stream) : launch<false, false>(a, sm_count, stream);
}

}  // namespace strassen
