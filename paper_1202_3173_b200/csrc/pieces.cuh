// Reading rows of 16-bit, 32-bit and 8-bit elements in pieces of 8, whatever their alignment.
#pragma once

#include <cstdint>

namespace strassen {

// A piece of 8 elements in 32-bit words, as they lie in memory.
template <class T> struct Words {
    static constexpr int N = 8 * int(sizeof(T)) / 4;
    uint32_t w[N];
};

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

// The same for elements of 8 bits: 8 bytes, from aligned words of 8.
__device__ __forceinline__ uint2 load_bytes8(const uint8_t *row, int64_t k, int64_t size, uintptr_t lo, uintptr_t hi)
{
    const uintptr_t at = reinterpret_cast<uintptr_t>(row + k), off = at & 7, from = at - off;
    if (k + 8 <= size && off == 0) return *reinterpret_cast<const uint2 *>(at);
    if (k + 8 <= size && from >= lo && from + 16 <= hi) {
        const uint2 u = reinterpret_cast<const uint2 *>(from)[0], v = reinterpret_cast<const uint2 *>(from)[1];
        const uint32_t a = off & 4 ? u.y : u.x, b = off & 4 ? v.x : u.y, c = off & 4 ? v.y : v.x;
        return make_uint2(__funnelshift_r(a, b, 8 * (off & 3)), __funnelshift_r(b, c, 8 * (off & 3)));
    }
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (k + i < size) w[i >> 2] |= uint32_t(row[k + i]) << (8 * (i & 3));
    return make_uint2(w[0], w[1]);
}

// The memory of a matrix of m rows, from its first element to its last.
template <class T> struct Range {
    uintptr_t lo, hi;
    __device__ Range(const void *p, int64_t m, int64_t k, int64_t ld) : lo(reinterpret_cast<uintptr_t>(p)), hi(lo + uintptr_t((m - 1) * ld + k) * sizeof(T)) {}
};

}  // namespace strassen
