// elements.h - element types of the operators that take more than binary32 (GRAVAC_FLOAT32, _BFLOAT16, _FLOAT16):
// conversion to and from binary32, and 16-byte accesses that need no more than the element's own alignment (global memory
// of gfx950 takes them at any byte).
#ifndef GRAVAC_ELEMENTS_H
#define GRAVAC_ELEMENTS_H

#include <hip/hip_runtime.h>

#include <cstdint>

#include "gravac.h"

namespace elements {

struct F32 { using word = uint32_t; static constexpr int SIZE = 4; };
struct BF16 { using word = uint16_t; static constexpr int SIZE = 2; };
struct F16 { using word = uint16_t; static constexpr int SIZE = 2; };

inline bool known(int type) { return type == GRAVAC_FLOAT32 || type == GRAVAC_BFLOAT16 || type == GRAVAC_FLOAT16; }
inline int size_of(int type) { return type == GRAVAC_FLOAT32 ? 4 : 2; }

// Rows of `length` that begin `stride` >= length apart; bytes or elements.
struct Rows { int64_t begin, rows, length, stride; };

// Whether two of them share anything.
inline bool share(const Rows& x, const Rows& y)
{
    typedef __int128 wide;
    if (x.rows < 1 || y.rows < 1) return false;
    const Rows &a = x.rows < y.rows ? y : x, &b = x.rows < y.rows ? x : y;   // b: the one with fewer rows
    const wide d = (wide)b.begin - a.begin;
    if (d >= (wide)(a.rows - 1) * a.stride + a.length || -d >= (wide)(b.rows - 1) * b.stride + b.length) return false;
    auto floor_of = [](wide p, wide q) { return p / q - (p % q < 0 ? 1 : 0); };
    if (a.stride == b.stride) {
        // a row of b begins d + k stride behind one of a, k = 1 - a.rows .. b.rows - 1: the first of these behind -b.length
        const wide k = floor_of(-(wide)b.length - d, a.stride) + 1, first = k < 1 - (wide)a.rows ? 1 - (wide)a.rows : k;
        return first < b.rows && d + first * a.stride < a.length;
    }
    for (int64_t j = 0; j < b.rows; ++j) {
        const wide at = d + (wide)j * b.stride;
        wide i = floor_of(at + b.length - 1, a.stride);   // the last row of a that begins before b's ends
        if (i >= a.rows) i = a.rows - 1;
        if (i >= 0 && i * a.stride + a.length > at) return true;
    }
    return false;
}

inline Rows rows_at(const void* p, int64_t rows, int64_t length, int64_t stride, int size)   // in bytes
{
    return {(int64_t)(uintptr_t)p, rows, length * size, stride * size};
}
inline Rows bytes_at(const void* p, int64_t bytes) { return {(int64_t)(uintptr_t)p, bytes > 0 ? 1 : 0, bytes, bytes}; }

template <typename E> __device__ __forceinline__ float to_float(typename E::word w);
template <> __device__ __forceinline__ float to_float<F32>(uint32_t w) { return __uint_as_float(w); }
template <> __device__ __forceinline__ float to_float<BF16>(uint16_t w) { return __uint_as_float((uint32_t)w << 16); }
template <> __device__ __forceinline__ float to_float<F16>(uint16_t w) { return (float)__builtin_bit_cast(_Float16, w); }

// one rounding to nearest, ties to even (gfx950 converts to bfloat16 and to binary16 in hardware)
template <typename E> __device__ __forceinline__ typename E::word from_float(float x);
template <> __device__ __forceinline__ uint32_t from_float<F32>(float x) { return __float_as_uint(x); }
template <> __device__ __forceinline__ uint16_t from_float<BF16>(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
template <> __device__ __forceinline__ uint16_t from_float<F16>(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }

// N consecutive elements as one access, at the alignment of an element
template <typename E, int N>
struct __attribute__((packed, aligned(E::SIZE))) Pack {
    typename E::word w[N];
};

template <typename E, int N>
__device__ __forceinline__ Pack<E, N> fetch(const typename E::word* p)
{
    Pack<E, N> v;
    __builtin_memcpy(&v, (const Pack<E, N>*)p, sizeof(v));
    return v;
}

template <typename E, int N>
__device__ __forceinline__ void unpack(const Pack<E, N>& v, float (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = to_float<E>(v.w[i]);
}

template <typename E, int N>
__device__ __forceinline__ void load(const typename E::word* p, float (&x)[N])
{
    unpack<E, N>(fetch<E, N>(p), x);
}

template <typename E, int N>
__device__ __forceinline__ void store(typename E::word* p, const float (&x)[N])
{
    Pack<E, N> v;
#pragma unroll
    for (int i = 0; i < N; ++i) v.w[i] = from_float<E>(x[i]);
    __builtin_memcpy((Pack<E, N>*)p, &v, sizeof(v));
}

// ... with the hint that the result is not read again soon
template <typename E, int N>
__device__ __forceinline__ void store_streaming(typename E::word* p, const float (&x)[N])
{
    constexpr int BYTES = N * E::SIZE, EACH = BYTES < 4 ? 4 : BYTES < 16 ? BYTES : 16;
    if (BYTES < 4) { store<E, N>(p, x); return; }
    typedef uint32_t words __attribute__((ext_vector_type(EACH / 4)));
    typedef words places __attribute__((aligned(E::SIZE)));
    typename E::word w[N];
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = from_float<E>(x[i]);
#pragma unroll
    for (int i = 0; i < BYTES / EACH; ++i) {
        words v;
        __builtin_memcpy(&v, (const char*)w + i * EACH, EACH);
        __builtin_nontemporal_store(v, (places*)p + i);
    }
}

// ... and the first `n` of them (the end of a row)
template <typename E, int N>
__device__ __forceinline__ void load_part(const typename E::word* p, int n, float (&x)[N])
{
    if (n >= N) { load<E, N>(p, x); return; }
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = i < n ? to_float<E>(p[i]) : 0.0f;
}

template <typename E, int N>
__device__ __forceinline__ void store_part(typename E::word* p, int n, const float (&x)[N])
{
    if (n >= N) { store<E, N>(p, x); return; }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < n) p[i] = from_float<E>(x[i]);
}

// A lane's N columns of a row of `dim` >= N: the last lane takes the last N, and of those the first `skip` belong to the lane
// before it.  So every access is a whole one: a load that ends a row by itself is a branch, and a wavefront waits at its end
// for the loads before it.  skip >= N: nothing is this lane's.
template <int N>
struct Columns {
    int at, skip;
    __device__ __forceinline__ Columns(int c, int dim) : at(c < dim - N ? c : dim - N), skip(c - at) {}
};

template <typename E, int N>
__device__ __forceinline__ void store_behind(typename E::word* p, int skip, const float (&x)[N])
{
    if (skip == 0) { store<E, N>(p, x); return; }
#pragma unroll
    for (int i = 1; i < N; ++i)
        if (i >= skip) p[i] = from_float<E>(x[i]);
}

// Results of more bytes than this are written with the hint that they are not read again soon: half of the 256 MB cache in
// front of memory.  Smaller ones may still be there when the next call reads them.
constexpr int64_t STREAM_BYTES = 128ll << 20;

}  // namespace elements

#endif
