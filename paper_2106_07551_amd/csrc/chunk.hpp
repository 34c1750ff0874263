// Elements of the learner's matrices (fp32 or bf16) in chunks of 16 bytes: loads
// and stores at any element's address that touch nothing behind a row's end.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device.hpp"

namespace malib {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// 16 bytes at any element's address (global memory takes unaligned vectors)
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

struct bf16_t {
    uint16_t b;
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16_t x) { return __uint_as_float((uint32_t)x.b << 16); }
template <typename E>
__device__ __forceinline__ E from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x)
{
    return x;
}
template <>
__device__ __forceinline__ bf16_t from_f32<bf16_t>(float x)
{
    return bf16_t{__builtin_bit_cast(uint16_t, (__bf16)x)};
}

// A chunk: 16 bytes of consecutive elements, the unit of every load.
template <typename E>
constexpr int kChunk = 16 / (int)sizeof(E);
template <typename E>
__device__ __forceinline__ void unpack(u32x4 v, float (&f)[kChunk<E>])
{
    if constexpr (sizeof(E) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            f[i] = __uint_as_float(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(v[i] << 16);
            f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
        }
    }
}

template <typename E>
__device__ __forceinline__ u32x4 pack(const float (&f)[kChunk<E>])
{
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v[i] = sizeof(E) == 4 ? __float_as_uint(f[i]) : pack_bf16x2(f[2 * i], f[2 * i + 1]);
    return v;
}

// v without its first `s` elements (0 <= s <= a chunk's), zeros behind the rest.
template <typename E>
__device__ __forceinline__ u32x4 drop_front(u32x4 v, int s)
{
    const int bits = s * 8 * (int)sizeof(E);
    uint64_t lo = (uint64_t)v[0] | (uint64_t)v[1] << 32, hi = (uint64_t)v[2] | (uint64_t)v[3] << 32;
    if (bits >= 64) {
        lo = bits >= 128 ? 0 : hi >> (bits - 64);
        hi = 0;
    } else if (bits > 0) {
        lo = lo >> bits | hi << (64 - bits);
        hi >>= bits;
    }
    return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// The first n (>= 1) elements of the chunk at p, zeros behind them.  Nothing behind
// them is read: a short chunk is the end of the 16 bytes before its own end, where
// `before` elements in front of p make that possible, and is read element by element
// only in arrays shorter than a chunk.  (Element by element everywhere, a row's short
// end cost its wavefront up to eight loads one after the other.)
template <typename E>
__device__ __forceinline__ u32x4 load_chunk(const E* p, int n, int64_t before)
{
    const int short_by = n < kChunk<E> ? kChunk<E> - n : 0;
    if (short_by <= before) {
        const u32x4 v = *(const u32x4_any*)(p - short_by);
        return short_by ? drop_front<E>(v, short_by) : v;
    }
    u32x4 v = {0, 0, 0, 0};
    if constexpr (sizeof(E) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n)
                v[i] = __float_as_uint(p[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n)
                v[i >> 1] |= (uint32_t)p[i].b << (16 * (i & 1));
    }
    return v;
}

template <typename E>
__device__ __forceinline__ void store_chunk(E* p, int n, u32x4 v)
{
    if (n >= kChunk<E>) {
        *(u32x4_any*)p = v;
        return;
    }
    if constexpr (sizeof(E) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n)
                p[i] = __uint_as_float(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n)
                p[i].b = (uint16_t)(v[i >> 1] >> (16 * (i & 1)));
    }
}

}  // namespace malib
