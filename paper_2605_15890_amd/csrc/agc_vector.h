// Eight consecutive values of a row, binary32 or bfloat16, as floats: what the element-wise operators move at a time; and a
// division for their indexes.
#pragma once

#include "agc_tile.h"

namespace agc {

// Division by a number that the host knows: n / d = n * magic >> shift for n < 2^31, with a magic of 32 bits.
struct Divider {
    uint32_t d, magic, shift;
    explicit Divider(uint32_t by) : d(by)
    {
        int bits = 0;
        while ((1u << bits) < by) ++bits;
        shift = 31 + bits;
        magic = (uint32_t)(((uint64_t)1 << shift) / by + ((by & (by - 1)) != 0));
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return (uint32_t)(((uint64_t)n * magic) >> shift); }
};

// 16 bytes from and to any address: the memory path takes unaligned vectors (a row of odd width begins anywhere), an aligned
// one costs nothing extra.
template <typename T>
__device__ __forceinline__ tile_u32x4 load16(const T* p)
{
    tile_u32x4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}

template <typename T>
__device__ __forceinline__ void store16(T* p, tile_u32x4 v)
{
    __builtin_memcpy(p, &v, 16);
}

// The first `count` of eight values; the others are zeros.
__device__ __forceinline__ void load8(const uint16_t* p, int count, float v[8])
{
    if (count >= 8) {
        bf16_unpack8(load16(p), v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < count ? __uint_as_float((uint32_t)p[i] << 16) : 0.0f;
    }
}

__device__ __forceinline__ void load8(const float* p, int count, float v[8])
{
    if (count >= 8) {
        const tile_u32x4 a = load16(p), b = load16(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(a[i]), v[4 + i] = __uint_as_float(b[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < count ? p[i] : 0.0f;
    }
}

__device__ __forceinline__ void store8(uint16_t* p, int count, const float v[8])
{
    if (count >= 8) {
        store16(p, bf16_pack8(v));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) p[i] = (uint16_t)bf16_bits(v[i]);
    }
}

__device__ __forceinline__ void store8(float* p, int count, const float v[8])
{
    if (count >= 8) {
        tile_u32x4 a, b;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(v[i]), b[i] = __float_as_uint(v[4 + i]);
        store16(p, a);
        store16(p + 4, b);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) p[i] = v[i];
    }
}

}  // namespace agc
