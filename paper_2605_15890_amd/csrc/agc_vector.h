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

// The first `count` of four or eight values; the others are zeros.  Runs that are not whole are fetched and stored by fours and
// at most three single values: 9066 tokens of 22 heads of 59 take 23.6 us, with up to seven single ones 30.6.
__device__ __forceinline__ void load4(const uint16_t* p, int count, float v[4])
{
    if (count >= 4) {
        uint32_t u[2];
        __builtin_memcpy(u, p, 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(i & 1 ? u[i / 2] & 0xFFFF0000u : u[i / 2] << 16);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < 3 && i < count ? __uint_as_float((uint32_t)p[i] << 16) : 0.0f;
    }
}

__device__ __forceinline__ void load8(const uint16_t* p, int count, float v[8])
{
    if (count >= 8) {
        bf16_unpack8(load16(p), v);
    } else {
        load4(p, count, v);
        load4(p + 4, count - 4, v + 4);
    }
}

__device__ __forceinline__ void load4(const float* p, int count, float v[4])
{
    if (count >= 4) {
        const tile_u32x4 a = load16(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(a[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < 3 && i < count ? p[i] : 0.0f;
    }
}

__device__ __forceinline__ void load8(const float* p, int count, float v[8])
{
    if (count >= 8) {
        const tile_u32x4 a = load16(p), b = load16(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(a[i]), v[4 + i] = __uint_as_float(b[i]);
    } else {
        load4(p, count, v);
        load4(p + 4, count - 4, v + 4);
    }
}

__device__ __forceinline__ void store4(uint16_t* p, int count, const uint32_t pairs[2])
{
    if (count >= 4) {
        __builtin_memcpy(p, pairs, 8);
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < count) p[i] = (uint16_t)(pairs[i / 2] >> (i & 1) * 16);
    }
}

__device__ __forceinline__ void store8(uint16_t* p, int count, const float v[8])
{
    const tile_u32x4 bits = bf16_pack8(v);
    if (count >= 8) {
        store16(p, bits);
    } else {
        const uint32_t low[2] = {bits[0], bits[1]}, high[2] = {bits[2], bits[3]};
        store4(p, count, low);
        store4(p + 4, count - 4, high);
    }
}

__device__ __forceinline__ void store4(float* p, int count, const float v[4])
{
    if (count >= 4) {
        tile_u32x4 a;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(v[i]);
        store16(p, a);
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < count) p[i] = v[i];
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
        store4(p, count, v);
        store4(p + 4, count - 4, v + 4);
    }
}

}  // namespace agc
