// What the norm, the adapters and the optimizer's step share: eight elements at a time, E4M3 codes and power-of-two scales.
#pragma once
#include <stdint.h>

#include "../fp4/mor_fp4.cuh"

namespace mor {
namespace {

constexpr int kPer = 8;                       // elements a thread holds side by side

// Eight consecutive elements from `at` on, of which `left` exist; the others are zero.
template <typename T> __device__ __forceinline__ void load8(float* v, const T* at, int left, bool whole)
{
    if (whole) {
        Piece<T, kPer * (int)sizeof(T)> piece;
        piece.load(at);
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] = piece.get(i);
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            Piece<T, (int)sizeof(T)> one;
            one.clear();
            if (i < left) one.load(at + i);
            v[i] = one.get(0);
        }
    }
}
template <typename T> __device__ __forceinline__ void store8(const float* v, T* at, int left, bool whole)
{
    if (whole) {
        Piece<T, kPer * (int)sizeof(T)> piece;
        piece.set_all(v);
        piece.store(at);
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            Piece<T, (int)sizeof(T)> one;
            one.set_all(v + i);
            if (i < left) one.store(at + i);
        }
    }
}
__device__ __forceinline__ uint2 load_codes(const uint8_t* at, int left, bool whole)
{
    if (whole) return *reinterpret_cast<const uint2*>(at);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (i < left) w[i >> 2] |= (uint32_t)at[i] << (8 * (i & 3));
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void store_codes(uint2 c, uint8_t* at, int left, bool whole)
{
    if (whole) {
        *reinterpret_cast<uint2*>(at) = c;
        return;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (i < left) at[i] = (uint8_t)((i < 4 ? c.x : c.y) >> (8 * (i & 3)));
}

// Biased exponent of the largest power of two that keeps a >= 0 within 448 = 1.75 * 2^8, at most `most`; 127 for zero.
__device__ __forceinline__ uint32_t power_scale(float a, uint32_t most)
{
    // 2 * 127 + 8 - field of a, one less where a's fraction is above 1.75: it then carries.  Subnormal values are far below what `most` leaves of it.
    const int e = 262 - (int)((__float_as_uint(a) + 0x1FFFFFu) >> 23);
    return a == 0.f ? 127u : min((uint32_t)max(e, 1), most);
}
// 1 / 2^(e - 127) for a biased exponent of 0 .. 254, exact.
__device__ __forceinline__ float inverse_power(uint32_t e) { return e >= 254u ? 0x1p-127f : __uint_as_float((254u - e) << 23); }

// Four codes of four values, the first in the lowest byte; nearest even, saturating, NaN is 0x7F.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d)
{
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | (uint32_t)hi << 16;
}
__device__ __forceinline__ uint2 e4m3x8(const float* v) { return make_uint2(e4m3x4(v[0], v[1], v[2], v[3]), e4m3x4(v[4], v[5], v[6], v[7])); }
__device__ __forceinline__ void e4m3x2_values(float* v, uint16_t c)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(c));
    const float2 f = __half22float2(*reinterpret_cast<__half2*>(&h));
    v[0] = f.x;
    v[1] = f.y;
}
__device__ __forceinline__ void e4m3x4_values(float* v, uint32_t c)
{
    e4m3x2_values(v, (uint16_t)c);
    e4m3x2_values(v + 2, (uint16_t)(c >> 16));
}
__device__ __forceinline__ void e4m3x8_values(float* v, uint2 c)
{
    e4m3x4_values(v, c.x);
    e4m3x4_values(v + 4, c.y);
}

}  // namespace
}  // namespace mor
