// What the 4-bit kernels share: the E2M1 and scale conversions of one unit (32 consecutive elements), vector accesses,
// the layout of the scale tiles, and the host-side checks of an operand.
#pragma once
#include <atomic>
#include <utility>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "mor.h"

namespace mor {
namespace {

constexpr int kUnit = 32;                 // elements one thread converts at a time: two E4M3_16 blocks or one E8M0_32 block
constexpr int kScaleTile = 512;           // bytes of a scale tile: 128 rows x 4 blocks

template <int FMT> struct Fp4 {
    static constexpr int kBlock = FMT == MOR_FP4_E4M3_16 ? 16 : 32;
    static constexpr int kBlocksPerUnit = kUnit / kBlock;
};

// Byte of a row and a block inside its scale tile.
__device__ __forceinline__ int scale_at(int row, int block) { return (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3); }

// What a thread needs of the tensor's maximum.
struct TensorScale {
    float t;        // tensor scale
    float den;      // A * 2^-16 (block scales are fl(448 a / A); both sides carry 2^-16 so that 448 a cannot overflow)
    float inv;      // fl(1 / den)
};
__device__ __forceinline__ TensorScale tensor_scale_of(float amax)
{
    const float a = fmaxf(amax, 0x1p-88f);      // below 2^-88 the reciprocal of s * t could overflow
    return {a * (1.0f / 2688.0f), a * 0x1p-16f, __frcp_rn(a * 0x1p-16f)};
}
// fl(448 a / A): the product with the rounded reciprocal, corrected once by its exact remainder, is the correctly rounded
// quotient (P. Markstein, "Computation of elementary functions on the IBM RISC System/6000 processor", 1990).  What exceeds
// 512 saturates anyway and is held there, so that no infinity meets a zero.
__device__ __forceinline__ float block_quotient(float a, const TensorScale& ts)
{
    const float num = a * (448.0f / 65536.0f), q = fminf(num * ts.inv, 512.0f);
    return fmaf(fmaf(-q, ts.den, num), ts.inv, q);
}
// fl(1 / fl(s t)) for the value s of each E4M3 code (zero for zero).
__device__ __forceinline__ void fill_factors(float* factors, float t, int tid)
{
    if (tid < 127) {
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)tid));
        const float s = __low2float(*reinterpret_cast<__half2*>(&h));
        factors[tid] = tid == 0 ? 0.f : __frcp_rn(s * t);
    } else if (tid == 127) {
        factors[127] = 0.f;
    }
}

// Largest magnitude; NaN if any element is NaN (then, and for infinities, the result is not below infinity).
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
    return r;
}
template <int N> __device__ __forceinline__ float amax_of(const float* v)
{
    float m0 = 0.f, m1 = 0.f;
#pragma unroll
    for (int i = 0; i < N; i += 2) { m0 = max_nan(m0, v[i]); m1 = max_nan(m1, v[i + 1]); }
    return max_nan(m0, m1);
}
// The same for pairs of BF16, each half by itself; the signs of the result mean nothing.
__device__ __forceinline__ uint32_t max_nan_pairs(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <int N> __device__ __forceinline__ uint32_t amax_of_words(const uint32_t* w)
{
    if constexpr (N == 1) return w[0];
    else return max_nan_pairs(amax_of_words<N / 2>(w), amax_of_words<N - N / 2>(w + N / 2));
}
__device__ __forceinline__ float amax_of_pair(uint32_t m)
{
    return max_nan(fabsf(__uint_as_float(m << 16)), __uint_as_float(m & 0xFFFF0000u));
}

// Eight E2M1 codes of v[0..7] * q, the first in the lowest four bits.
__device__ __forceinline__ uint32_t e2m1x8(const float* v, float q)
{
    uint32_t r;
    asm("{ .reg .b8 b0, b1, b2, b3;\n"
        ".reg .b64 q, p0, p1, p2, p3;\n"
        ".reg .f32 x0, x1, x2, x3, x4, x5, x6, x7;\n"
        "mov.b64 q, {%9, %9};\n"
        "mov.b64 p0, {%1, %2};\nmov.b64 p1, {%3, %4};\nmov.b64 p2, {%5, %6};\nmov.b64 p3, {%7, %8};\n"
        "mul.rn.f32x2 p0, p0, q;\nmul.rn.f32x2 p1, p1, q;\nmul.rn.f32x2 p2, p2, q;\nmul.rn.f32x2 p3, p3, q;\n"
        "mov.b64 {x0, x1}, p0;\nmov.b64 {x2, x3}, p1;\nmov.b64 {x4, x5}, p2;\nmov.b64 {x6, x7}, p3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b0, x1, x0;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b1, x3, x2;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b2, x5, x4;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b3, x7, x6;\n"
        "mov.b32 %0, {b0, b1, b2, b3}; }"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(q));
    return r;
}

// The same for BF16 values where they lie in words, without taking the halves apart first (that costs an integer instruction per
// element, and the integer pipe is what bounds these kernels): PAIRS, the two halves of four words one after the other;
// LOW or HIGH, that half of eight words.  Widened by the mixed-precision subtract x - 0 (keeps -0), multiplied in pairs, cast in
// pairs: two instructions per element.
enum Halves : int { PAIRS = 0, LOW = 1, HIGH = 2 };
#define MOR_TAKE_PAIRS                                                                                                                \
    "mov.b32 {h0, h1}, %1;\nmov.b32 {h2, h3}, %2;\nmov.b32 {h4, h5}, %3;\nmov.b32 {h6, h7}, %4;\n"
#define MOR_TAKE_LOW                                                                                                                  \
    "mov.b32 {h0, g}, %1;\nmov.b32 {h1, g}, %2;\nmov.b32 {h2, g}, %3;\nmov.b32 {h3, g}, %4;\n"                                      \
    "mov.b32 {h4, g}, %5;\nmov.b32 {h5, g}, %6;\nmov.b32 {h6, g}, %7;\nmov.b32 {h7, g}, %8;\n"
#define MOR_TAKE_HIGH                                                                                                                 \
    "mov.b32 {g, h0}, %1;\nmov.b32 {g, h1}, %2;\nmov.b32 {g, h2}, %3;\nmov.b32 {g, h3}, %4;\n"                                      \
    "mov.b32 {g, h4}, %5;\nmov.b32 {g, h5}, %6;\nmov.b32 {g, h6}, %7;\nmov.b32 {g, h7}, %8;\n"
#define MOR_REGS ".reg .b8 b0, b1, b2, b3;\n.reg .b16 h0, h1, h2, h3, h4, h5, h6, h7, g;\n.reg .f32 x0, x1, x2, x3, x4, x5, x6, x7;\n"
#define MOR_CAST                                                                                                                      \
    "cvt.rn.satfinite.e2m1x2.f32 b0, x1, x0;\ncvt.rn.satfinite.e2m1x2.f32 b1, x3, x2;\n"                                             \
    "cvt.rn.satfinite.e2m1x2.f32 b2, x5, x4;\ncvt.rn.satfinite.e2m1x2.f32 b3, x7, x6;\nmov.b32 %0, {b0, b1, b2, b3}; }"
#define MOR_WIDEN                                                                                                                     \
    ".reg .b64 q, p0, p1, p2, p3;\nmov.b64 q, {%9, %9};\n"                                                                           \
    "sub.f32.bf16 x0, h0, %10;\nsub.f32.bf16 x1, h1, %10;\nsub.f32.bf16 x2, h2, %10;\nsub.f32.bf16 x3, h3, %10;\n"                  \
    "sub.f32.bf16 x4, h4, %10;\nsub.f32.bf16 x5, h5, %10;\nsub.f32.bf16 x6, h6, %10;\nsub.f32.bf16 x7, h7, %10;\n"                  \
    "mov.b64 p0, {x0, x1};\nmov.b64 p1, {x2, x3};\nmov.b64 p2, {x4, x5};\nmov.b64 p3, {x6, x7};\n"                                  \
    "mul.rn.f32x2 p0, p0, q;\nmul.rn.f32x2 p1, p1, q;\nmul.rn.f32x2 p2, p2, q;\nmul.rn.f32x2 p3, p3, q;\n"                          \
    "mov.b64 {x0, x1}, p0;\nmov.b64 {x2, x3}, p1;\nmov.b64 {x4, x5}, p2;\nmov.b64 {x6, x7}, p3;\n"
template <int WHICH> __device__ __forceinline__ uint32_t e2m1x8_of(const uint32_t* w, float q)
{
    uint32_t r;
    constexpr int k = WHICH == PAIRS ? 0 : 1;                         // PAIRS uses four words only
#define MOR_ASM(TAKE)                                                                                                                 \
    asm("{ " MOR_REGS TAKE MOR_WIDEN MOR_CAST                                                                                         \
        : "=r"(r) : "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4 * k]), "r"(w[5 * k]), "r"(w[6 * k]), "r"(w[7 * k]), "f"(q), "f"(0.0f))
    if constexpr (WHICH == PAIRS) MOR_ASM(MOR_TAKE_PAIRS);
    else if constexpr (WHICH == LOW) MOR_ASM(MOR_TAKE_LOW);
    else MOR_ASM(MOR_TAKE_HIGH);
    return r;
}
#undef MOR_ASM
#undef MOR_WIDEN
#undef MOR_CAST
#undef MOR_REGS
#undef MOR_TAKE_HIGH
#undef MOR_TAKE_LOW
#undef MOR_TAKE_PAIRS

// Where the 32 values of a unit are: FP32 registers, or BF16 in words.
struct UnitF32 {
    const float* v;
    __device__ __forceinline__ uint32_t cast8(int i, float q) const { return e2m1x8(v + 8 * i, q); }
};
template <int WHICH> struct UnitBf16 {
    const uint32_t* w;
    __device__ __forceinline__ uint32_t cast8(int i, float q) const { return e2m1x8_of<WHICH>(w + (WHICH == PAIRS ? 4 : 8) * i, q); }
};

// Codes (16 bytes) and scale bytes (low byte first) of one unit, given the largest magnitude of each of its blocks.
template <int FMT, typename U> __device__ __forceinline__ uint4 quantise_unit(const U& unit, const float* a, const TensorScale& ts, const float* factors, uint32_t& scales)
{
    float q0, q1;
    bool bad0, bad1;
    if constexpr (FMT == MOR_FP4_E8M0_32) {
        bad0 = bad1 = !(a[0] < INFINITY);
        // floor(log2 a) - 2 with a bias of 127 is the exponent field less two; the fields 0 (subnormal or zero), 1 and 2 meet
        // the bound at 0
        const int byte = max((int)(__float_as_uint(a[0]) >> 23) - 2, 0);
        q0 = q1 = __uint_as_float((uint32_t)(254 - byte) << 23);
        scales = bad0 ? 0xFFu : (uint32_t)byte;
    } else {
        bad0 = !(a[0] < INFINITY);
        bad1 = !(a[1] < INFINITY);
        uint16_t s;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(s) : "f"(block_quotient(a[1], ts)), "f"(block_quotient(a[0], ts)));
        scales = s;
        q0 = factors[s & 127];
        q1 = factors[(s >> 8) & 127];
        if (bad0) scales = (scales & 0xFF00u) | 0x7Fu;
        if (bad1) scales = (scales & 0x00FFu) | 0x7F00u;
    }
    uint4 c = make_uint4(unit.cast8(0, q0), unit.cast8(1, q0), unit.cast8(2, q1), unit.cast8(3, q1));
    if (bad0) c.x = c.y = 0;
    if (bad1) c.z = c.w = 0;
    return c;
}

// Value of a scale byte.
template <int FMT> __device__ __forceinline__ float scale_value(uint32_t byte)
{
    if constexpr (FMT == MOR_FP4_E8M0_32) {
        if (byte == 0xFFu) return __uint_as_float(0x7FC00000u);
        return byte == 0 ? 0x1p-127f : __uint_as_float(byte << 23);
    } else {
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)byte));
        return __low2float(*reinterpret_cast<__half2*>(&h));
    }
}

// Two E2M1 codes (a byte) as values, the low half first.
__device__ __forceinline__ float2 e2m1x2_value(uint32_t byte)
{
    uint32_t h;
    asm("{ .reg .b8 b, z0, z1, z2; mov.b32 {b, z0, z1, z2}, %1; cvt.rn.f16x2.e2m1x2 %0, b; }" : "=r"(h) : "r"(byte));
    return __half22float2(*reinterpret_cast<__half2*>(&h));
}

// ---- vector accesses: 32 bytes (one sector) per thread, 16 bytes, or one element

__device__ __forceinline__ void ldg256(uint32_t* r, const void* p)
{
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "l"(p));
}
__device__ __forceinline__ void stg256(void* p, const uint32_t* r)
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t bf16x2_of(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float weight_at(const void* w, int dtype, int64_t i)
{
    return dtype == MOR_DTYPE_BF16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(w)[i]) : static_cast<const float*>(w)[i];
}

// What one thread moves at a time: BYTES bytes as 32-bit values.  LOAD: bytes of a load at most, where an address is a multiple of fewer.
template <typename T, int BYTES, int LOAD = BYTES> struct Piece {
    static constexpr int kElems = BYTES / (int)sizeof(T);
    static constexpr int kWords = BYTES < 4 ? 1 : BYTES / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T* p)
    {
        if constexpr (BYTES >= 32 && LOAD >= 32) {
#pragma unroll
            for (int i = 0; i < kWords; i += 8) ldg256(w + i, reinterpret_cast<const uint32_t*>(p) + i);
        } else if constexpr (BYTES >= 16) {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const uint4 q = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint32_t*>(p) + i);
                w[i] = q.x; w[i + 1] = q.y; w[i + 2] = q.z; w[i + 3] = q.w;
            }
        } else if constexpr (BYTES == 4) w[0] = *reinterpret_cast<const uint32_t*>(p);
        else w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
    __device__ __forceinline__ void store(T* p) const
    {
        if constexpr (BYTES >= 32) {
#pragma unroll
            for (int i = 0; i < kWords; i += 8) stg256(reinterpret_cast<uint32_t*>(p) + i, w + i);
        } else if constexpr (BYTES == 16) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else if constexpr (BYTES == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
        else *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
    }
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return i & 1 ? bf16_high(w[i >> 1]) : bf16_low(w[i >> 1]);
    }
    __device__ __forceinline__ void set_all(const float* v)
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < kElems; ++i) w[i] = __float_as_uint(v[i]);
        } else if constexpr (kElems == 1) w[0] = bf16x2_of(v[0], 0.f);
        else {
#pragma unroll
            for (int i = 0; i < kElems; i += 2) w[i >> 1] = bf16x2_of(v[i], v[i + 1]);
        }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (uint32_t& u : w) u = 0;
    }
    __device__ __forceinline__ Piece scaled(float s) const
    {
        float v[kElems];
        Piece r;
#pragma unroll
        for (int i = 0; i < kElems; ++i) v[i] = get(i) * s;
        r.set_all(v);
        return r;
    }
};

// BYTES bytes from an address that need not be aligned, as words: the aligned 16-byte chunks that hold them (one more than there are
// bytes for, unless the address is aligned), put in place by shifts.  Both ends' whole chunks have to be readable.
template <typename T, int BYTES> __device__ __forceinline__ void load_shifted(uint32_t* w, const T* from)
{
    static_assert(BYTES % 16 == 0, "whole chunks");
    constexpr int kWords = BYTES / 4;
    const uint32_t phase = (uint32_t)reinterpret_cast<uintptr_t>(from) & 15u;
    const uint4* chunks = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(from) - phase);
    uint32_t v[kWords + 4];
#pragma unroll
    for (int i = 0; i < kWords; i += 4) {
        const uint4 q = chunks[i / 4];
        v[i] = q.x; v[i + 1] = q.y; v[i + 2] = q.z; v[i + 3] = q.w;
    }
    uint4 q = make_uint4(0, 0, 0, 0);
    if (phase != 0) q = chunks[kWords / 4];
    v[kWords] = q.x; v[kWords + 1] = q.y; v[kWords + 2] = q.z; v[kWords + 3] = q.w;
#pragma unroll
    for (int i = 0; i < kWords + 2; ++i) v[i] = phase & 8u ? v[i + 2] : v[i];
#pragma unroll
    for (int i = 0; i < kWords + 1; ++i) v[i] = phase & 4u ? v[i + 1] : v[i];
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = sizeof(T) == 4 ? v[i] : __funnelshift_r(v[i], v[i + 1], (phase & 2u) * 8u);
}
// How many elements an address lies past a 16-byte boundary.
template <typename T> __device__ __forceinline__ int phase_of(const T* p) { return (int)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T)); }
// Elements [at, at + BYTES / sizeof(T)), at >= 0, of a row of n that may start anywhere; from n on they are zero.  Where the chunks would
// reach past the row's ends, element by element.
template <typename T, int BYTES> __device__ __forceinline__ void load_any(uint32_t* w, const T* row, int64_t at, int64_t n)
{
    constexpr int kElems = BYTES / (int)sizeof(T), kWords = BYTES / 4, kPer = 16 / (int)sizeof(T);
    const int phase = phase_of(row + at);
    if (at >= phase && at - phase + kElems + (phase != 0 ? kPer : 0) <= n) {
        load_shifted<T, BYTES>(w, row + at);
    } else if constexpr (sizeof(T) == 2) {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(row) + at;
        const int left = (int)min((int64_t)kElems, n - at);
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = (2 * i < left ? h[2 * i] : 0u) | (2 * i + 1 < left ? (uint32_t)h[2 * i + 1] << 16 : 0u);
    } else {
        const int left = (int)min((int64_t)kElems, n - at);
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = i < left ? reinterpret_cast<const uint32_t*>(row)[at + i] : 0u;
    }
}

// ---- host side

inline bool is_dtype(int d) { return d == MOR_DTYPE_BF16 || d == MOR_DTYPE_F32; }
inline size_t dtype_bytes(int d) { return d == MOR_DTYPE_BF16 ? 2 : 4; }
inline bool is_aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t scale_blocks(int64_t cols, int format) { return ceil_div(cols, format == MOR_FP4_E4M3_16 ? 16 : 32); }
inline int64_t scale_ktiles(int64_t cols, int format) { return ceil_div(scale_blocks(cols, format), 4); }

// Widest access that base, pitch and batch pitch (bytes) allow: 32, 16, 8, 4, or `element`.
inline int access_bytes(const void* p, int64_t pitch, int64_t batch_pitch, int element)
{
    const uint64_t all = reinterpret_cast<uintptr_t>(p) | (uint64_t)pitch | (uint64_t)batch_pitch;
    return all % 32 == 0 ? 32 : all % 16 == 0 ? 16 : all % 8 == 0 ? 8 : all % 4 == 0 ? 4 : element;
}

// Sizes that every index computation of the kernels can hold.
inline bool shape_ok(int64_t batch, int64_t rows, int64_t cols)
{
    const int64_t lim = (int64_t)1 << 31;
    if (batch < 0 || rows < 0 || cols < 0 || batch >= lim || rows >= lim - 128 || cols >= lim - 128) return false;
    const int64_t tiles = ceil_div(rows, 128) * ceil_div(cols, 64);
    return tiles < lim && (batch == 0 || tiles == 0 || batch <= (lim - 1) / tiles);
}

inline mor_status_t check_matrix(const mor_fp4_matrix_t& m)
{
    if (!shape_ok(m.batch, m.rows, m.cols)) return MOR_ERR_INVALID_ARG;
    if (m.format != MOR_FP4_E4M3_16 && m.format != MOR_FP4_E8M0_32) return MOR_ERR_INVALID_ARG;
    if (m.ld < ceil_div(m.cols, 32) * 16) return MOR_ERR_INVALID_ARG;
    if (m.tensor_scale == nullptr) return MOR_ERR_INVALID_ARG;
    const bool empty = m.batch == 0 || m.rows == 0 || m.cols == 0;
    if (!empty && (m.codes == nullptr || m.scales == nullptr)) return MOR_ERR_INVALID_ARG;
    if (m.ld % 16 != 0 || !is_aligned(m.codes, 16) || !is_aligned(m.scales, 16) || !is_aligned(m.tensor_scale, 4)) return MOR_ERR_ALIGNMENT;
    return MOR_OK;
}

// Lets a kernel use more than 48 KiB of dynamic shared memory, once per device and kernel (`done`: a bit per device).
template <typename K> inline bool allow_smem(K kernel, int bytes, std::atomic<uint64_t>& done)
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    const uint64_t bit = 1ull << (dev & 63);
    if (done.load(std::memory_order_acquire) & bit) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
    if (dev < 64) done.fetch_or(bit, std::memory_order_release);
    return true;
}

// A kernel may be launched so that it starts while the stream's previous kernel ends; each calls this before it touches anything that
// kernel may have written.  It lets the next kernel start only after its own wait, so that whatever starts early finds everything
// older than its direct predecessor complete.
__device__ __forceinline__ void wait_for_predecessor()
{
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();
}

// An early start saves two to four microseconds where a kernel is over soon or fills the GPU exactly.  One of many small CTAs should
// not have it: its first CTAs crowd the multiprocessors that fall free first, and neighbouring tiles then run at different times for
// the whole kernel (quantising 8192 x 14336 both ways and back: 239 us with early starts throughout, 213 without).
constexpr uint32_t kEarlyGrid = 148 * 2;

template <typename... P, typename... A>
inline cudaError_t launch(void (*kernel)(P...), uint32_t grid, uint32_t block, size_t smem, cudaStream_t stream, bool early, A&&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = early ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<A>(args)...);
}

}  // namespace
}  // namespace mor
