// Root-mean-square norm of rows with the residual's addition before it, its gradient, its output as E4M3 codes with scales, and the values of
// such codes.
//
// Everything here is bound by memory: a row stays in registers between its reductions, so that each matrix is read and written once.  A
// row belongs to a group of G threads with N pieces of 8 columns each, piece c of thread i at columns (c G + i) 8: 16 neighbouring lanes then hold the
// 128 columns of a scale.  Up to 1024 columns a row is a warp's and no barrier is needed.  Rows of more than 16384 columns do not fit and
// are walked two or three times by a CTA, from L2 after the first.
#include <math.h>

#include "mor_layers.cuh"

namespace mor {
namespace {

constexpr int kSms = 148;
constexpr int kWideThreads = 1024;
constexpr int64_t kRowLimit = 16384;          // columns that a group holds

struct NormParams {
    int64_t rows;
    int32_t cols;
    int32_t weight_dtype;
    const void *x, *r, *w;      // gradient: h, gradient of h
    int64_t ldx, ldr;
    float eps, inv_cols;
    // norm
    void *h, *y;
    uint8_t *codes, *e8m0;
    float* f32;
    int64_t ldh, ldy, ldc;
    int32_t by_row;             // one scale for a row
    // gradient
    const void* dy;
    void *dx, *dr;
    int64_t lddy, lddx, lddr;
    float* partial;             // [CTAs][cols]
};

template <typename T, bool ANY> __device__ __forceinline__ void load_piece(float* v, const T* row, int32_t at, int32_t cols)
{
    Piece<T, kPer * (int)sizeof(T)> piece;
    if constexpr (ANY) {
        piece.clear();
        if (at < cols) load_any<T, kPer * (int)sizeof(T)>(piece.w, row, at, cols);
    } else {
        piece.clear();
        if (at < cols) piece.load(row + at);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = piece.get(i);
}
template <typename T, bool ANY> __device__ __forceinline__ void store_piece(const float* v, T* row, int32_t at, int32_t cols)
{
    if (at >= cols) return;
    if constexpr (ANY) store8(v, row + at, cols - at, at + kPer <= cols && (reinterpret_cast<uintptr_t>(row + at) & (kPer * sizeof(T) - 1)) == 0);
    else store8(v, row + at, kPer, true);
}
template <bool ANY> __device__ __forceinline__ void store_code_piece(uint2 c, uint8_t* row, int32_t at, int32_t cols)
{
    if (at >= cols) return;
    if constexpr (ANY) store_codes(c, row + at, cols - at, at + kPer <= cols && (reinterpret_cast<uintptr_t>(row + at) & 7u) == 0);
    else store_codes(c, row + at, kPer, true);
}
__device__ __forceinline__ void load_weight(float* v, const void* w, int dtype, int32_t at, int32_t cols)
{
    const bool whole = at + kPer <= cols;
    if (dtype == MOR_DTYPE_BF16) {
        const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(w) + at;
        load8(v, p, cols - at, whole && (reinterpret_cast<uintptr_t>(p) & 15u) == 0);
    } else {
        const float* p = static_cast<const float*>(w) + at;
        load8(v, p, cols - at, whole && (reinterpret_cast<uintptr_t>(p) & 31u) == 0);
    }
}

// x + residual as it is kept: rounded to the residual's type.
template <typename R> __device__ __forceinline__ float kept(float v)
{
    if constexpr (sizeof(R) == 2) return __bfloat162float(__float2bfloat16(v));
    else return v;
}

template <int G> __device__ __forceinline__ void group_barrier(int group)
{
    if constexpr (G > 32) asm volatile("barrier.cta.sync %0, %1;" ::"r"(group + 1), "n"(G) : "memory");
}
// Sum (or largest) over the threads of a group, in a fixed order.  `shared`: the group's G / 32 values; it may be written again once the
// group has met twice.
template <int G, bool MAX> __device__ __forceinline__ float group_reduce(float v, float* shared, int group)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float u = __shfl_xor_sync(0xFFFFFFFFu, v, o);
        v = MAX ? fmaxf(v, u) : v + u;
    }
    if constexpr (G > 32) {
        const int i = threadIdx.x % G;
        if ((i & 31) == 0) shared[i >> 5] = v;
        group_barrier<G>(group);
        v = shared[0];
#pragma unroll
        for (int k = 1; k < G / 32; ++k) v = MAX ? fmaxf(v, shared[k]) : v + shared[k];
    }
    return v;
}
__device__ __forceinline__ float finite_abs(float v)
{
    const float a = fabsf(v);
    return a < INFINITY ? a : 0.f;
}
// Scale from the largest magnitude; stored by one thread.
__device__ __forceinline__ float make_scale(const NormParams& p, float a, int64_t at, bool store)
{
    if (p.e8m0 != nullptr) {
        const uint32_t e = power_scale(a, 254u);
        if (store) p.e8m0[at] = (uint8_t)e;
        return __uint_as_float(e << 23);
    }
    const float s = a == 0.f ? 1.f : fminf(448.f / a, 3.402823466e+38f);
    if (store) p.f32[at] = s;
    return s;
}

// A thread's pieces of its next row come by asynchronous copies into its own part of shared memory while it works on this one; that asks for no
// barrier and no registers.  Places are counted in 16 bytes of every thread.
constexpr int kRing = 2;
template <typename T, int N, int THREADS, int G> struct RowRing {
    static constexpr int kUnits = kPer * (int)sizeof(T) / 16, kPlaces = N * kUnits;
    static __device__ __forceinline__ void fetch(uint32_t to, const T* row, int i, int32_t cols)
    {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const int32_t at = (c * G + i) * kPer;
            const int bytes = at < cols ? 16 : 0;
#pragma unroll
            for (int k = 0; k < kUnits; ++k)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                             ::"r"(to + (c * kUnits + k) * THREADS * 16), "l"(reinterpret_cast<const uint4*>(row + (at < cols ? at : 0)) + k), "r"(bytes) : "memory");
        }
    }
    static __device__ __forceinline__ void take(float* v, uint32_t from, int c)
    {
        Piece<T, kPer * (int)sizeof(T)> piece;
#pragma unroll
        for (int k = 0; k < kUnits; ++k)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(piece.w[4 * k]), "=r"(piece.w[4 * k + 1]), "=r"(piece.w[4 * k + 2]), "=r"(piece.w[4 * k + 3])
                         : "r"(from + (c * kUnits + k) * THREADS * 16) : "memory");
#pragma unroll
        for (int k = 0; k < kPer; ++k) v[k] = piece.get(k);
    }
};
__device__ __forceinline__ void ring_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void ring_wait() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }
// Rows' bytes that one thread has in the ring.
template <typename T, typename R, int N> constexpr int kForwardRing = kRing * N * kPer * (int)(sizeof(T) + sizeof(R));
template <typename T, typename R, int G, int N> constexpr bool kAhead = kForwardRing<T, R, N> * (G > 256 ? G : 256) <= 220 * 1024;    // else the row alone fills it
template <typename T, typename R, int N> constexpr int kGradRing = kRing * N * kPer * (int)(sizeof(T) + 2 * sizeof(R));

// 8192 x 4096 BF16 with a residual: 40 us for h and y (268 MB, the copy rate), 42 for h and codes (235 MB, 5.6 TB/s; conversions fill 73 % of the issue slots).
template <int G> constexpr int kForwardThreads = G > 256 ? G : 256;

template <typename T, typename R, int G, int N, bool ANY> __global__ void __launch_bounds__(kForwardThreads<G>) norm_kernel(const __grid_constant__ NormParams p)
{
    constexpr int kGroups = kForwardThreads<G> / G;
    __shared__ float shared[kGroups][2][2][G / 32];
    const int group = threadIdx.x / G, i = threadIdx.x % G;
    wait_for_predecessor();
    float w[N][kPer];
#pragma unroll
    for (int c = 0; c < N; ++c) load_weight(w[c], p.w, p.weight_dtype, (c * G + i) * kPer, p.cols);
    const int32_t blocks = p.by_row ? 1 : (p.cols + 127) >> 7;
    // where there is more than one row for a group, the next one is on its way
    constexpr int kThreads = kForwardThreads<G>;
    using XRing = RowRing<T, N, kThreads, G>;
    using RRing = RowRing<R, N, kThreads, G>;
    extern __shared__ __align__(16) uint8_t ring[];
    const int64_t step = (int64_t)gridDim.x * kGroups;
    const bool ahead = !ANY && kAhead<T, R, G, N> && p.rows > step;
    const uint32_t own = (uint32_t)__cvta_generic_to_shared(ring) + threadIdx.x * 16;
    auto place = [&](int turn) { return own + turn * (XRing::kPlaces + RRing::kPlaces) * kThreads * 16; };
    auto fetch = [&](int64_t row, int turn) {
        if (row < p.rows) {
            XRing::fetch(place(turn), static_cast<const T*>(p.x) + row * p.ldx, i, p.cols);
            if (p.r != nullptr) RRing::fetch(place(turn) + XRing::kPlaces * kThreads * 16, static_cast<const R*>(p.r) + row * p.ldr, i, p.cols);
        }
        ring_commit();
    };
    int turn = 0;
    if (ahead) fetch((int64_t)blockIdx.x * kGroups + group, 0);
    for (int64_t row = (int64_t)blockIdx.x * kGroups + group; row < p.rows; row += step, turn ^= 1) {
        float v[N][kPer];
        if (ahead) {
            fetch(row + step, turn ^ 1);
            ring_wait();
        }
        const T* x = static_cast<const T*>(p.x) + row * p.ldx;
#pragma unroll
        for (int c = 0; c < N; ++c) {
            if (ahead) XRing::take(v[c], place(turn), c);
            else load_piece<T, ANY>(v[c], x, (c * G + i) * kPer, p.cols);
        }
        if (p.r != nullptr) {
            const R* r = static_cast<const R*>(p.r) + row * p.ldr;
            float add[N][kPer];
#pragma unroll
            for (int c = 0; c < N; ++c) {
                if (ahead) RRing::take(add[c], place(turn) + XRing::kPlaces * kThreads * 16, c);
                else load_piece<R, ANY>(add[c], r, (c * G + i) * kPer, p.cols);
            }
#pragma unroll
            for (int c = 0; c < N; ++c) {
#pragma unroll
                for (int k = 0; k < kPer; ++k) v[c][k] = kept<R>(v[c][k] + add[c][k]);
                if (p.h != nullptr) store_piece<R, ANY>(v[c], static_cast<R*>(p.h) + row * p.ldh, (c * G + i) * kPer, p.cols);
            }
        }
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < N; ++c)
#pragma unroll
            for (int k = 0; k < kPer; ++k) sum = fmaf(v[c][k], v[c][k], sum);
        sum = group_reduce<G, false>(sum, shared[group][turn][0], group);
        const float rs = 1.f / sqrtf(fmaf(sum, p.inv_cols, p.eps));
#pragma unroll
        for (int c = 0; c < N; ++c) {
#pragma unroll
            for (int k = 0; k < kPer; ++k) v[c][k] = v[c][k] * rs * w[c][k];
            if (p.y != nullptr) store_piece<T, ANY>(v[c], static_cast<T*>(p.y) + row * p.ldy, (c * G + i) * kPer, p.cols);
        }
        if (p.codes == nullptr) continue;
        float a[N];
#pragma unroll
        for (int c = 0; c < N; ++c) {
            a[c] = 0.f;
#pragma unroll
            for (int k = 0; k < kPer; ++k) a[c] = fmaxf(a[c], finite_abs(v[c][k]));
        }
        if (p.by_row) {
#pragma unroll
            for (int c = 1; c < N; ++c) a[0] = fmaxf(a[0], a[c]);
            a[0] = make_scale(p, group_reduce<G, true>(a[0], shared[group][turn][1], group), row, i == 0);
#pragma unroll
            for (int c = 1; c < N; ++c) a[c] = a[0];
        } else {
#pragma unroll
            for (int c = 0; c < N; ++c) {
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) a[c] = fmaxf(a[c], __shfl_xor_sync(0xFFFFFFFFu, a[c], o));
                const int32_t at = (c * G + i) * kPer;
                a[c] = make_scale(p, a[c], row * blocks + (at >> 7), (i & 15) == 0 && at < p.cols);
            }
        }
#pragma unroll
        for (int c = 0; c < N; ++c) {
#pragma unroll
            for (int k = 0; k < kPer; ++k) v[c][k] *= a[c];
            store_code_piece<ANY>(e4m3x8(v[c]), p.codes + row * p.ldc, (c * G + i) * kPer, p.cols);
        }
    }
}

// Scales of rows without columns, that of a largest magnitude of 0.
__global__ void __launch_bounds__(256) norm_no_columns_kernel(const __grid_constant__ NormParams p)
{
    wait_for_predecessor();
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row < p.rows) make_scale(p, 0.f, row, true);
}

// Rows of any width, one a CTA.
template <typename T, typename R> __global__ void __launch_bounds__(kWideThreads) norm_wide_kernel(const __grid_constant__ NormParams p)
{
    __shared__ float shared[2][kWideThreads / 32];
    wait_for_predecessor();
    const int64_t row = blockIdx.x;
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    const R* r = p.r != nullptr ? static_cast<const R*>(p.r) + row * p.ldr : nullptr;
    R* h = p.h != nullptr && r != nullptr ? static_cast<R*>(p.h) + row * p.ldh : nullptr;
    constexpr int kStride = kWideThreads * kPer;
    const int32_t at0 = threadIdx.x * kPer;
    bool first = true;
    // h of the columns from `at` on: made in the first pass, in later ones read back where it is kept (it may lie over the residual)
    auto take = [&](float* v, int32_t at) {
        if (!first && h != nullptr) {
            load_piece<R, true>(v, h, at, p.cols);
            return;
        }
        load_piece<T, true>(v, x, at, p.cols);
        if (r == nullptr) return;
        float add[kPer];
        load_piece<R, true>(add, r, at, p.cols);
#pragma unroll
        for (int k = 0; k < kPer; ++k) v[k] = kept<R>(v[k] + add[k]);
        if (h != nullptr) store_piece<R, true>(v, h, at, p.cols);
    };
    float sum = 0.f;
    for (int32_t at = at0; at < p.cols; at += kStride) {
        float v[kPer];
        take(v, at);
#pragma unroll
        for (int k = 0; k < kPer; ++k) sum = fmaf(v[k], v[k], sum);
    }
    first = false;
    sum = group_reduce<kWideThreads, false>(sum, shared[0], 0);
    const float rs = 1.f / sqrtf(fmaf(sum, p.inv_cols, p.eps));
    auto normed = [&](float* v, int32_t at) {
        float w[kPer];
        take(v, at);
        load_weight(w, p.w, p.weight_dtype, at, p.cols);
#pragma unroll
        for (int k = 0; k < kPer; ++k) v[k] = v[k] * rs * w[k];
    };
    float scale = 0.f;
    if (p.codes != nullptr && p.by_row) {
        float a = 0.f;
        for (int32_t at = at0; at < p.cols; at += kStride) {
            float v[kPer];
            normed(v, at);
#pragma unroll
            for (int k = 0; k < kPer; ++k) a = fmaxf(a, finite_abs(v[k]));
        }
        scale = make_scale(p, group_reduce<kWideThreads, true>(a, shared[1], 0), row, threadIdx.x == 0);
    }
    for (int32_t base = 0; base < p.cols; base += kStride) {      // the same turns for all lanes: they exchange maxima
        const int32_t at = base + at0;
        float v[kPer];
        if (at < p.cols) normed(v, at);
        else
#pragma unroll
            for (int k = 0; k < kPer; ++k) v[k] = 0.f;
        if (p.y != nullptr) store_piece<T, true>(v, static_cast<T*>(p.y) + row * p.ldy, at, p.cols);
        if (p.codes == nullptr) continue;
        float s = scale;
        if (!p.by_row) {
            float a = 0.f;
#pragma unroll
            for (int k = 0; k < kPer; ++k) a = fmaxf(a, finite_abs(v[k]));
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, o));
            s = make_scale(p, a, row * ((p.cols + 127) >> 7) + (at >> 7), (threadIdx.x & 15) == 0 && at < p.cols);
        }
#pragma unroll
        for (int k = 0; k < kPer; ++k) v[k] *= s;
        store_code_piece<true>(e4m3x8(v), p.codes + row * p.ldc, at, p.cols);
    }
}

// ------------------------------------------------------------------------------------------- gradient ----

// dh = rs (g - xh mean(g xh)) + dh_in with g = dy w, xh = h rs: both sums of a row come from one reduction.  The weight's gradient is summed by
// each thread over its group's rows, then over the CTA's groups in shared memory and over the CTAs by the join, always in the same order.  One CTA an SM, since every
// CTA's sums are written and read again: 8192 x 4096 BF16, 47 us (268 MB, 5.7 TB/s), and 6 for the join, which is latency.
template <int G> constexpr int kGradThreads = G > 512 ? G : 512;

template <typename T, typename R, int G, int N, bool ANY> __global__ void __launch_bounds__(kGradThreads<G>) norm_grad_kernel(const __grid_constant__ NormParams p)
{
    constexpr int kGroups = kGradThreads<G> / G;
    __shared__ float shared[kGroups][2][2][G / 32];
    extern __shared__ __align__(16) float total[];  // [cols] with more than one group, after the rows; before, the ring
    const int group = threadIdx.x / G, i = threadIdx.x % G;
    wait_for_predecessor();
    float w[N][kPer], dw[N][kPer];
#pragma unroll
    for (int c = 0; c < N; ++c) {
        load_weight(w[c], p.w, p.weight_dtype, (c * G + i) * kPer, p.cols);
#pragma unroll
        for (int k = 0; k < kPer; ++k) dw[c][k] = 0.f;
    }
    constexpr int kThreads = kGradThreads<G>;
    using HRing = RowRing<R, N, kThreads, G>;
    using GRing = RowRing<T, N, kThreads, G>;
    const int64_t step = (int64_t)gridDim.x * kGroups;
    const bool ahead = !ANY && p.rows > step;
    const uint32_t own = (uint32_t)__cvta_generic_to_shared(total) + threadIdx.x * 16;
    constexpr uint32_t kG = HRing::kPlaces * kThreads * 16, kD = kG + GRing::kPlaces * kThreads * 16, kStage = kD + HRing::kPlaces * kThreads * 16;
    auto fetch = [&](int64_t row, int turn) {
        if (row < p.rows) {
            HRing::fetch(own + turn * kStage, static_cast<const R*>(p.x) + row * p.ldx, i, p.cols);
            GRing::fetch(own + turn * kStage + kG, static_cast<const T*>(p.dy) + row * p.lddy, i, p.cols);
            if (p.r != nullptr) HRing::fetch(own + turn * kStage + kD, static_cast<const R*>(p.r) + row * p.ldr, i, p.cols);
        }
        ring_commit();
    };
    int turn = 0;
    if (ahead) fetch((int64_t)blockIdx.x * kGroups + group, 0);
    for (int64_t row = (int64_t)blockIdx.x * kGroups + group; row < p.rows; row += step, turn ^= 1) {
        float h[N][kPer], g[N][kPer];
        if (ahead) {
            fetch(row + step, turn ^ 1);
            ring_wait();
        }
        const R* hr = static_cast<const R*>(p.x) + row * p.ldx;
        const T* dy = static_cast<const T*>(p.dy) + row * p.lddy;
#pragma unroll
        for (int c = 0; c < N; ++c) {
            if (ahead) HRing::take(h[c], own + turn * kStage, c);
            else load_piece<R, ANY>(h[c], hr, (c * G + i) * kPer, p.cols);
        }
#pragma unroll
        for (int c = 0; c < N; ++c) {
            if (ahead) GRing::take(g[c], own + turn * kStage + kG, c);
            else load_piece<T, ANY>(g[c], dy, (c * G + i) * kPer, p.cols);
        }
        float square = 0.f, dot = 0.f;
#pragma unroll
        for (int c = 0; c < N; ++c)
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                square = fmaf(h[c][k], h[c][k], square);
                dot = fmaf(g[c][k] * w[c][k], h[c][k], dot);
            }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            square += __shfl_xor_sync(0xFFFFFFFFu, square, o);
            dot += __shfl_xor_sync(0xFFFFFFFFu, dot, o);
        }
        if constexpr (G > 32) {
            float(*s)[G / 32] = shared[group][turn];
            if ((i & 31) == 0) {
                s[0][i >> 5] = square;
                s[1][i >> 5] = dot;
            }
            group_barrier<G>(group);
            square = s[0][0];
            dot = s[1][0];
#pragma unroll
            for (int k = 1; k < G / 32; ++k) {
                square += s[0][k];
                dot += s[1][k];
            }
        }
        const float rs = 1.f / sqrtf(fmaf(square, p.inv_cols, p.eps));
        const float mean = dot * rs * p.inv_cols;
#pragma unroll
        for (int c = 0; c < N; ++c) {
            float d[kPer];
            const int32_t at = (c * G + i) * kPer;
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                const float xh = h[c][k] * rs;
                dw[c][k] = fmaf(g[c][k], xh, dw[c][k]);
                d[k] = rs * fmaf(-xh, mean, g[c][k] * w[c][k]);
            }
            if (p.r != nullptr) {
                float add[kPer];
                if (ahead) HRing::take(add, own + turn * kStage + kD, c);
                else load_piece<R, ANY>(add, static_cast<const R*>(p.r) + row * p.ldr, at, p.cols);
#pragma unroll
                for (int k = 0; k < kPer; ++k) d[k] += add[k];
            }
            if (p.dx != nullptr) store_piece<T, ANY>(d, static_cast<T*>(p.dx) + row * p.lddx, at, p.cols);
            if (p.dr != nullptr) store_piece<R, ANY>(d, static_cast<R*>(p.dr) + row * p.lddr, at, p.cols);
        }
    }
    if (p.partial == nullptr) return;
    float* out = p.partial + (int64_t)blockIdx.x * p.cols;
    if constexpr (kGroups > 1) {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();                            // the ring's place is free
    }
#pragma unroll 1
    for (int turn = 0; turn < kGroups; ++turn) {
        if (group == turn) {
#pragma unroll
            for (int c = 0; c < N; ++c)
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    const int32_t at = (c * G + i) * kPer + k;
                    if (at >= p.cols) continue;
                    const float sum = turn > 0 ? total[at] + dw[c][k] : dw[c][k];
                    if (turn == kGroups - 1) out[at] = sum;
                    else total[at] = sum;
                }
        }
        if constexpr (kGroups > 1) __syncthreads();
    }
}

// Rows of any width, read twice.  The weight's gradient is summed in shared memory, or where the join reads it if there are too many columns; a
// column is one thread's.
constexpr int32_t kWideSums = 48 * 1024;
template <typename T, typename R> __global__ void __launch_bounds__(kWideThreads) norm_grad_wide_kernel(const __grid_constant__ NormParams p)
{
    __shared__ float shared[2][2][kWideThreads / 32];
    wait_for_predecessor();
    extern __shared__ float total[];
    float* const out = p.partial != nullptr ? p.partial + (int64_t)blockIdx.x * p.cols : nullptr;
    float* const sums = out != nullptr && p.cols <= kWideSums ? total : out;
    int turn = 0;
    bool first = true;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, turn ^= 1, first = false) {
        const R* hr = static_cast<const R*>(p.x) + row * p.ldx;
        const T* dy = static_cast<const T*>(p.dy) + row * p.lddy;
        float square = 0.f, dot = 0.f, h[kPer], g[kPer], w[kPer];
        for (int32_t at = threadIdx.x * kPer; at < p.cols; at += kWideThreads * kPer) {
            load_piece<R, true>(h, hr, at, p.cols);
            load_piece<T, true>(g, dy, at, p.cols);
            load_weight(w, p.w, p.weight_dtype, at, p.cols);
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                square = fmaf(h[k], h[k], square);
                dot = fmaf(g[k] * w[k], h[k], dot);
            }
        }
        square = group_reduce<kWideThreads, false>(square, shared[turn][0], 0);
        dot = group_reduce<kWideThreads, false>(dot, shared[turn][1], 0);
        const float rs = 1.f / sqrtf(fmaf(square, p.inv_cols, p.eps));
        const float mean = dot * rs * p.inv_cols;
        for (int32_t at = threadIdx.x * kPer; at < p.cols; at += kWideThreads * kPer) {
            load_piece<R, true>(h, hr, at, p.cols);
            load_piece<T, true>(g, dy, at, p.cols);
            load_weight(w, p.w, p.weight_dtype, at, p.cols);
            float d[kPer];
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                const float xh = h[k] * rs;
                if (sums != nullptr && at + k < p.cols) sums[at + k] = first ? g[k] * xh : fmaf(g[k], xh, sums[at + k]);
                d[k] = rs * fmaf(-xh, mean, g[k] * w[k]);
            }
            if (p.r != nullptr) {
                float add[kPer];
                load_piece<R, true>(add, static_cast<const R*>(p.r) + row * p.ldr, at, p.cols);
#pragma unroll
                for (int k = 0; k < kPer; ++k) d[k] += add[k];
            }
            if (p.dx != nullptr) store_piece<T, true>(d, static_cast<T*>(p.dx) + row * p.lddx, at, p.cols);
            if (p.dr != nullptr) store_piece<R, true>(d, static_cast<R*>(p.dr) + row * p.lddr, at, p.cols);
        }
    }
    if (sums == out) return;
    for (int32_t at = threadIdx.x * kPer; at < p.cols; at += kWideThreads * kPer)
#pragma unroll
        for (int k = 0; k < kPer; ++k)
            if (at + k < p.cols) out[at + k] = sums[at + k];
}

constexpr int kJoinCols = 32, kJoinParts = 8;

// Sum of the CTAs' parts of the weight's gradient, in a fixed order.
template <typename W> __global__ void __launch_bounds__(kJoinCols* kJoinParts) norm_join_kernel(const float* partial, int parts, int32_t cols, W* out)
{
    __shared__ float shared[kJoinParts][kJoinCols];
    wait_for_predecessor();
    const int32_t at = blockIdx.x * kJoinCols + threadIdx.x % kJoinCols;
    const int k = threadIdx.x / kJoinCols;
    float sum = 0.f;
    if (at < cols) {
#pragma unroll 8
        for (int i = k; i < parts; i += kJoinParts) sum += __ldcg(partial + (int64_t)i * cols + at);
    }
    shared[k][threadIdx.x % kJoinCols] = sum;
    __syncthreads();
    if (k != 0 || at >= cols) return;
#pragma unroll
    for (int j = 1; j < kJoinParts; ++j) sum += shared[j][threadIdx.x];
    Piece<W, (int)sizeof(W)> one;
    one.set_all(&sum);
    one.store(out + at);
}

// ------------------------------------------------------------------------------------------- values ----

// 16 codes a thread at a time, of kValueRows rows: 16 bytes in, 32 or 64 out.  8192 x 4096 to BF16: 25 us (101 MB, 4.0 TB/s),
// issue slots 68 % full: neither is a bound, what is left are the loads' latency and the quotients one after the other.
constexpr int kValueRows = 4;
template <typename T> __global__ void __launch_bounds__(256) codes_values_kernel(const uint8_t* codes, int64_t rows, int32_t cols, int64_t ldc, int32_t by_row,
                                                                                 const uint8_t* e8m0, const float* f32, T* out, int64_t ldo, bool aligned)
{
    wait_for_predecessor();
    const int32_t at = (blockIdx.y * blockDim.x + threadIdx.x) * 16, blocks = by_row ? 1 : (cols + 127) >> 7;
    const int64_t row0 = (int64_t)blockIdx.x * (kValueRows * blockDim.y) + threadIdx.y;
    if (at >= cols) return;
    const bool whole = aligned && at + 16 <= cols;
    uint4 c[kValueRows];
    float s[kValueRows];
#pragma unroll
    for (int k = 0; k < kValueRows; ++k) {
        const int64_t row = row0 + k * blockDim.y;
        if (row >= rows) break;
        const uint8_t* from = codes + row * ldc + at;
        if (whole) {
            c[k] = *reinterpret_cast<const uint4*>(from);
        } else {
            const uint2 lo = load_codes(from, cols - at, false), hi = load_codes(from + 8, cols - at - 8, false);
            c[k] = make_uint4(lo.x, lo.y, hi.x, hi.y);
        }
        const int64_t i = row * blocks + (by_row ? 0 : at >> 7);
        s[k] = e8m0 != nullptr ? inverse_power(e8m0[i]) : f32[i];
    }
#pragma unroll
    for (int k = 0; k < kValueRows; ++k) {
        const int64_t row = row0 + k * blockDim.y;
        if (row >= rows) break;
        float v[16];
        e4m3x8_values(v, make_uint2(c[k].x, c[k].y));
        e4m3x8_values(v + 8, make_uint2(c[k].z, c[k].w));
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = e8m0 != nullptr ? v[j] * s[k] : v[j] / s[k];
        T* to = out + row * ldo + at;
        store8(v, to, cols - at, whole);
        store8(v + 8, to + 8, cols - at - 8, whole);
    }
}

// ------------------------------------------------------------------------------------------- host side ----

template <typename T, typename R, int G, int N> cudaError_t norm_launch(const NormParams& p, bool any, cudaStream_t st)
{
    constexpr int kThreads = kForwardThreads<G>, kGroups = kThreads / G;
    constexpr int kSmem = kAhead<T, R, G, N> ? kForwardRing<T, R, N> * kThreads : 0, kFit = 227 * 1024 / (kSmem + 1024), kMost = 1024 / kThreads;      // 64 registers a thread
    static std::atomic<uint64_t> done{0};
    if (!allow_smem(norm_kernel<T, R, G, N, false>, kSmem, done)) return cudaErrorUnknown;
    const int64_t need = ceil_div(p.rows, kGroups), held = kSms * (kFit < kMost ? kFit : kMost);
    const uint32_t grid = (uint32_t)(need < held ? need : held);
    return any ? launch(norm_kernel<T, R, G, N, true>, grid, kThreads, 0, st, true, p)
               : launch(norm_kernel<T, R, G, N, false>, grid, kThreads, need > held ? (size_t)kSmem : 0, st, true, p);
}
template <typename T, typename R> cudaError_t norm_width(const NormParams& p, bool any, cudaStream_t st)
{
    if (p.cols <= 256) return norm_launch<T, R, 32, 1>(p, any, st);
    if (p.cols <= 512) return norm_launch<T, R, 32, 2>(p, any, st);
    if (p.cols <= 1024) return norm_launch<T, R, 32, 4>(p, any, st);
    if (p.cols <= 2048) return norm_launch<T, R, 128, 2>(p, any, st);
    if (p.cols <= 4096) return norm_launch<T, R, 256, 2>(p, any, st);
    if (p.cols <= 8192) return norm_launch<T, R, 512, 2>(p, any, st);
    if (p.cols <= kRowLimit) return norm_launch<T, R, 1024, 2>(p, any, st);
    return launch(norm_wide_kernel<T, R>, (uint32_t)p.rows, kWideThreads, 0, st, false, p);
}

int grad_groups(int64_t cols) { return cols <= 512 ? 16 : cols <= 1024 ? 8 : cols <= 2048 ? 4 : cols <= 4096 ? 2 : 1; }
int64_t grad_ctas(int64_t rows, int64_t cols)
{
    const int64_t need = ceil_div(rows, grad_groups(cols));
    return need < kSms ? need : kSms;
}

template <typename T, typename R, int G, int N> cudaError_t grad_launch(const NormParams& p, uint32_t grid, bool any, cudaStream_t st)
{
    constexpr int kThreads = kGradThreads<G>, kGroups = kThreads / G;
    const size_t sums = kGroups > 1 ? (size_t)p.cols * 4 : 0, ring = (size_t)kGradRing<T, R, N> * kThreads;
    static std::atomic<uint64_t> done{0};
    if (!allow_smem(norm_grad_kernel<T, R, G, N, false>, (int)ring, done)) return cudaErrorUnknown;
    const size_t smem = !any && p.rows > (int64_t)grid * kGroups && ring > sums ? ring : sums;
    return any ? launch(norm_grad_kernel<T, R, G, N, true>, grid, kThreads, smem, st, true, p)
               : launch(norm_grad_kernel<T, R, G, N, false>, grid, kThreads, smem, st, true, p);
}
template <typename T, typename R> cudaError_t grad_width(const NormParams& p, uint32_t grid, bool any, cudaStream_t st)
{
    if (p.cols <= 256) return grad_launch<T, R, 32, 1>(p, grid, any, st);
    if (p.cols <= 512) return grad_launch<T, R, 32, 2>(p, grid, any, st);
    if (p.cols <= 1024) return grad_launch<T, R, 64, 2>(p, grid, any, st);
    if (p.cols <= 2048) return grad_launch<T, R, 128, 2>(p, grid, any, st);
    if (p.cols <= 4096) return grad_launch<T, R, 256, 2>(p, grid, any, st);
    if (p.cols <= 8192) return grad_launch<T, R, 512, 2>(p, grid, any, st);
    // beyond, a thread's share of the row and of the weight's gradient no longer fits the registers (1024 threads: 64 each, 280 bytes spilt)
    static std::atomic<uint64_t> done{0};
    if (!allow_smem(norm_grad_wide_kernel<T, R>, kWideSums * 4, done)) return cudaErrorUnknown;
    return launch(norm_grad_wide_kernel<T, R>, grid, kWideThreads, p.partial != nullptr && p.cols <= kWideSums ? (size_t)p.cols * 4 : 0, st, true, p);
}

bool norm_shape_ok(int64_t rows, int64_t cols) { return rows >= 0 && rows < (1ll << 31) && cols >= 0 && cols < (1ll << 31) - 16384; }

// A matrix argument that exists: pitch, element alignment, and whether whole pieces of 8 may be taken.
mor_status_t check_matrix_arg(const void* m, int64_t rows, int64_t cols, int64_t ld, int element, bool& any)
{
    if (ld < cols || (rows > 0 && cols > 0 && m == nullptr)) return MOR_ERR_INVALID_ARG;
    if (!is_aligned(m, element)) return MOR_ERR_ALIGNMENT;
    if (access_bytes(m, rows > 1 ? ld * element : 0, 0, element) < kPer * element) any = true;
    return MOR_OK;
}
mor_status_t check_norm(const mor_norm_desc_t* d)
{
    if (d == nullptr || !norm_shape_ok(d->rows, d->cols) || !is_dtype(d->dtype) || !is_dtype(d->weight_dtype) || !(d->eps >= 0.f) || !(d->eps < INFINITY))
        return MOR_ERR_INVALID_ARG;
    if (d->cols > 0 && d->weight == nullptr) return MOR_ERR_INVALID_ARG;
    return is_aligned(d->weight, dtype_bytes(d->weight_dtype)) ? MOR_OK : MOR_ERR_ALIGNMENT;
}
template <typename F> mor_status_t by_types(int dtype, int other, F&& f)
{
    using B = __nv_bfloat16;
    cudaError_t e;
    if (dtype == MOR_DTYPE_BF16) e = other == MOR_DTYPE_BF16 ? f(B{}, B{}) : f(B{}, float{});
    else e = other == MOR_DTYPE_BF16 ? f(float{}, B{}) : f(float{}, float{});
    return e == cudaSuccess ? MOR_OK : MOR_ERR_CUDA;
}

}  // namespace
}  // namespace mor

using namespace mor;

extern "C" {

mor_status_t mor_rms_norm(const mor_norm_desc_t* d, const mor_norm_outputs_t* o, void* cuda_stream)
{
    mor_status_t s = check_norm(d);
    if (s != MOR_OK) return s;
    if (o == nullptr || (o->block != 0 && o->block != 128)) return MOR_ERR_INVALID_ARG;
    const bool empty = d->rows == 0 || d->cols == 0;
    if (d->residual == nullptr && o->h != nullptr) return MOR_ERR_INVALID_ARG;
    if (d->residual != nullptr && !is_dtype(d->residual_dtype)) return MOR_ERR_INVALID_ARG;
    if (!empty && o->h == nullptr && o->y == nullptr && o->codes == nullptr) return MOR_ERR_INVALID_ARG;
    if (!empty && o->codes != nullptr && (o->scale_e8m0 == nullptr) == (o->scale_f32 == nullptr)) return MOR_ERR_INVALID_ARG;
    const int es = (int)dtype_bytes(d->dtype), rt = d->residual != nullptr ? d->residual_dtype : d->dtype, rs = (int)dtype_bytes(rt);
    bool any = d->cols % kPer != 0;
    if ((s = check_matrix_arg(d->x, d->rows, d->cols, d->ldx, es, any)) != MOR_OK) return s;
    if (d->residual != nullptr && (s = check_matrix_arg(d->residual, d->rows, d->cols, d->ldr, rs, any)) != MOR_OK) return s;
    if (o->h != nullptr && (s = check_matrix_arg(o->h, d->rows, d->cols, o->ldh, rs, any)) != MOR_OK) return s;
    if (o->y != nullptr && (s = check_matrix_arg(o->y, d->rows, d->cols, o->ldy, es, any)) != MOR_OK) return s;
    if (o->codes != nullptr && (s = check_matrix_arg(o->codes, d->rows, d->cols, o->ldc, 1, any)) != MOR_OK) return s;
    if (!is_aligned(o->scale_f32, 4)) return MOR_ERR_ALIGNMENT;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    NormParams p = {};
    p.rows = d->rows;
    if (empty) {                                            // a scale for a row is there without columns too
        if (d->rows == 0 || o->block != 0 || (o->scale_e8m0 == nullptr) == (o->scale_f32 == nullptr)) return MOR_OK;
        p.e8m0 = o->scale_e8m0;
        p.f32 = o->scale_f32;
        const uint32_t grid = (uint32_t)ceil_div(d->rows, 256);
        return launch(norm_no_columns_kernel, grid, 256, 0, st, grid <= kEarlyGrid, p) == cudaSuccess ? MOR_OK : MOR_ERR_CUDA;
    }
    p.cols = (int32_t)d->cols;
    p.weight_dtype = d->weight_dtype;
    p.x = d->x;
    p.r = d->residual;
    p.w = d->weight;
    p.ldx = d->ldx;
    p.ldr = d->ldr;
    p.eps = d->eps;
    p.inv_cols = 1.f / (float)d->cols;
    p.h = o->h;
    p.y = o->y;
    p.codes = o->codes;
    p.e8m0 = o->scale_e8m0;
    p.f32 = o->scale_f32;
    p.ldh = o->ldh;
    p.ldy = o->ldy;
    p.ldc = o->ldc;
    p.by_row = o->block == 0;
    return by_types(d->dtype, rt, [&](auto t, auto r) { return norm_width<decltype(t), decltype(r)>(p, any, st); });
}

size_t mor_rms_norm_grad_workspace_bytes(int64_t rows, int64_t cols)
{
    if (!norm_shape_ok(rows, cols)) return 0;
    return (size_t)grad_ctas(rows, cols) * (size_t)cols * 4;
}

mor_status_t mor_rms_norm_grad(const mor_norm_desc_t* d, int has_residual, const void* dy, int64_t lddy, void* dx, int64_t lddx, void* dr, int64_t lddr,
                               void* dweight, void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    mor_status_t s = check_norm(d);
    if (s != MOR_OK) return s;
    if (has_residual && !is_dtype(d->residual_dtype)) return MOR_ERR_INVALID_ARG;
    const int es = (int)dtype_bytes(d->dtype), rt = has_residual ? d->residual_dtype : d->dtype, rs = (int)dtype_bytes(rt), ws = (int)dtype_bytes(d->weight_dtype);
    if (d->cols > 0 && d->rows > 0 && dx == nullptr && dr == nullptr && dweight == nullptr) return MOR_ERR_INVALID_ARG;
    bool any = d->cols % kPer != 0;
    if ((s = check_matrix_arg(d->x, d->rows, d->cols, d->ldx, rs, any)) != MOR_OK) return s;
    if ((s = check_matrix_arg(dy, d->rows, d->cols, lddy, es, any)) != MOR_OK) return s;
    if (d->residual != nullptr && (s = check_matrix_arg(d->residual, d->rows, d->cols, d->ldr, rs, any)) != MOR_OK) return s;
    if (dx != nullptr && (s = check_matrix_arg(dx, d->rows, d->cols, lddx, es, any)) != MOR_OK) return s;
    if (dr != nullptr && (s = check_matrix_arg(dr, d->rows, d->cols, lddr, rs, any)) != MOR_OK) return s;
    if (!is_aligned(dweight, ws)) return MOR_ERR_ALIGNMENT;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (d->cols == 0) return MOR_OK;
    if (d->rows == 0) {
        if (dweight != nullptr && cudaMemsetAsync(dweight, 0, (size_t)d->cols * ws, st) != cudaSuccess) return MOR_ERR_CUDA;     // sums over nothing
        return MOR_OK;
    }
    if (dweight != nullptr) {
        if (workspace == nullptr || workspace_bytes < mor_rms_norm_grad_workspace_bytes(d->rows, d->cols)) return MOR_ERR_WORKSPACE;
        if (!is_aligned(workspace, 16)) return MOR_ERR_ALIGNMENT;
    }
    NormParams p = {};
    p.rows = d->rows;
    p.cols = (int32_t)d->cols;
    p.weight_dtype = d->weight_dtype;
    p.x = d->x;
    p.r = d->residual;
    p.w = d->weight;
    p.ldx = d->ldx;
    p.ldr = d->ldr;
    p.eps = d->eps;
    p.inv_cols = 1.f / (float)d->cols;
    p.dy = dy;
    p.dx = dx;
    p.dr = dr;
    p.lddy = lddy;
    p.lddx = lddx;
    p.lddr = lddr;
    p.partial = dweight != nullptr ? static_cast<float*>(workspace) : nullptr;
    const uint32_t grid = (uint32_t)grad_ctas(d->rows, d->cols);
    s = by_types(d->dtype, rt, [&](auto t, auto r) { return grad_width<decltype(t), decltype(r)>(p, grid, any, st); });
    if (s != MOR_OK || dweight == nullptr) return s;
    const uint32_t join = (uint32_t)ceil_div(d->cols, kJoinCols);
    const cudaError_t e = ws == 2 ? launch(norm_join_kernel<__nv_bfloat16>, join, kJoinCols * kJoinParts, 0, st, true, p.partial, (int)grid, p.cols, static_cast<__nv_bfloat16*>(dweight))
                                  : launch(norm_join_kernel<float>, join, kJoinCols * kJoinParts, 0, st, true, p.partial, (int)grid, p.cols, static_cast<float*>(dweight));
    return e == cudaSuccess ? MOR_OK : MOR_ERR_CUDA;
}

mor_status_t mor_codes_dequantize(const uint8_t* codes, int64_t rows, int64_t cols, int64_t ldc, int block, const uint8_t* scale_e8m0, const float* scale_f32,
                                  void* out, int dtype, int64_t ldo, void* cuda_stream)
{
    if (!norm_shape_ok(rows, cols) || !is_dtype(dtype) || (block != 0 && block != 128) || ldc < cols || ldo < cols) return MOR_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return MOR_OK;
    if (codes == nullptr || out == nullptr || (scale_e8m0 == nullptr) == (scale_f32 == nullptr)) return MOR_ERR_INVALID_ARG;
    const int es = (int)dtype_bytes(dtype);
    if (!is_aligned(out, es) || !is_aligned(scale_f32, 4)) return MOR_ERR_ALIGNMENT;
    const bool aligned = access_bytes(codes, rows > 1 ? ldc : 0, 0, 1) >= 16 && access_bytes(out, rows > 1 ? ldo * es : 0, 0, es) >= kPer * es;
    const int64_t pieces = ceil_div(cols, 16);
    const uint32_t x = pieces >= 256 ? 256u : (uint32_t)ceil_div(pieces, 32) * 32, y = 256 / x;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((uint32_t)ceil_div(rows, y * kValueRows), (uint32_t)ceil_div(pieces, x));
    if (cfg.gridDim.y > 65535u) return MOR_ERR_INVALID_ARG;
    cfg.blockDim = dim3(x, y);
    cfg.stream = static_cast<cudaStream_t>(cuda_stream);
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = cfg.gridDim.x <= kEarlyGrid ? 1 : 0;
    const cudaError_t e = dtype == MOR_DTYPE_BF16 ? cudaLaunchKernelEx(&cfg, codes_values_kernel<__nv_bfloat16>, codes, rows, (int32_t)cols, ldc, (int32_t)(block == 0),
                                                                       scale_e8m0, scale_f32, static_cast<__nv_bfloat16*>(out), ldo, aligned)
                                                  : cudaLaunchKernelEx(&cfg, codes_values_kernel<float>, codes, rows, (int32_t)cols, ldc, (int32_t)(block == 0), scale_e8m0,
                                                                       scale_f32, static_cast<float*>(out), ldo, aligned);
    return e == cudaSuccess ? MOR_OK : MOR_ERR_CUDA;
}

}  // extern "C"
