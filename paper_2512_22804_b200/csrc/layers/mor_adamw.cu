// One AdamW step over many tensors, moments in 32 bits or as E4M3 codes with one scale for 128 elements, and the values of such codes.
//
// Every element is read and written once: the kernel is bound by memory.  A launch takes the addresses of up to 512 tensors as its
// parameters (a captured graph then needs no table in memory that has to outlive it), the smallest of three sizes of that table that holds them,
// since a launch costs more the more it carries; each CTA finds its tensor by bisection and takes 4096 of its elements.
// A thread holds 8 consecutive elements, so 16 lanes hold a block of 128 and its maximum takes four shuffles.
#include <math.h>

#include "mor_layers.cuh"

namespace mor {
namespace {

constexpr int kThreads = 256;
constexpr int kPass = kThreads * kPer;
constexpr int kChunk = 2 * kPass;             // elements of a CTA

struct AdamwEntry {
    void* param;
    const void* grad;
    void *m, *v;
    uint8_t* scales;
    int64_t numel;
    uint32_t first;            // first CTA
    uint32_t aligned;          // whole pieces may be read and written
};

struct AdamwScalars {
    float lr, beta1, beta2, rest1, rest2, eps, decay;      // rest: 1 - beta; decay: weight decay
    float bias1, bias2;                                    // 1 / (1 - beta1^step), 1 / sqrt(1 - beta2^step)
    float log1, log2;                                      // log beta
    uint32_t seed, step, number, count;                    // number: of the first tensor in the call; count: tensors of this launch
    const int32_t* device_step;
    const float *device_lr, *grad_scale, *found_inf;
};

template <int N> struct AdamwParams {
    AdamwScalars s;
    AdamwEntry e[N];
};

__host__ __device__ __forceinline__ uint32_t mix(uint32_t z)
{
    z ^= z >> 16;
    z *= 0x7FEB352Du;
    z ^= z >> 15;
    z *= 0x846CA68Bu;
    return z ^ (z >> 16);
}

// Largest magnitude of a block of 128: of 16 lanes with 8 elements each; NaN if any is NaN.  Where the result is not finite, that of the finite ones is
// taken with a second look (a check per element would cost every block what few need).
__device__ __forceinline__ float block_amax(const float* v)
{
    float a = amax_of<kPer>(v);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) a = max_nan(a, __shfl_xor_sync(0xFFFFFFFFu, a, o));
    return a;
}
__device__ __noinline__ float block_amax_finite(float a)          // of this lane's largest finite magnitude
{
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, o));
    return a;
}
__device__ __forceinline__ float largest_finite(const float* v)
{
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) a = fmaxf(a, fabsf(v[i]) < INFINITY ? fabsf(v[i]) : 0.f);
    return a;
}

// Between its neighbours among the E4M3 values a magnitude w <= 448 has 20 fraction bits below the three that are kept, if it is a normal one (2^-6 and up).
// Below, the distance stays that of 2^-6: with 2^-6 added the bits lie the same way (and the sum is off by 2^-21 of a distance at most).
// Up where t + u >= n + 1: the random bits are added below the kept ones and what is below is cut off.
__device__ __forceinline__ float round_mean(float w, uint32_t z)
{
    const float off = fabsf(w) < 0x1p-6f ? copysignf(0x1p-6f, w) : 0.f;
    return __uint_as_float((__float_as_uint(w + off) + (z << 16 >> 12)) & 0xFFF00000u) - off;
}
// Of a w that is not negative.  Up where u (2 n + 1) < (t - n)(t + n), all of it times the distance's square; never zero above zero.
__device__ __forceinline__ float round_square_mean(float w, uint32_t z)
{
    const float off = w < 0x1p-6f ? 0x1p-6f : 0.f, s = w + off;
    const float lo = __uint_as_float(__float_as_uint(s) & 0xFFF00000u) - off, d = __uint_as_float(__float_as_uint(s) & 0x7F800000u) * 0.125f;
    const float u = __uint_as_float(0x3F800000u | (z >> 16 << 7)) - 1.f;
    const float q = u * d * fmaf(2.f, lo, d) < (w - lo) * (w + lo) ? lo + d : lo;
    return fmaxf(q, w > 0.f ? 0x1p-9f : 0.f);
}
// One instruction each, within 2 units of the last place: far below what a step is worth.  A second moment below 2^-126 counts as zero, and what is divided by
// is at least the root of that.
__device__ __forceinline__ float root_of(float v)
{
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float quotient(float m, float d)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(fmaxf(d, 0x1p-63f)));
    return m * r;
}

template <typename P, typename G, bool EIGHT, int N> __global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ AdamwParams<N> p)
{
    wait_for_predecessor();
    const AdamwScalars& s = p.s;
    if (s.found_inf != nullptr && !(*s.found_inf == 0.f)) return;
    uint32_t lo = 0, hi = s.count;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (p.e[mid].first <= blockIdx.x) lo = mid;
        else hi = mid;
    }
    const AdamwEntry& e = p.e[lo];
    float lr = s.lr, bias1 = s.bias1, bias2 = s.bias2;
    uint32_t step = s.step;
    if (s.device_lr != nullptr) lr = *s.device_lr;
    if (s.device_step != nullptr) {
        step = (uint32_t)*s.device_step;
        bias1 = 1.f / -expm1f((float)step * s.log1);
        bias2 = rsqrtf(-expm1f((float)step * s.log2));
    }
    const float scale = s.grad_scale != nullptr ? *s.grad_scale : 1.f;
    const float keep = fmaf(-lr, s.decay, 1.f), rate = lr * bias1;
    const uint32_t key = mix(mix(s.seed + 0x9E3779B9u * step) + s.number + lo);
    const int64_t begin = (int64_t)(blockIdx.x - e.first) * kChunk;
    const bool aligned = e.aligned != 0;
#pragma unroll 1
    for (int pass = 0; pass < kChunk / kPass; ++pass) {
        const int64_t at = begin + pass * kPass + threadIdx.x * kPer;
        if (begin + pass * kPass >= e.numel) return;                 // the same for all threads
        const int left = (int)min((int64_t)kPer, e.numel - at);     // may be negative: nothing of the thread's exists
        const bool whole = aligned && left == kPer;
        float w[kPer], g[kPer], m[kPer], v[kPer];
        load8(g, static_cast<const G*>(e.grad) + at, left, whole);
        load8(w, static_cast<const P*>(e.param) + at, left, whole);
        if constexpr (EIGHT) {
            const uint2 cm = load_codes(static_cast<const uint8_t*>(e.m) + at, left, whole), cv = load_codes(static_cast<const uint8_t*>(e.v) + at, left, whole);
            const uint32_t sc = left > 0 ? *reinterpret_cast<const uint16_t*>(e.scales + at / 128 * 2) : 0x7F7Fu;
            const float sm = inverse_power(sc & 255u), sv = inverse_power(sc >> 8);
            e4m3x8_values(m, cm);
            e4m3x8_values(v, cv);
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                m[i] *= sm;
                v[i] *= sv;
                v[i] *= v[i];
            }
        } else {
            load8(m, static_cast<const float*>(e.m) + at, left, whole);
            load8(v, static_cast<const float*>(e.v) + at, left, whole);
        }
        float root[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const float x = g[i] * scale;
            m[i] = fmaf(s.rest1, x, s.beta1 * m[i]);
            v[i] = fmaf(s.rest2 * x, x, s.beta2 * v[i]);
            root[i] = root_of(v[i]);
            w[i] = fmaf(-rate, quotient(m[i], fmaf(root[i], bias2, s.eps)), w[i] * keep);
        }
        const uint32_t high = mix((uint32_t)((uint64_t)at >> 32) ^ key);
        uint32_t z[kPer];
        if constexpr (EIGHT || sizeof(P) == 2)
#pragma unroll
            for (int i = 0; i < kPer; ++i) z[i] = mix(high + (uint32_t)at + i);
        if constexpr (sizeof(P) == 2) {
            // NaN, whose bits may all be set, must not be carried into the sign
            const bool any_nan = !(amax_of<kPer>(w) <= INFINITY);
            uint32_t b[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i) b[i] = __float_as_uint(w[i]) + (mix(z[i] ^ 0x9E3779B9u) & 0xFFFFu);
            if (any_nan)
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (isnan(w[i])) b[i] = 0x7FC00000u;
            if (whole) {
                *reinterpret_cast<uint4*>(static_cast<P*>(e.param) + at) =
                    make_uint4(__byte_perm(b[0], b[1], 0x7632), __byte_perm(b[2], b[3], 0x7632), __byte_perm(b[4], b[5], 0x7632), __byte_perm(b[6], b[7], 0x7632));
            } else {
#pragma unroll
                for (int i = 0; i < kPer; ++i) w[i] = __uint_as_float(b[i] & 0xFFFF0000u);
                store8(w, static_cast<P*>(e.param) + at, left, false);
            }
        } else {
            store8(w, static_cast<P*>(e.param) + at, left, whole);
        }
        if constexpr (EIGHT) {
            float am = block_amax(m), av = block_amax(root);
            const bool finite = am < INFINITY && av < INFINITY;
            if (__any_sync(0xFFFFFFFFu, !finite)) {
                am = block_amax_finite(largest_finite(m));
                av = block_amax_finite(largest_finite(root));
            }
            const uint32_t em = power_scale(am, 253u), ev = power_scale(av, 253u);
            const float sm = __uint_as_float(em << 23), sv = __uint_as_float(ev << 23);
            uint32_t bad = 0;                                         // elements that are not finite
            if (!finite)
#pragma unroll
                for (int i = 0; i < kPer; ++i) bad |= (fabsf(m[i]) < INFINITY ? 0u : 1u << i) | (root[i] < INFINITY ? 0u : 256u << i);
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                m[i] = round_mean(m[i] * sm, z[i]);
                v[i] = round_square_mean(root[i] * sv, z[i]);
            }
            if (bad != 0)
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    if (bad >> i & 1) m[i] = NAN;
                    if (bad >> (8 + i) & 1) v[i] = NAN;
                }
            store_codes(e4m3x8(m), static_cast<uint8_t*>(e.m) + at, left, whole);
            store_codes(e4m3x8(v), static_cast<uint8_t*>(e.v) + at, left, whole);
            if (left > 0 && (threadIdx.x & 15) == 0) *reinterpret_cast<uint16_t*>(e.scales + at / 128 * 2) = (uint16_t)(em | ev << 8);
        } else {
            store8(m, static_cast<float*>(e.m) + at, left, whole);
            store8(v, static_cast<float*>(e.v) + at, left, whole);
        }
    }
}

template <typename T> __global__ void __launch_bounds__(kThreads) moments_kernel(const uint8_t* m, const uint8_t* v, const uint8_t* scales, int64_t numel, T* m_out,
                                                                                T* v_out, bool aligned)
{
    wait_for_predecessor();
    const int64_t at = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kPer;
    if (at >= numel) return;
    const int left = (int)min((int64_t)kPer, numel - at);
    const bool whole = aligned && left == kPer;
    const uint32_t sc = *reinterpret_cast<const uint16_t*>(scales + at / 128 * 2);
    uint2 cm = make_uint2(0, 0), cv = cm;
    if (m_out != nullptr) cm = load_codes(m + at, left, whole);
    if (v_out != nullptr) cv = load_codes(v + at, left, whole);
    float x[kPer];
    if (m_out != nullptr) {
        const float s = inverse_power(sc & 255u);
        e4m3x8_values(x, cm);
#pragma unroll
        for (int i = 0; i < kPer; ++i) x[i] *= s;
        store8(x, m_out + at, left, whole);
    }
    if (v_out != nullptr) {
        const float s = inverse_power(sc >> 8);
        e4m3x8_values(x, cv);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            x[i] *= s;
            x[i] *= x[i];
        }
        store8(x, v_out + at, left, whole);
    }
}

template <typename P, typename G, bool EIGHT, int N>
mor_status_t adamw_launch(const AdamwScalars& s, const mor_adamw_tensor_t* t, int n, cudaStream_t st)
{
    AdamwParams<N> p;
    p.s = s;
    int at = 0;
    while (at < n) {
        int64_t ctas = 0;
        int k = 0;
        p.s.number = s.number + (uint32_t)at;
        for (; at < n && k < N; ++at) {
            const mor_adamw_tensor_t& x = t[at];
            const int64_t need = ceil_div(x.numel, kChunk);
            if (need >= (1ll << 31)) return MOR_ERR_INVALID_ARG;      // checked before the first launch: not reached
            if (k > 0 && ctas + need >= (1ll << 31)) break;
            AdamwEntry& e = p.e[k++];
            const size_t state = EIGHT ? 8 : 32;
            e = {x.param, x.grad, x.exp_avg, x.exp_avg_sq, x.scales, x.numel, (uint32_t)ctas,
                 (uint32_t)(is_aligned(x.param, kPer * sizeof(P)) && is_aligned(x.grad, kPer * sizeof(G)) && is_aligned(x.exp_avg, state) && is_aligned(x.exp_avg_sq, state))};
            ctas += need;
        }
        p.s.count = (uint32_t)k;
        if (ctas == 0) continue;
        if (launch(adamw_kernel<P, G, EIGHT, N>, (uint32_t)ctas, kThreads, 0, st, ctas <= kEarlyGrid, p) != cudaSuccess) return MOR_ERR_CUDA;
    }
    return MOR_OK;
}
template <typename P, typename G, bool EIGHT> mor_status_t adamw_table(const AdamwScalars& s, const mor_adamw_tensor_t* t, int n, cudaStream_t st)
{
    if (n <= 16) return adamw_launch<P, G, EIGHT, 16>(s, t, n, st);
    if (n <= 128) return adamw_launch<P, G, EIGHT, 128>(s, t, n, st);
    return adamw_launch<P, G, EIGHT, 512>(s, t, n, st);
}
template <typename P, typename G> mor_status_t adamw_state(bool eight, const AdamwScalars& s, const mor_adamw_tensor_t* t, int n, cudaStream_t st)
{
    return eight ? adamw_table<P, G, true>(s, t, n, st) : adamw_table<P, G, false>(s, t, n, st);
}

bool in_unit(double v) { return v >= 0.0 && v < 1.0; }

}  // namespace
}  // namespace mor

using namespace mor;

extern "C" {

mor_status_t mor_adamw(const mor_adamw_desc_t* d, const mor_adamw_tensor_t* t, int n, void* cuda_stream)
{
    if (d == nullptr || n < 0 || (n > 0 && t == nullptr) || !is_dtype(d->param_dtype) || !is_dtype(d->grad_dtype)) return MOR_ERR_INVALID_ARG;
    if (!(d->lr >= 0.0 && d->lr < 1e30) || !in_unit(d->beta1) || !in_unit(d->beta2) || !(d->eps >= 0.0 && d->eps < 1e30) ||
        !(d->weight_decay >= 0.0 && d->weight_decay < 1e30))
        return MOR_ERR_INVALID_ARG;
    if (d->device_step == nullptr && d->step < 1) return MOR_ERR_INVALID_ARG;
    if (!is_aligned(d->device_step, 4) || !is_aligned(d->device_lr, 4) || !is_aligned(d->grad_scale, 4) || !is_aligned(d->found_inf, 4)) return MOR_ERR_ALIGNMENT;
    const size_t state = d->eight_bits ? 1 : 4;
    for (int i = 0; i < n; ++i) {
        const mor_adamw_tensor_t& x = t[i];
        if (x.numel < 0 || x.numel >= (1ll << 40)) return MOR_ERR_INVALID_ARG;
        if (x.numel == 0) continue;
        if (x.param == nullptr || x.grad == nullptr || x.exp_avg == nullptr || x.exp_avg_sq == nullptr || (d->eight_bits && x.scales == nullptr)) return MOR_ERR_INVALID_ARG;
        if (!is_aligned(x.param, dtype_bytes(d->param_dtype)) || !is_aligned(x.grad, dtype_bytes(d->grad_dtype)) || !is_aligned(x.exp_avg, state) ||
            !is_aligned(x.exp_avg_sq, state) || (d->eight_bits && !is_aligned(x.scales, 2)))
            return MOR_ERR_ALIGNMENT;
    }
    AdamwScalars s = {};
    s.lr = (float)d->lr;
    s.beta1 = (float)d->beta1;
    s.beta2 = (float)d->beta2;
    s.rest1 = (float)(1.0 - d->beta1);
    s.rest2 = (float)(1.0 - d->beta2);
    s.eps = (float)d->eps;
    s.decay = (float)d->weight_decay;
    s.bias1 = (float)(1.0 / (1.0 - pow(d->beta1, (double)d->step)));
    s.bias2 = (float)(1.0 / sqrt(1.0 - pow(d->beta2, (double)d->step)));
    s.log1 = (float)log(d->beta1);                                   // beta 0: -infinity, and 1 - beta^step is 1
    s.log2 = (float)log(d->beta2);
    s.seed = (uint32_t)d->seed;
    s.step = (uint32_t)d->step;
    s.device_step = d->device_step;
    s.device_lr = d->device_lr;
    s.grad_scale = d->grad_scale;
    s.found_inf = d->found_inf;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const bool eight = d->eight_bits != 0, g16 = d->grad_dtype == MOR_DTYPE_BF16;
    if (d->param_dtype == MOR_DTYPE_BF16)
        return g16 ? adamw_state<__nv_bfloat16, __nv_bfloat16>(eight, s, t, n, st) : adamw_state<__nv_bfloat16, float>(eight, s, t, n, st);
    return g16 ? adamw_state<float, __nv_bfloat16>(eight, s, t, n, st) : adamw_state<float, float>(eight, s, t, n, st);
}

mor_status_t mor_adamw_moments(const uint8_t* exp_avg, const uint8_t* exp_avg_sq, const uint8_t* scales, int64_t numel, void* exp_avg_out, void* exp_avg_sq_out,
                               int dtype, void* cuda_stream)
{
    if (numel < 0 || numel >= (1ll << 40) || !is_dtype(dtype)) return MOR_ERR_INVALID_ARG;
    if (numel == 0) return MOR_OK;
    if (scales == nullptr || (exp_avg_out != nullptr && exp_avg == nullptr) || (exp_avg_sq_out != nullptr && exp_avg_sq == nullptr)) return MOR_ERR_INVALID_ARG;
    if (exp_avg_out == nullptr && exp_avg_sq_out == nullptr) return MOR_ERR_INVALID_ARG;
    const size_t es = dtype_bytes(dtype);
    if (!is_aligned(scales, 2) || !is_aligned(exp_avg_out, es) || !is_aligned(exp_avg_sq_out, es)) return MOR_ERR_ALIGNMENT;
    const bool aligned = is_aligned(exp_avg, 8) && is_aligned(exp_avg_sq, 8) && is_aligned(exp_avg_out, kPer * es) && is_aligned(exp_avg_sq_out, kPer * es);
    const int64_t grid = ceil_div(numel, kPass);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = dtype == MOR_DTYPE_BF16
                              ? launch(moments_kernel<__nv_bfloat16>, (uint32_t)grid, kThreads, 0, st, grid <= kEarlyGrid, exp_avg, exp_avg_sq, scales, numel,
                                       static_cast<__nv_bfloat16*>(exp_avg_out), static_cast<__nv_bfloat16*>(exp_avg_sq_out), aligned)
                              : launch(moments_kernel<float>, (uint32_t)grid, kThreads, 0, st, grid <= kEarlyGrid, exp_avg, exp_avg_sq, scales, numel,
                                       static_cast<float*>(exp_avg_out), static_cast<float*>(exp_avg_sq_out), aligned);
    return e == cudaSuccess ? MOR_OK : MOR_ERR_CUDA;
}

}  // extern "C"
