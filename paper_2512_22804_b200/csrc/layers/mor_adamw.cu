// One AdamW step over many tensors, moments in 32 bits or as E4M3 codes with one scale for 128 elements, and the values of such codes.
//
// Every element is read and written once.  With FP32 moments the kernel is bound by memory (103 M elements, 2.88 GB: 421 us, 6.8 TB/s), with 8-bit ones by its
// instructions (84 an element: 285-289 us for 1.44 GB; with the read-back of the moments' values 411-421, of which about 8 are the sums and roots that are
// rounded as formulas without fused operations round them).  A launch takes the addresses of up to 512 tensors as its
// parameters (a captured graph then needs no table in memory that has to outlive it), the smallest of three sizes of that table that holds them,
// since a launch costs the host more the more it carries (tensors of 4096 elements: 16 take a call 4.5 us, 17 5.8; 128 17.2, 129 18.7; on the GPU there is
// no difference, 4.1 and 6.2 us as graphs on either side); each CTA finds its tensor by bisection and takes 2048 or 4096 of its elements.
// A thread holds 8 consecutive elements, so 16 lanes hold a block of 128 and its maximum takes four shuffles.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "mor_layers.cuh"

namespace mor {
namespace {

constexpr int kThreads = 256;
constexpr int kPass = kThreads * kPer;
constexpr int kMostPasses = 2;                // of a CTA (1: 427 us for a layer of 103 M elements and its moments' values, 2: 411-421, 4: 449)
constexpr int kRing = 2;                      // passes whose inputs a thread has in its part of shared memory

struct AdamwEntry {
    void* param;
    const void* grad;
    void *m, *v;
    uint8_t* scales;
    int64_t numel;
    uint32_t first;            // first CTA
    uint32_t number_aligned;   // twice the tensor's number, and whether whole pieces may be read and written
};

struct AdamwScalars {
    float lr, beta1, beta2, rest1, rest2, eps, decay;      // rest: 1 - beta; decay: weight decay
    float one;                                             // 1
    float bias1, bias2;                                    // 1 / (1 - beta1^step), 1 / sqrt(1 - beta2^step)
    float log1, log2;                                      // log beta
    uint32_t seed, step, count;                            // count: tensors of this launch
    int32_t chunk;                                         // elements of a CTA
    uint32_t each;                                         // tensors' steps apart in device_step: 1, or 0 if they share one
    const int32_t* device_step;
    const float *device_lr, *grad_scale, *found_inf;
};

template <int N> struct AdamwParams {
    AdamwScalars s;
    AdamwEntry e[N];
};

// A published hash of 32 bits (C. Wellons, "Prospecting for hash functions", 2018, in the public domain); all of mix() but its last step.
__device__ __forceinline__ uint32_t mix_most(uint32_t z)
{
    z ^= z >> 16;
    z *= 0x7FEB352Du;
    z ^= z >> 15;
    return z * 0x846CA68Bu;
}
__device__ __forceinline__ uint32_t mix(uint32_t z)
{
    z = mix_most(z);
    return z ^ (z >> 16);
}

// The kernel with 8-bit moments has to make some eighty instructions an element fit beside 14 bytes of traffic.  Two things help: operations on two values in
// a register pair, and steps written as saturating products where a comparison and a choice would go to the integer pipe, which is half as wide and was
// what bounded the kernel (38 of 80 instructions an element; a layer of 103 M elements 322 us).
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair(float lo, float hi)
{
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ Pair both(float v) { return pair(v, v); }
__device__ __forceinline__ void apart(Pair p, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p)); }
__device__ __forceinline__ Pair mul(Pair a, Pair b)
{
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair add(Pair a, Pair b)
{
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair fma(Pair a, Pair b, Pair c)
{
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

__device__ __forceinline__ Pair fma_cut(Pair a, Pair b, Pair c)
{
    Pair r;
    asm("fma.rz.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// What power_scale() needs of a magnitude, as a whole number that grows with it (a 16-bit one, above 254 for what is not finite), so that the maxima of both
// moments of a block of 128 take one exchange: 16 lanes with 8 elements each.
__device__ __forceinline__ uint32_t rank_of(float a) { return (__float_as_uint(a) + 0x1FFFFFu) >> 23; }
__device__ __forceinline__ uint32_t block_ranks(float m, float root)
{
    uint32_t r = rank_of(m) | rank_of(root) << 16;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) r = __vmaxu2(r, __shfl_xor_sync(0xFFFFFFFFu, r, o));
    return r;
}
// power_scale() of a maximum's rank; zero (and what is far below 2^-126) has the ranks 0 and below.
__device__ __forceinline__ uint32_t scale_of_rank(uint32_t rank, bool zero) { return zero ? 127u : min(262u - rank, 253u); }
// Largest magnitude, NaN if any is.
__device__ __forceinline__ float max3_nan(float a, float b, float c)
{
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float amax8(const float* v) { return max3_nan(max3_nan(v[0], v[1], v[2]), max3_nan(v[3], v[4], v[5]), max3_nan(v[6], v[7], v[6])); }
__device__ __forceinline__ float largest_finite(const float* v)
{
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) a = fmaxf(a, fabsf(v[i]) < INFINITY ? fabsf(v[i]) : 0.f);
    return a;
}

// Between its neighbours among the E4M3 values a magnitude w <= 448 has 20 fraction bits below the three that are kept, if it is a normal one (2^-6 and up).
// Below, the distance stays that of 2^-6: with 2^-6 added the bits lie the same way (what is cut off there lies below the 16 random bits).  Where w is below, 2^30
// times the (exact) difference is at least 1, and for squares 2^37 times theirs.
// Up where t + u >= n + 1: the random bits (16 of them) are added below the kept ones and what is below is cut off.
__device__ __forceinline__ Pair round_mean(Pair w, uint32_t r0, uint32_t r1)
{
    float w0, w1, x0, x1, s0, s1;
    apart(w, w0, w1);
    apart(mul(w, w), x0, x1);
    const Pair below = pair(copysignf(__saturatef(fmaf(x0, -0x1p37f, 0x1p25f)), w0), copysignf(__saturatef(fmaf(x1, -0x1p37f, 0x1p25f)), w1));
    apart(fma_cut(below, both(0x1p-6f), w), s0, s1);
    s0 = __uint_as_float((r0 * 16u + __float_as_uint(s0)) & 0xFFF00000u);
    s1 = __uint_as_float((r1 * 16u + __float_as_uint(s1)) & 0xFFF00000u);
    return fma(below, both(-0x1p-6f), pair(s0, s1));
}
// Of a w that is not negative.  Up where u (2 n + 1) < (t - n)(t + n), all of it times the distance's square; from zero always, if w is above it.
__device__ __forceinline__ Pair round_square_mean(Pair w, uint32_t r0, uint32_t r1)
{
    float w0, w1, s0, s1, n0, n1, l0, l1, c0, c1;
    apart(w, w0, w1);
    const Pair below = pair(__saturatef(fmaf(w0, -0x1p30f, 0x1p24f)), __saturatef(fmaf(w1, -0x1p30f, 0x1p24f)));
    const Pair s = fma_cut(below, both(0x1p-6f), w);
    apart(s, s0, s1);
    const uint32_t b0 = __float_as_uint(s0), b1 = __float_as_uint(s1);
    const Pair kept = pair(__uint_as_float(b0 & 0xFFF00000u), __uint_as_float(b1 & 0xFFF00000u));
    const Pair lo = fma(below, both(-0x1p-6f), kept), f = fma(lo, both(-1.f), w);                                    // w is lo + f, exactly
    apart(lo, n0, n1);
    const Pair d = mul(pair(__uint_as_float(b0 & 0x7F800000u), __uint_as_float(b1 & 0x7F800000u)), both(0.125f));
    // From lo > 0 both sides are 2^-60 or more apart, or the same: 2^100 times the difference is 0 or at least 1.  From lo = 0 the random side is 0 and the other
    // one w (w + 2^20) instead of w^2: a root is 2^-63 at least (or 0) and a scale that of a maximum below 2^64, so w is 2^-120 at least and 2^100 times this at least 1.
    const Pair some = pair(__saturatef(n0 * 0x1p10f), __saturatef(n1 * 0x1p10f));                                     // 0 from lo = 0, else 1
    const Pair a = mul(mul(d, some), fma(both(2.f), lo, d)), c = mul(f, fma(both(2.f), lo, add(f, fma(some, both(-0x1p20f), both(0x1p20f)))));
    const Pair u = add(pair(__uint_as_float(r0 * 128u + 0x3F800000u), __uint_as_float(r1 * 128u + 0x3F800000u)), both(-1.f));
    apart(mul(mul(u, both(-0x1p100f)), a), l0, l1);
    apart(c, c0, c1);
    const Pair up = pair(__saturatef(fmaf(c0, 0x1p100f, l0)), __saturatef(fmaf(c1, 0x1p100f, l1)));
    return fma(up, d, lo);
}
// One instruction each, within 2 units of the last place: far below what a step is worth.  A second moment below 2^-126 counts as zero; eps is at least the
// root of that, so that nothing is divided by zero.
__device__ __forceinline__ Pair about_root_of(Pair v)
{
    float v0, v1, r0, r1;
    apart(v, v0, v1);
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(v0));
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(v1));
    return pair(r0, r1);
}
// With Newton's step, r + (v - r^2) / 2 r, for roots that become codes: one unit off, and of 103 M elements some twenty were rounded to the other neighbour.  The
// quotient needs a digit only, so 1 / 2 r is read off r's exponent and fraction (within a tenth).  An infinite root's remainder is NaN and counts as anything finite.
__device__ __forceinline__ Pair root_of(Pair v)
{
    const Pair r = about_root_of(v);
    float r0, r1, e0, e1;
    apart(r, r0, r1);
    Pair e;
    asm("fma.rn.ftz.f32x2 %0, %1, %2, %3;" : "=l"(e) : "l"(mul(r, both(-1.f))), "l"(r), "l"(v));
    apart(e, e0, e1);
    const Pair half = pair(__uint_as_float(0x7E740000u - __float_as_uint(r0)), __uint_as_float(0x7E740000u - __float_as_uint(r1)));
    return fma(pair(fmaxf(e0, -0x1p127f), fmaxf(e1, -0x1p127f)), half, r);
}
__device__ __forceinline__ float reciprocal(float d)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d));
    return r;
}

// With 8-bit moments a thread's inputs of the next passes come by asynchronous copies into its own part of shared memory, which asks for no barrier: held in
// registers they left room for too few threads (64 registers and no copies ahead: 437 us for 103 M elements, 48 and spills: 415).
template <typename P, typename G> struct OwnRing {
    static constexpr int kP = kPer * (int)sizeof(P) / 16, kG = kPer * (int)sizeof(G) / 16;         // 16-byte pieces
    static constexpr int kStage = kThreads * (kP * 16 + kG * 16 + 16);
    static constexpr int kBytes = kRing * kStage;
    uint32_t at;
    __device__ __forceinline__ uint32_t stage(int i) const { return at + (uint32_t)(i % kRing) * kStage; }
    static __device__ __forceinline__ void copy16(uint32_t to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); }
    static __device__ __forceinline__ void copy8(uint32_t to, const void* from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory"); }
    __device__ __forceinline__ void fetch(int i, const P* p, const G* g, const uint8_t* m, const uint8_t* v) const
    {
        uint32_t to = stage(i) + threadIdx.x * 16;
#pragma unroll
        for (int k = 0; k < kP; ++k, to += kThreads * 16) copy16(to, reinterpret_cast<const uint4*>(p) + k);
#pragma unroll
        for (int k = 0; k < kG; ++k, to += kThreads * 16) copy16(to, reinterpret_cast<const uint4*>(g) + k);
        copy8(to, m);
        copy8(to + 8, v);
    }
    template <typename T> static __device__ __forceinline__ void words(float* v, uint32_t from)
    {
        Piece<T, kPer * (int)sizeof(T)> piece;
#pragma unroll
        for (int k = 0; k < kPer * (int)sizeof(T) / 16; ++k, from += kThreads * 16)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(piece.w[4 * k]), "=r"(piece.w[4 * k + 1]), "=r"(piece.w[4 * k + 2]), "=r"(piece.w[4 * k + 3]) : "r"(from) : "memory");
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] = piece.get(i);
    }
    __device__ __forceinline__ void take(int i, float* p, float* g, uint2& m, uint2& v) const
    {
        const uint32_t from = stage(i) + threadIdx.x * 16;
        words<P>(p, from);
        words<G>(g, from + kP * kThreads * 16);
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(m.x), "=r"(m.y), "=r"(v.x), "=r"(v.y) : "r"(from + (kP + kG) * kThreads * 16) : "memory");
    }
};

template <typename P, typename G, bool EIGHT, int N> __global__ void __launch_bounds__(kThreads, EIGHT ? 4 : 1) adamw_kernel(const __grid_constant__ AdamwParams<N> p)
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
        step = (uint32_t)s.device_step[lo * s.each];
        bias1 = 1.f / -expm1f((float)step * s.log1);
        bias2 = rsqrtf(-expm1f((float)step * s.log2));
    }
    const float scale = s.grad_scale != nullptr ? *s.grad_scale : 1.f;
    const float keep = fmaf(-lr, s.decay, 1.f), rate = lr * bias1;
    const uint32_t key = mix(mix(s.seed + 0x9E3779B9u * step) + (e.number_aligned >> 1));
    // from here on everything is counted from the CTA's first element
    const int64_t begin = (int64_t)(blockIdx.x - e.first) * s.chunk;
    const int count = (int)min((int64_t)s.chunk, e.numel - begin);
    const bool aligned = (e.number_aligned & 1u) != 0;
    P* const param = static_cast<P*>(e.param) + begin;
    const G* const grad = static_cast<const G*>(e.grad) + begin;
    using M = std::conditional_t<EIGHT, uint8_t, float>;
    M *const em = static_cast<M*>(e.m) + begin, *const ev = static_cast<M*>(e.v) + begin;
    uint8_t* const scales = EIGHT ? e.scales + begin / 64 : nullptr;
    const Pair one = both(s.one), beta1 = both(s.beta1), beta2 = both(s.beta2), rest1 = both(s.rest1), rest2 = both(s.rest2);
    // whole passes of an aligned tensor are copied ahead
    const int ahead = EIGHT && aligned ? count / kPass : 0;
    extern __shared__ __align__(16) uint8_t own[];
    OwnRing<P, G> ring;
    auto fetch = [&](int i) {
        if constexpr (EIGHT) {
            const int at = i * kPass + (int)threadIdx.x * kPer;
            if (i < ahead) ring.fetch(i, param + at, grad + at, em + at, ev + at);
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    uint32_t next = 0x7F7Fu;                                          // the next pass's scales
    auto look = [&](int i) {
        const int at = i * kPass + (int)threadIdx.x * kPer;
        if (at < count) next = *reinterpret_cast<const uint16_t*>(scales + at / 128 * 2);
    };
    if constexpr (EIGHT) {
        look(0);
        ring.at = (uint32_t)__cvta_generic_to_shared(own);
#pragma unroll
        for (int i = 0; i < kRing - 1; ++i) fetch(i);
    }
#pragma unroll 1
    for (int i0 = 0; i0 * kPass < count; ++i0) {
        const int at = i0 * kPass + (int)threadIdx.x * kPer, left = count - at;       // not above 0: nothing of the thread's exists
        const bool whole = aligned && left >= kPer;
        float w[kPer], x[kPer];
        Pair g[kPer / 2], m[kPer / 2], v[kPer / 2];
        if constexpr (EIGHT) {
            uint2 cm, cv;
            const uint32_t sc = next;
            look(i0 + 1);
            fetch(i0 + kRing - 1);
            if (i0 < ahead) {
                asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
                ring.take(i0, w, x, cm, cv);
            } else {
                load8(x, grad + at, left, whole);
                load8(w, param + at, left, whole);
                cm = load_codes(em + at, left, whole);
                cv = load_codes(ev + at, left, whole);
            }
#pragma unroll
            for (int i = 0; i < kPer / 2; ++i) g[i] = pair(x[2 * i], x[2 * i + 1]);
            const Pair sm = both(inverse_power(sc & 255u)), sv = both(inverse_power(sc >> 8));
            float y[kPer];
            e4m3x8_values(x, cm);
            e4m3x8_values(y, cv);
#pragma unroll
            for (int i = 0; i < kPer / 2; ++i) {
                m[i] = mul(pair(x[2 * i], x[2 * i + 1]), sm);
                v[i] = mul(pair(y[2 * i], y[2 * i + 1]), sv);
                v[i] = mul(v[i], v[i]);
            }
        } else {
            float y[kPer];
            load8(x, grad + at, left, whole);
            load8(w, param + at, left, whole);
#pragma unroll
            for (int i = 0; i < kPer / 2; ++i) g[i] = pair(x[2 * i], x[2 * i + 1]);
            load8(x, em + at, left, whole);
            load8(y, ev + at, left, whole);
#pragma unroll
            for (int i = 0; i < kPer / 2; ++i) {
                m[i] = pair(x[2 * i], x[2 * i + 1]);
                v[i] = pair(y[2 * i], y[2 * i + 1]);
            }
        }
        if (s.grad_scale != nullptr)
#pragma unroll
            for (int i = 0; i < kPer / 2; ++i) g[i] = mul(g[i], both(scale));
        float root[kPer];
#pragma unroll
        for (int i = 0; i < kPer / 2; ++i) {
            // each product and sum rounded by itself, so that a formula without fused operations rounds its codes alike; the sums' factor of 1 keeps the compiler from fusing
            m[i] = fma(mul(beta1, m[i]), one, mul(rest1, g[i]));
            v[i] = fma(mul(beta2, v[i]), one, mul(mul(rest2, g[i]), g[i]));
            float d0, d1;
            const Pair r = EIGHT ? root_of(v[i]) : about_root_of(v[i]);
            apart(r, root[2 * i], root[2 * i + 1]);
            apart(fma(r, both(bias2), both(s.eps)), d0, d1);
            const Pair q = mul(m[i], pair(reciprocal(d0), reciprocal(d1)));
            apart(fma(both(-rate), q, mul(pair(w[2 * i], w[2 * i + 1]), both(keep))), w[2 * i], w[2 * i + 1]);
        }
        const uint64_t number = (uint64_t)(begin + at);
        const uint32_t high = mix((uint32_t)(number >> 32) ^ key) + (uint32_t)number;
        uint32_t rm[kPer], rv[kPer];                                  // 16 random bits for either moment
        if constexpr (EIGHT || sizeof(P) == 2)
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const uint32_t z = mix_most(high + i);
                rv[i] = z >> 16;
                rm[i] = (z ^ rv[i]) & 0xFFFFu;
            }
        if constexpr (sizeof(P) == 2) {
            // NaN, whose bits may all be set, must not be carried into the sign
            const bool any_nan = !(amax8(w) <= INFINITY);
            uint32_t b[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i) b[i] = __float_as_uint(w[i]) + (mix((rm[i] | rv[i] << 16) ^ 0x9E3779B9u) & 0xFFFFu);
            if (any_nan)
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (isnan(w[i])) b[i] = 0x7FC00000u;
            if (whole) {
                *reinterpret_cast<uint4*>(param + at) =
                    make_uint4(__byte_perm(b[0], b[1], 0x7632), __byte_perm(b[2], b[3], 0x7632), __byte_perm(b[4], b[5], 0x7632), __byte_perm(b[6], b[7], 0x7632));
            } else {
#pragma unroll
                for (int i = 0; i < kPer; ++i) w[i] = __uint_as_float(b[i] & 0xFFFF0000u);
                store8(w, param + at, left, false);
            }
        } else {
            store8(w, param + at, left, whole);
        }
#pragma unroll
        for (int i = 0; i < kPer / 2; ++i) apart(m[i], x[2 * i], x[2 * i + 1]);
        if constexpr (EIGHT) {
            float am = amax8(x), av = amax8(root);
            uint32_t ranks = block_ranks(am, av), bad = 0;
            const bool finite = (ranks & 0xFFFFu) < 255u && ranks >> 16 < 255u;
            if (__any_sync(0xFFFFFFFFu, !finite)) {                   // take the maxima of the finite ones, and note (32 bits) which are not
                am = largest_finite(x);
                av = largest_finite(root);
                ranks = block_ranks(am, av);
#pragma unroll
                for (int i = 0; i < kPer; ++i) bad |= (fabsf(x[i]) < INFINITY ? 0u : 1u << i) | (root[i] < INFINITY ? 0u : 256u << i);
            }
            // what is far below 2^-126 has a rank of 0, as zero has: blocks of zeros alone are told apart by a vote
            uint32_t some = (am > 0.f ? 1u : 0u) | (av > 0.f ? 65536u : 0u);
            if (__any_sync(0xFFFFFFFFu, (ranks & 0xFFFFu) == 0 || ranks >> 16 == 0))
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) some |= __shfl_xor_sync(0xFFFFFFFFu, some, o);
            const uint32_t sm = scale_of_rank(ranks & 0xFFFFu, (ranks & 0xFFFFu) == 0 && (some & 1u) == 0), sv = scale_of_rank(ranks >> 16, ranks >> 16 == 0 && some >> 16 == 0);
            const Pair fm = both(__uint_as_float(sm << 23)), fv = both(__uint_as_float(sv << 23));
            float y[kPer];
#pragma unroll
            for (int i = 0; i < kPer / 2; ++i) {
                apart(round_mean(mul(m[i], fm), rm[2 * i], rm[2 * i + 1]), x[2 * i], x[2 * i + 1]);
                apart(round_square_mean(mul(pair(root[2 * i], root[2 * i + 1]), fv), rv[2 * i], rv[2 * i + 1]), y[2 * i], y[2 * i + 1]);
            }
            if (bad != 0)
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    if (bad >> i & 1) x[i] = NAN;
                    if (bad >> (8 + i) & 1) y[i] = NAN;
                }
            store_codes(e4m3x8(x), em + at, left, whole);
            store_codes(e4m3x8(y), ev + at, left, whole);
            if (left > 0 && (threadIdx.x & 15) == 0) *reinterpret_cast<uint16_t*>(scales + at / 128 * 2) = (uint16_t)(sm | sv << 8);
        } else {
            float y[kPer];
#pragma unroll
            for (int i = 0; i < kPer / 2; ++i) apart(v[i], y[2 * i], y[2 * i + 1]);
            store8(x, em + at, left, whole);
            store8(y, ev + at, left, whole);
        }
    }
}

// The values that codes stand for, 8 elements a thread: 29 M elements to BF16 28 us, 6.3 TB/s.
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
mor_status_t adamw_launch(const AdamwScalars& s, const mor_adamw_tensor_t* t, const uint32_t* numbers, int n, cudaStream_t st)
{
    static std::atomic<uint64_t> done{0};
    constexpr int kSmem = EIGHT ? OwnRing<P, G>::kBytes : 0;
    if (EIGHT && !allow_smem(adamw_kernel<P, G, EIGHT, N>, kSmem, done)) return MOR_ERR_CUDA;
    AdamwParams<N> p;
    p.s = s;
    for (int at = 0; at < n; at += N) {
        const int k = n - at < N ? n - at : N;
        int64_t passes = 0;
        for (int i = 0; i < k; ++i) passes += ceil_div(t[at + i].numel, kPass);
        if (passes == 0) continue;
        // a CTA takes several passes where that leaves the GPU full (four CTAs an SM): its copies ahead then pay
        int64_t per = passes / (148 * 4);
        per = per < 1 ? 1 : per > kMostPasses ? kMostPasses : per;
        p.s.chunk = (int32_t)per * kPass;
        p.s.count = (uint32_t)k;
        if (s.each != 0) p.s.device_step = s.device_step + at;
        int64_t ctas = 0;
        for (int i = 0; i < k; ++i) {
            const mor_adamw_tensor_t& x = t[at + i];
            const size_t state = EIGHT ? 8 : 32;
            const bool aligned = is_aligned(x.param, kPer * sizeof(P)) && is_aligned(x.grad, kPer * sizeof(G)) && is_aligned(x.exp_avg, state) && is_aligned(x.exp_avg_sq, state);
            const uint32_t number = numbers != nullptr ? numbers[at + i] : (uint32_t)(at + i);
            p.e[i] = {x.param, x.grad, x.exp_avg, x.exp_avg_sq, x.scales, x.numel, (uint32_t)ctas, number * 2 + (aligned ? 1u : 0u)};
            ctas += ceil_div(x.numel, p.s.chunk);
        }
        if (launch(adamw_kernel<P, G, EIGHT, N>, (uint32_t)ctas, kThreads, kSmem, st, ctas <= kEarlyGrid, p) != cudaSuccess) return MOR_ERR_CUDA;
    }
    return MOR_OK;
}
template <typename P, typename G, bool EIGHT> mor_status_t adamw_table(const AdamwScalars& s, const mor_adamw_tensor_t* t, const uint32_t* numbers, int n, cudaStream_t st)
{
    if (n <= 16) return adamw_launch<P, G, EIGHT, 16>(s, t, numbers, n, st);
    if (n <= 128) return adamw_launch<P, G, EIGHT, 128>(s, t, numbers, n, st);
    return adamw_launch<P, G, EIGHT, 512>(s, t, numbers, n, st);
}
template <typename P, typename G> mor_status_t adamw_state(const mor_adamw_desc_t& d, const AdamwScalars& s, const mor_adamw_tensor_t* t, int n, cudaStream_t st)
{
    return d.eight_bits ? adamw_table<P, G, true>(s, t, d.numbers, n, st) : adamw_table<P, G, false>(s, t, d.numbers, n, st);
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
    int64_t all = 0;
    for (int i = 0; i < n; ++i) {
        const mor_adamw_tensor_t& x = t[i];
        if (d->numbers != nullptr && d->numbers[i] >= 1u << 31) return MOR_ERR_INVALID_ARG;
        if (x.numel < 0 || x.numel >= (1ll << 40) || (all += x.numel) >= (1ll << 42)) return MOR_ERR_INVALID_ARG;     // what a grid holds
        if (x.numel == 0) continue;
        if (x.param == nullptr || x.grad == nullptr || x.exp_avg == nullptr || x.exp_avg_sq == nullptr || (d->eight_bits && x.scales == nullptr)) return MOR_ERR_INVALID_ARG;
        if (!is_aligned(x.param, dtype_bytes(d->param_dtype)) || !is_aligned(x.grad, dtype_bytes(d->grad_dtype)) || !is_aligned(x.exp_avg, state) ||
            !is_aligned(x.exp_avg_sq, state) || (d->eight_bits && !is_aligned(x.scales, 2)))
            return MOR_ERR_ALIGNMENT;
    }
    if (all == 0) return MOR_OK;
    AdamwScalars s = {};
    s.lr = (float)d->lr;
    s.one = 1.f;
    s.beta1 = (float)d->beta1;
    s.beta2 = (float)d->beta2;
    s.rest1 = (float)(1.0 - d->beta1);
    s.rest2 = (float)(1.0 - d->beta2);
    s.eps = std::max((float)d->eps, 0x1p-63f);
    s.decay = (float)d->weight_decay;
    s.bias1 = (float)(1.0 / (1.0 - pow(d->beta1, (double)d->step)));
    s.bias2 = (float)(1.0 / sqrt(1.0 - pow(d->beta2, (double)d->step)));
    s.log1 = (float)log(d->beta1);                                   // beta 0: -infinity, and 1 - beta^step is 1
    s.log2 = (float)log(d->beta2);
    s.seed = (uint32_t)d->seed;
    s.step = (uint32_t)d->step;
    s.device_step = d->device_step;
    s.each = d->device_step != nullptr && d->device_step_each ? 1 : 0;
    s.device_lr = d->device_lr;
    s.grad_scale = d->grad_scale;
    s.found_inf = d->found_inf;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const bool g16 = d->grad_dtype == MOR_DTYPE_BF16;
    if (d->param_dtype == MOR_DTYPE_BF16)
        return g16 ? adamw_state<__nv_bfloat16, __nv_bfloat16>(*d, s, t, n, st) : adamw_state<__nv_bfloat16, float>(*d, s, t, n, st);
    return g16 ? adamw_state<float, __nv_bfloat16>(*d, s, t, n, st) : adamw_state<float, float>(*d, s, t, n, st);
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
