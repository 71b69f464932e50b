// Low-rank adapters beside a shared projection: out = base + s (x a^T) b^T with an adapter for every token, and the gradients.
//
// The ranks are small, so every product here moves far more than it multiplies: the wide matrices (x, base, out, dy) are read and written
// once, by fragments that go straight between memory and the registers of the tensor instructions (mma.sync, BF16 in, FP32 sums), without a
// stop in shared memory.  Which element of the reduction axis meets which slot of an instruction does not matter as long as both operands agree,
// and neither does the order of the result's columns: slots are dealt out so that a thread's fragments are 16 neighbouring bytes.
//
//   shrink   h = s x a^T              reduction over the width, cut over the warps and a cluster's CTAs, joined through distributed shared memory
//   expand   out = base + h b^T       h as the sum of two BF16 (16 bits and more), columns in registers
//   outer    db = dy^T h, da = u^T x  reduction over an adapter's tokens, cut and joined like shrink
//   small    shrink and expand of up to 16 tokens of an adapter by one cluster, in one launch, for few tokens
//
// More tokens are sorted by adapter first (each adapter's rows start at a multiple of 32, a warp's rows).  All sums run in an order that depends on
// the sizes and ids alone.
#include "mor_layers.cuh"

namespace mor {
namespace {

using bf16 = __nv_bfloat16;

constexpr int kRows = 32;                 // rows of a warp; rows of an adapter start at multiples of it
constexpr int kMaxCluster = 8;
constexpr int kSmallRows = 16;            // tokens of a cluster in the small kernel
constexpr int kSmallWarps = 8;
constexpr int64_t kMaxWidth = 1 << 21;    // of the token matrices: what the grids hold
constexpr int64_t kSmallTokens = 256;     // most tokens that the small kernel takes

// d += a b for 16 x 16 by 16 x 8.
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t a0, const uint32_t a1, const uint32_t a2, const uint32_t a3, const uint32_t b0, const uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The transpose of an 8 x 8 matrix of 16-bit elements that is spread over the warp.
__device__ __forceinline__ uint32_t transposed(uint32_t v)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// A float of another CTA's shared memory, at the place that `own` has in this one's.
__device__ __forceinline__ float load_remote(const float* own, uint32_t rank)
{
    float v;
    asm volatile("{ .reg .u32 a; mapa.shared::cluster.u32 a, %1, %2; ld.shared::cluster.f32 %0, [a]; }"
                 : "=f"(v) : "r"((uint32_t)__cvta_generic_to_shared(own)), "r"(rank) : "memory");
    return v;
}

// Tokens sorted by adapter, or (starts null) as they come, all of adapter 0.
struct Sorted {
    const int32_t *starts, *row_of_token, *token_of_row;
    int64_t rows, tokens;
    int32_t adapters;
};
__device__ __forceinline__ int64_t used_rows(const Sorted& s) { return s.starts != nullptr ? s.starts[s.adapters] : s.rows; }
__device__ __forceinline__ int32_t token_at(const Sorted& s, int64_t row)
{
    if (s.starts != nullptr) return s.token_of_row[row];
    return row < s.tokens ? (int32_t)row : -1;
}
// The adapter of a row, found by a warp.
__device__ __forceinline__ int adapter_of(const Sorted& s, int64_t row, int lane)
{
    if (s.starts == nullptr) return 0;
    int n = 0;
    for (int e = 0; e < s.adapters; e += 32) {
        const bool before = e + lane < s.adapters && s.starts[e + lane + 1] <= row;
        n += __popc(__ballot_sync(0xFFFFFFFFu, before));
    }
    return min(n, s.adapters - 1);
}

// 8 BF16 of a row of n from `at` on, zero from n on.
template <bool ANY> __device__ __forceinline__ uint4 load_frag(const bf16* row, int64_t at, int64_t n)
{
    uint32_t w[4] = {0, 0, 0, 0};
    if (row != nullptr && at < n) {
        if constexpr (ANY) load_any<bf16, 16>(w, row, at, n);
        else return *reinterpret_cast<const uint4*>(row + at);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ uint16_t bits_of(bf16 v) { return __bfloat16_as_ushort(v); }
// v as the sum of two BF16; a value that is not finite is the first alone.
__device__ __forceinline__ void split(float v, bf16& hi, bf16& lo)
{
    hi = __float2bfloat16(v);
    const float r = v - __bfloat162float(hi);
    lo = __float2bfloat16(fabsf(r) < INFINITY ? r : 0.f);
}

// ------------------------------------------------------------------------------------------- shrink ----

struct ShrinkParams {
    Sorted s;
    const bf16* x;             // [tokens, ldx], n wide
    const bf16* m;             // [adapters][m_rows, ldm]
    const float* scale;
    float factor;
    int64_t ldx, n, ldm, m_stride;
    int32_t m_rows;            // rows of m that exist
    int32_t padded;            // rank as the outputs have it
    bf16* natural;             // [rows][2][padded]
    bf16* turned;              // [2][padded][rows], optional
};

// A CTA of 4 warps takes ROW_WARPS x 32 rows and R of the ranks (blockIdx.y); a cluster's CTAs share the reduction axis, and so do the CTA's warps
// where they are more than the rows need (few tokens).
template <int R, int ROW_WARPS, bool ANY> __global__ void __launch_bounds__(128) adapter_shrink_kernel(const __grid_constant__ ShrinkParams p)
{
    constexpr int kSplit = 4 / ROW_WARPS, kTiles = R / 8, kPitch = R + 8;       // pitch: 8 rows of 8-byte pairs in distinct banks
    __shared__ float part[4][kRows][kPitch];
    __shared__ float scales[ROW_WARPS];
    wait_for_predecessor();
    const uint32_t rank = cluster_rank(), ctas = cluster_size();
    const int64_t first = (int64_t)(blockIdx.x / ctas) * (ROW_WARPS * kRows);
    if (first >= used_rows(p.s)) return;                                          // the whole cluster
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int64_t row0 = first + warp / kSplit * kRows;
    const int r0 = blockIdx.y * R;
    float acc[2][kTiles][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < kTiles; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[i][j][k] = 0.f;
    if (row0 < used_rows(p.s)) {
        const int adapter = adapter_of(p.s, row0, lane);
        if (lane == 0 && warp % kSplit == 0) scales[warp / kSplit] = (p.scale != nullptr ? p.scale[adapter] : 1.f) * p.factor;
        const bf16* xr[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t t = token_at(p.s, row0 + i * 8 + g);
            xr[i] = t >= 0 ? p.x + (int64_t)t * p.ldx : nullptr;
        }
        const bf16* m = p.m + (int64_t)adapter * p.m_stride + (int64_t)(r0 + g) * p.ldm;
        const int left = p.m_rows - r0 - g;                                       // rows of m from this thread's first on
        const int64_t steps = (p.n + 31) / 32, share = (steps + ctas * kSplit - 1) / (ctas * kSplit);
        const int64_t begin = min((int64_t)(rank * kSplit + warp % kSplit) * share, steps), end = min(begin + share, steps);
        uint4 xs[4], next[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) xs[i] = begin < end ? load_frag<ANY>(xr[i], begin * 32 + q * 8, p.n) : make_uint4(0, 0, 0, 0);
        for (int64_t step = begin; step < end; ++step) {
            const int64_t at = step * 32 + q * 8;
#pragma unroll
            for (int i = 0; i < 4; ++i) next[i] = step + 1 < end ? load_frag<ANY>(xr[i], at + 32, p.n) : make_uint4(0, 0, 0, 0);
            uint4 w[kTiles];
#pragma unroll
            for (int j = 0; j < kTiles; ++j) w[j] = load_frag<ANY>(j * 8 < left ? m + (int64_t)j * 8 * p.ldm : nullptr, at, p.n);
#pragma unroll
            for (int j = 0; j < kTiles; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    mma(acc[i][j], xs[2 * i].x, xs[2 * i + 1].x, xs[2 * i].y, xs[2 * i + 1].y, w[j].x, w[j].y);
                    mma(acc[i][j], xs[2 * i].z, xs[2 * i + 1].z, xs[2 * i].w, xs[2 * i + 1].w, w[j].z, w[j].w);
                }
#pragma unroll
            for (int i = 0; i < 4; ++i) xs[i] = next[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
            *reinterpret_cast<float2*>(&part[warp][i * 16 + g][j * 8 + 2 * q]) = make_float2(acc[i][j][0], acc[i][j][1]);
            *reinterpret_cast<float2*>(&part[warp][i * 16 + g + 8][j * 8 + 2 * q]) = make_float2(acc[i][j][2], acc[i][j][3]);
        }
    __syncthreads();
    cluster_arrive();
    cluster_wait();
    // a column of four rows is a task; the cluster's CTAs take the groups of rows in turn
    constexpr int kGroups = ROW_WARPS * kRows / 4;
    for (int task = threadIdx.x; task < kGroups * R; task += 128) {
        const int col = task % R, group = task / R;
        if ((uint32_t)group % ctas != rank) continue;
        const int rw = group / (kRows / 4), at = group % (kRows / 4) * 4;
        const int64_t row = first + rw * kRows + at;
        if (row >= used_rows(p.s)) continue;
        const float s = scales[rw];
        bf16 hi[4], lo[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float sum = 0.f;
            for (uint32_t c = 0; c < ctas; ++c)
#pragma unroll
                for (int w = 0; w < kSplit; ++w) sum += load_remote(&part[rw * kSplit + w][at + k][col], c);
            split(sum * s, hi[k], lo[k]);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            bf16* to = p.natural + (row + k) * 2 * p.padded + r0 + col;
            to[0] = hi[k];
            to[p.padded] = lo[k];
        }
        if (p.turned != nullptr) {
            uint16_t* to = reinterpret_cast<uint16_t*>(p.turned) + (int64_t)(r0 + col) * p.s.rows + row;
            *reinterpret_cast<ushort4*>(to) = make_ushort4(bits_of(hi[0]), bits_of(hi[1]), bits_of(hi[2]), bits_of(hi[3]));
            *reinterpret_cast<ushort4*>(to + (int64_t)p.padded * p.s.rows) = make_ushort4(bits_of(lo[0]), bits_of(lo[1]), bits_of(lo[2]), bits_of(lo[3]));
        }
    }
    cluster_arrive();                    // nobody leaves while its sums are read
    cluster_wait();
}

// ------------------------------------------------------------------------------------------- expand ----

struct ExpandParams {
    Sorted s;
    const bf16* h;             // [rows][2][padded]
    const bf16* m;             // [adapters][n, ldm], `m_cols` of them
    int64_t n, ldm, m_stride;
    int32_t m_cols, padded;
    const void* base;          // optional
    void* out;
    int64_t ldb, ldo;
    uint32_t row_ctas;         // CTAs of rows; those behind copy the tokens without an adapter
    int32_t share;             // steps of 32 columns of a CTA
    bool m_whole, base_whole, out_whole;
};

// Row `n` of m for the slots of a thread: 8 neighbouring ranks for R >= 32, 4 for R = 16.
template <int R> __device__ __forceinline__ void load_m(uint32_t* w, const bf16* row, int at, int cols, bool whole)
{
    constexpr int kWords = R == 16 ? 2 : 4;
    if (whole && row != nullptr && at < cols) {
        if constexpr (R == 16) {
            const uint2 v = *reinterpret_cast<const uint2*>(row + at);
            w[0] = v.x;
            w[1] = v.y;
        } else {
            const uint4 v = *reinterpret_cast<const uint4*>(row + at);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        }
        return;
    }
    const uint16_t* u = reinterpret_cast<const uint16_t*>(row);
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
        w[i] = 0;
        if (row != nullptr && at + 2 * i < cols) w[i] = u[at + 2 * i];
        if (row != nullptr && at + 2 * i + 1 < cols) w[i] |= (uint32_t)u[at + 2 * i + 1] << 16;
    }
}
template <typename T> __device__ __forceinline__ void load_base(float* v, const T* row, int64_t at, int64_t n, bool whole)
{
    Piece<T, kPer * (int)sizeof(T), 16> piece;
    piece.clear();
    if (row != nullptr && at < n) {
        if (whole) piece.load(row + at);
        else load_any<T, kPer * (int)sizeof(T)>(piece.w, row, at, n);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = piece.get(i);
}
template <typename T> __device__ __forceinline__ void store_out(const float* v, T* row, int64_t at, int64_t n, bool whole)
{
    if (at >= n) return;
    if (whole && at + kPer <= n) {
        Piece<T, kPer * (int)sizeof(T)> piece;
        piece.set_all(v);
#pragma unroll
        for (int i = 0; i < Piece<T, kPer * (int)sizeof(T)>::kWords; i += 4)
            *reinterpret_cast<uint4*>(reinterpret_cast<uint32_t*>(row + at) + i) = make_uint4(piece.w[i], piece.w[i + 1], piece.w[i + 2], piece.w[i + 3]);
    } else {
        store8(v, row + at, (int)min((int64_t)kPer, n - at), false);
    }
}

// Fragments of 16 rows of h (g and g + 8 of `rows`, null: zero) for the slots that load_m() gives a thread.
template <int R> struct HFrags {
    static constexpr int kPairs = R / 16;
    uint32_t a[kPairs][4];
    __device__ __forceinline__ void load(const bf16* upper, const bf16* lower, int q)
    {
        if constexpr (R == 16) {
            const uint2 u = *reinterpret_cast<const uint2*>(upper + q * 4), l = *reinterpret_cast<const uint2*>(lower + q * 4);
            a[0][0] = u.x; a[0][1] = l.x; a[0][2] = u.y; a[0][3] = l.y;
        } else {
#pragma unroll
            for (int c = 0; c < R / 32; ++c) {
                const uint4 u = *reinterpret_cast<const uint4*>(upper + c * 32 + q * 8), l = *reinterpret_cast<const uint4*>(lower + c * 32 + q * 8);
                a[2 * c][0] = u.x; a[2 * c][1] = l.x; a[2 * c][2] = u.y; a[2 * c][3] = l.y;
                a[2 * c + 1][0] = u.z; a[2 * c + 1][1] = l.z; a[2 * c + 1][2] = u.w; a[2 * c + 1][3] = l.w;
            }
        }
    }
};

// 32 columns from c0 on of TILES x 16 rows: acc += h m^T.  Column c of instruction j is column 8 (c / 2) + 2 j + c % 2 of the 32, so that a thread's
// results are 8 neighbouring columns, 8 q and on.
template <int R, int TILES> struct Columns {
    uint32_t w[4][R / 8];
    __device__ __forceinline__ void load(const bf16* m, int64_t c0, int64_t n, int64_t ldm, int r0, int cols, bool whole, int g, int q)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t c = c0 + 8 * (g >> 1) + 2 * j + (g & 1);
            const bf16* row = c < n ? m + c * ldm : nullptr;
            if constexpr (R == 16) load_m<R>(w[j], row, r0 + q * 4, cols, whole);
            else
#pragma unroll
                for (int k = 0; k < R / 32; ++k) load_m<R>(w[j] + 4 * k, row, r0 + k * 32 + q * 8, cols, whole);
        }
    }
    __device__ __forceinline__ void add(float (&acc)[TILES][4][4], const HFrags<R> (&hi)[TILES], const HFrags<R> (&lo)[TILES]) const
    {
#pragma unroll
        for (int k = 0; k < R / 16; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < TILES; ++i) {
                    mma(acc[i][j], hi[i].a[k][0], hi[i].a[k][1], hi[i].a[k][2], hi[i].a[k][3], w[j][2 * k], w[j][2 * k + 1]);
                    mma(acc[i][j], lo[i].a[k][0], lo[i].a[k][1], lo[i].a[k][2], lo[i].a[k][3], w[j][2 * k], w[j][2 * k + 1]);
                }
    }
};

template <typename T> __device__ void copy_row(const ExpandParams& p, int64_t token, int64_t from, int64_t to, int lane)
{
    const T* base = p.base != nullptr ? static_cast<const T*>(p.base) + token * p.ldb : nullptr;
    T* out = static_cast<T*>(p.out) + token * p.ldo;
    for (int64_t at = from + lane * kPer; at < to; at += 32 * kPer) {
        float v[kPer];
        load_base(v, base, at, p.n, p.base_whole);
        store_out(v, out, at, p.n, p.out_whole);
    }
}

template <int R, typename T> __global__ void __launch_bounds__(128) adapter_expand_kernel(const __grid_constant__ ExpandParams p)
{
    wait_for_predecessor();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int64_t c_begin = (int64_t)blockIdx.y * p.share * 32, c_end = min(c_begin + (int64_t)p.share * 32, p.n);
    if (blockIdx.x >= p.row_ctas) {
        const int64_t t0 = (int64_t)(blockIdx.x - p.row_ctas) * 32;
        const uint32_t none = __ballot_sync(0xFFFFFFFFu, t0 + lane < p.s.tokens && p.s.row_of_token[t0 + lane] < 0);
        for (int i = warp; i < 32; i += 4)
            if (none >> i & 1) copy_row<T>(p, t0 + i, c_begin, c_end, lane);
        return;
    }
    const int64_t row0 = (int64_t)blockIdx.x * (4 * kRows) + warp * kRows;
    if (row0 >= used_rows(p.s)) return;
    const int adapter = adapter_of(p.s, row0, lane);
    const bf16* m = p.m + (int64_t)adapter * p.m_stride;
    const T* base[4];
    T* out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int32_t t = token_at(p.s, row0 + i * 8 + g);
        base[i] = t >= 0 && p.base != nullptr ? static_cast<const T*>(p.base) + (int64_t)t * p.ldb : nullptr;
        out[i] = t >= 0 ? static_cast<T*>(p.out) + (int64_t)t * p.ldo : nullptr;
    }
    HFrags<R> hi[2], lo[2];
    auto load_h = [&](int r0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const bf16* h = p.h + (row0 + i * 16 + g) * 2 * p.padded + r0;
            const int64_t below = (int64_t)8 * 2 * p.padded;
            hi[i].load(h, h + below, q);
            lo[i].load(h + p.padded, h + below + p.padded, q);
        }
    };
    if (p.padded == R) load_h(0);
    for (int64_t c0 = c_begin; c0 < c_end; c0 += 32) {
        float v[4][kPer], acc[2][4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) load_base(v[i], base[i], c0 + q * 8, p.n, p.base_whole);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[i][j][k] = 0.f;
        for (int r0 = 0; r0 < p.padded; r0 += R) {
            if (p.padded > R) load_h(r0);
            Columns<R, 2> w;
            w.load(m, c0, p.n, p.ldm, r0, p.m_cols, p.m_whole, g, q);
            w.add(acc, hi, lo);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (out[i] == nullptr) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[i][2 * j] += acc[i >> 1][j][(i & 1) * 2];
                v[i][2 * j + 1] += acc[i >> 1][j][(i & 1) * 2 + 1];
            }
            store_out(v[i], out[i], c0 + q * 8, p.n, p.out_whole);
        }
    }
}

// -------------------------------------------------------------------------------------------- outer ----

struct OuterParams {
    Sorted s;
    const bf16* h;             // [2][padded][rows]
    const bf16* z;             // [tokens, ldz], n wide
    int64_t ldz, n;
    int32_t rank, padded;
    bf16* out;                 // [adapters][rank][n], or [adapters][n][rank]
    int32_t by_column;         // the latter
};

// R ranks x 64 columns of an adapter.  The reduction runs over its rows, 32 at a time: warp by warp through the cluster.
template <int R, bool ANY> __global__ void __launch_bounds__(128) adapter_outer_kernel(const __grid_constant__ OuterParams p)
{
    constexpr int kCols = 64, kTiles = R / 16, kPitch = kCols + 8;
    __shared__ float part[R][kPitch];
    wait_for_predecessor();
    const uint32_t rank = cluster_rank(), ctas = cluster_size();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int chunks = p.padded / R, adapter = blockIdx.z / chunks, r0 = blockIdx.z % chunks * R;
    const int64_t c0 = (int64_t)blockIdx.y * kCols;
    const int64_t begin = p.s.starts != nullptr ? p.s.starts[adapter] : 0, end = p.s.starts != nullptr ? p.s.starts[adapter + 1] : adapter == 0 ? p.s.rows : 0;
    float acc[kTiles][8][4];
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[i][j][k] = 0.f;
    const bf16* hr = p.h + (int64_t)(r0 + g) * p.s.rows;
    const int64_t low = (int64_t)p.padded * p.s.rows;
    for (int64_t row = begin + (int64_t)(rank * 4 + warp) * kRows; row < end; row += (int64_t)ctas * 4 * kRows) {
        uint4 z[4][2];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int32_t t = token_at(p.s, row + 8 * (g >> 1) + (g & 1) + 2 * k);
            const bf16* zr = t >= 0 ? p.z + (int64_t)t * p.ldz : nullptr;
            z[k][0] = load_frag<ANY>(zr, c0 + q * 8, p.n);
            z[k][1] = load_frag<ANY>(zr, c0 + 32 + q * 8, p.n);
        }
        // z's fragments as the second operand: its rows are the reduction axis
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int f = 0; f < 2; ++f)
                z[k][f] = make_uint4(transposed(z[k][f].x), transposed(z[k][f].y), transposed(z[k][f].z), transposed(z[k][f].w));
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const bf16* h = hr + (int64_t)i * 16 * p.s.rows + row + q * 8 + half * low;
                const uint4 u = *reinterpret_cast<const uint4*>(h), l = *reinterpret_cast<const uint4*>(h + 8 * p.s.rows);
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    mma(acc[i][4 * f], u.x, l.x, u.y, l.y, z[0][f].x, z[1][f].x);
                    mma(acc[i][4 * f + 1], u.x, l.x, u.y, l.y, z[0][f].y, z[1][f].y);
                    mma(acc[i][4 * f + 2], u.x, l.x, u.y, l.y, z[0][f].z, z[1][f].z);
                    mma(acc[i][4 * f + 3], u.x, l.x, u.y, l.y, z[0][f].w, z[1][f].w);
                    mma(acc[i][4 * f], u.z, l.z, u.w, l.w, z[2][f].x, z[3][f].x);
                    mma(acc[i][4 * f + 1], u.z, l.z, u.w, l.w, z[2][f].y, z[3][f].y);
                    mma(acc[i][4 * f + 2], u.z, l.z, u.w, l.w, z[2][f].z, z[3][f].z);
                    mma(acc[i][4 * f + 3], u.z, l.z, u.w, l.w, z[2][f].w, z[3][f].w);
                }
            }
    }
#pragma unroll 1
    for (int turn = 0; turn < 4; ++turn) {
        if (warp == turn) {
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        float2* at = reinterpret_cast<float2*>(&part[i * 16 + b * 8 + g][(j >> 2) * 32 + q * 8 + (j & 3) * 2]);
                        float2 v = turn > 0 ? *at : make_float2(0.f, 0.f);
                        v.x += acc[i][j][2 * b];
                        v.y += acc[i][j][2 * b + 1];
                        *at = v;
                    }
        }
        __syncthreads();
    }
    cluster_arrive();
    cluster_wait();
    bf16* out = p.out + (int64_t)adapter * p.rank * p.n;
    for (uint32_t at = rank * 128 + threadIdx.x; at < R * kCols; at += ctas * 128) {
        const int r = p.by_column ? at % R : at / kCols, c = p.by_column ? at / R : at % kCols;
        if (r0 + r >= p.rank || c0 + c >= p.n) continue;
        float sum = 0.f;
        for (uint32_t k = 0; k < ctas; ++k) sum += load_remote(&part[r][c], k);
        out[p.by_column ? (c0 + c) * p.rank + r0 + r : (int64_t)(r0 + r) * p.n + c0 + c] = __float2bfloat16(sum);
    }
    cluster_arrive();
    cluster_wait();
}

// ---------------------------------------------------------------------------------------- transposes ----

struct TurnParams {
    const bf16 *a, *b;
    bf16 *at, *bt;             // [adapters][n_in][padded] and [adapters][padded][wide], zero where there is no element
    int64_t n_in, n_out, wide;
    int32_t rank, padded;
    uint32_t a_ctas;           // CTAs of a for one adapter
};

// Both matrices of the adapters with their axes swapped, for the gradients' products: tiles of 32 x 32.
__global__ void __launch_bounds__(256) adapter_turn_kernel(const __grid_constant__ TurnParams p)
{
    __shared__ bf16 tile[32][33];
    wait_for_predecessor();
    const bool is_a = blockIdx.x < p.a_ctas;
    const uint32_t cta = is_a ? blockIdx.x : blockIdx.x - p.a_ctas;
    const int64_t rows = is_a ? p.rank : p.n_out, cols = is_a ? p.n_in : p.rank;               // of what is read
    const int64_t out_rows = is_a ? p.n_in : p.padded, out_cols = is_a ? p.padded : p.wide;
    const uint32_t across = (uint32_t)((out_cols + 31) / 32);
    const int64_t i0 = (int64_t)(cta % across) * 32, j0 = (int64_t)(cta / across) * 32;        // first row and column of what is read
    const bf16* in = (is_a ? p.a : p.b) + (int64_t)blockIdx.y * rows * cols;
    bf16* out = (is_a ? p.at : p.bt) + (int64_t)blockIdx.y * out_rows * out_cols;
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
#pragma unroll
    for (int k = y; k < 32; k += 8) tile[k][x] = i0 + k < rows && j0 + x < cols ? in[(i0 + k) * cols + j0 + x] : __float2bfloat16(0.f);
    __syncthreads();
#pragma unroll
    for (int k = y; k < 32; k += 8)
        if (j0 + k < out_rows && i0 + x < out_cols) out[(j0 + k) * out_cols + i0 + x] = tile[x][k];
}

// -------------------------------------------------------------------------------------------- small ----

struct SmallParams {
    const bf16 *x, *a, *b;
    const int32_t* ids;
    const float* scale;
    float factor;
    int32_t adapters, rank;
    int32_t tokens;
    int64_t ldx, n_in, n_out;
    const void* base;
    void* out;
    int64_t ldb, ldo;
    bool b_whole, base_whole, out_whole;
};

// A cluster of 8 for every token (every 16 without ids).  The first of each 16 tokens of an adapter, in token order, leads: its cluster takes all of
// them and the others' clusters end.  Every CTA sums its part of the width over its warps, then all parts are joined from the 8 shared
// memories, and each CTA makes an eighth of the columns.  Bound by the latency of four dependent reads (ids, x and a, b and base, and the exchange).
template <int R, typename T, bool ANY> __global__ void __cluster_dims__(kMaxCluster, 1, 1) __launch_bounds__(kSmallWarps * 32)
    adapter_small_kernel(const __grid_constant__ SmallParams p)
{
    constexpr int kTiles = R / 8, kPitch = R + 8;
    __shared__ float part[kSmallWarps][kSmallRows][kPitch];
    __shared__ float own[kSmallRows][kPitch], whole[kSmallRows][kPitch];
    __shared__ uint32_t same[kSmallTokens / 32];
    __shared__ int32_t members[kSmallRows];
    wait_for_predecessor();
    const uint32_t rank = cluster_rank();
    const int tile = blockIdx.x / kMaxCluster, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    int adapter = 0;
    if (p.ids != nullptr) {
        static_assert(kSmallTokens <= kSmallWarps * 32, "a token a thread");
        int32_t own_id = -2;
        if ((int)threadIdx.x < p.tokens) {
            own_id = p.ids[threadIdx.x];
            if (own_id < 0 || own_id >= p.adapters) own_id = -1;
        }
        adapter = p.ids[tile];
        if (adapter < 0 || adapter >= p.adapters) adapter = -1;
        const uint32_t mask = __ballot_sync(0xFFFFFFFFu, own_id == adapter);
        if (lane == 0) same[warp] = mask;
        if (threadIdx.x < kSmallRows) members[threadIdx.x] = -1;
        __syncthreads();
        int before = 0;                                        // tokens of the adapter before this one, and before this thread's
        for (int w = 0; w < tile >> 5; ++w) before += __popc(same[w]);
        before += __popc(same[tile >> 5] & ((1u << (tile & 31)) - 1u));
        if (before % kSmallRows != 0) return;                  // the whole cluster
        int mine = 0;
        for (int w = 0; w < warp; ++w) mine += __popc(same[w]);
        mine += __popc(mask & ((1u << lane) - 1u)) - before;
        if (own_id == adapter && mine >= 0 && mine < kSmallRows) members[mine] = (int32_t)threadIdx.x;
    } else if (threadIdx.x < kSmallRows) {
        const int t = tile * kSmallRows + (int)threadIdx.x;
        members[threadIdx.x] = t < p.tokens ? t : -1;
    }
    __syncthreads();
    const int64_t steps = (p.n_out + 31) / 32, share = (steps + kMaxCluster - 1) / kMaxCluster;
    const int64_t c_first = min((int64_t)rank * share, steps), c_last = min(c_first + share, steps);
    const int32_t upper = members[g], lower = members[g + 8];
    const T* base0 = upper >= 0 ? static_cast<const T*>(p.base) + (int64_t)upper * p.ldb : nullptr;
    const T* base1 = lower >= 0 ? static_cast<const T*>(p.base) + (int64_t)lower * p.ldb : nullptr;
    T* out0 = upper >= 0 ? static_cast<T*>(p.out) + (int64_t)upper * p.ldo : nullptr;
    T* out1 = lower >= 0 ? static_cast<T*>(p.out) + (int64_t)lower * p.ldo : nullptr;
    if (adapter < 0) {                                         // tokens without an adapter: the whole cluster copies
        for (int64_t step = c_first + warp; step < c_last; step += kSmallWarps) {
            float v[kPer];
            load_base(v, base0, step * 32 + q * 8, p.n_out, p.base_whole);
            if (out0 != nullptr) store_out(v, out0, step * 32 + q * 8, p.n_out, p.out_whole);
            load_base(v, base1, step * 32 + q * 8, p.n_out, p.base_whole);
            if (out1 != nullptr) store_out(v, out1, step * 32 + q * 8, p.n_out, p.out_whole);
        }
        return;
    }
    float acc[kTiles][4];
#pragma unroll
    for (int j = 0; j < kTiles; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[j][k] = 0.f;
    const bf16* x0 = upper >= 0 ? p.x + (int64_t)upper * p.ldx : nullptr;
    const bf16* x1 = lower >= 0 ? p.x + (int64_t)lower * p.ldx : nullptr;
    const bf16* a = p.a + ((int64_t)adapter * p.rank + g) * p.n_in;
    const bf16* b = p.b + (int64_t)adapter * p.n_out * p.rank;
    const int64_t in_steps = (p.n_in + 31) / 32;
#pragma unroll 2
    for (int64_t step = rank * kSmallWarps + warp; step < in_steps; step += kMaxCluster * kSmallWarps) {
        const int64_t at = step * 32 + q * 8;
        const uint4 u = load_frag<ANY>(x0, at, p.n_in), l = load_frag<ANY>(x1, at, p.n_in);
        uint4 w[kTiles];
#pragma unroll
        for (int j = 0; j < kTiles; ++j) w[j] = load_frag<ANY>(j * 8 + g < p.rank ? a + (int64_t)j * 8 * p.n_in : nullptr, at, p.n_in);
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
            mma(acc[j], u.x, l.x, u.y, l.y, w[j].x, w[j].y);
            mma(acc[j], u.z, l.z, u.w, l.w, w[j].z, w[j].w);
        }
    }
    // the first columns' share of b and base is on its way while the sums are joined
    Columns<R, 1> cols;
    float v0[kPer], v1[kPer];
    int64_t step = c_first + warp;
    auto fetch = [&] {
        if (step >= c_last) return;
        cols.load(b, step * 32, p.n_out, p.rank, 0, p.rank, p.b_whole, g, q);
        load_base(v0, base0, step * 32 + q * 8, p.n_out, p.base_whole);
        load_base(v1, base1, step * 32 + q * 8, p.n_out, p.base_whole);
    };
    fetch();
#pragma unroll
    for (int j = 0; j < kTiles; ++j) {
        *reinterpret_cast<float2*>(&part[warp][g][j * 8 + 2 * q]) = make_float2(acc[j][0], acc[j][1]);
        *reinterpret_cast<float2*>(&part[warp][g + 8][j * 8 + 2 * q]) = make_float2(acc[j][2], acc[j][3]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kSmallRows * R; i += kSmallWarps * 32) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kSmallWarps; ++w) sum += part[w][i / R][i % R];
        own[i / R][i % R] = sum;
    }
    cluster_arrive();
    cluster_wait();
    const float s = (p.scale != nullptr ? p.scale[adapter] : 1.f) * p.factor;
    for (int i = threadIdx.x; i < kSmallRows * R; i += kSmallWarps * 32) {
        float sum = 0.f;
        if (members[i / R] >= 0)
#pragma unroll
            for (uint32_t c = 0; c < kMaxCluster; ++c) sum += load_remote(&own[i / R][i % R], c);
        whole[i / R][i % R] = sum * s;
    }
    cluster_arrive();                                          // the sums have been read
    __syncthreads();
    HFrags<R> hi[1], lo[1];
    constexpr int kLane = R == 16 ? 4 : 8;
#pragma unroll
    for (int k = 0; k < R / 16; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // slot i of pair k: row g + 8 (i & 1); neighbouring ranks as load_m() deals them out
            const int r = R == 16 ? q * kLane + (i >> 1) * 2 : k / 2 * 32 + q * kLane + (k & 1) * 4 + (i >> 1) * 2;
            const float2 f = *reinterpret_cast<const float2*>(&whole[g + 8 * (i & 1)][r]);
            bf16 h0, h1, l0, l1;
            split(f.x, h0, l0);
            split(f.y, h1, l1);
            hi[0].a[k][i] = (uint32_t)bits_of(h0) | (uint32_t)bits_of(h1) << 16;
            lo[0].a[k][i] = (uint32_t)bits_of(l0) | (uint32_t)bits_of(l1) << 16;
        }
    while (step < c_last) {
        float sum[1][4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[0][j][k] = 0.f;
        cols.add(sum, hi, lo);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v0[2 * j] += sum[0][j][0];
            v0[2 * j + 1] += sum[0][j][1];
            v1[2 * j] += sum[0][j][2];
            v1[2 * j + 1] += sum[0][j][3];
        }
        if (out0 != nullptr) store_out(v0, out0, step * 32 + q * 8, p.n_out, p.out_whole);
        if (out1 != nullptr) store_out(v1, out1, step * 32 + q * 8, p.n_out, p.out_whole);
        step += kSmallWarps;
        fetch();
    }
    cluster_wait();
}

// ---------------------------------------------------------------------------------------- host side ----

template <typename... P, typename... A>
cudaError_t launch_clusters(void (*kernel)(P...), dim3 grid, uint32_t cluster, uint32_t block, cudaStream_t st, A&&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 0 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<A>(args)...);
}

int padded_rank(int rank) { return rank <= 16 ? 16 : rank <= 32 ? 32 : (rank + 63) / 64 * 64; }
int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// Parts of a workspace, each on 256 bytes.
struct Parts {
    uint8_t* base;
    size_t used = 0;
    void* take(size_t bytes)
    {
        void* p = base != nullptr ? base + used : nullptr;
        used += (bytes + 255) / 256 * 256;
        return p;
    }
};

struct Forward {
    Sorted s;
    void* sort;
    size_t sort_bytes;
    bf16 *natural, *turned;
    size_t bytes;
};
Forward forward_parts(const mor_adapter_desc_t& d, bool train, void* workspace)
{
    Forward f = {};
    Parts parts = {static_cast<uint8_t*>(workspace)};
    const int pad = padded_rank(d.rank);
    f.s.tokens = d.tokens;
    f.s.adapters = d.adapters;
    f.s.rows = d.ids != nullptr ? mor_expert_rows(d.tokens, d.adapters, kRows) : up(d.tokens, kRows);
    if (d.ids != nullptr) {
        f.s.starts = static_cast<int32_t*>(parts.take((size_t)(d.adapters + 1) * 4));
        f.s.row_of_token = static_cast<int32_t*>(parts.take((size_t)d.tokens * 4));
        f.s.token_of_row = static_cast<int32_t*>(parts.take((size_t)f.s.rows * 4));
        f.sort_bytes = mor_expert_workspace_bytes(d.tokens, d.adapters);
        f.sort = parts.take(f.sort_bytes);
    }
    f.natural = static_cast<bf16*>(parts.take((size_t)f.s.rows * 2 * pad * 2));
    if (train) f.turned = static_cast<bf16*>(parts.take((size_t)f.s.rows * 2 * pad * 2));
    f.bytes = parts.used;
    return f;
}
struct Backward {
    bf16 *natural, *turned, *at, *bt;
    int64_t wide;
    size_t bytes;
};
Backward backward_parts(const mor_adapter_desc_t& d, void* workspace)
{
    Backward f = {};
    Parts parts = {static_cast<uint8_t*>(workspace)};
    const int pad = padded_rank(d.rank);
    const int64_t rows = d.ids != nullptr ? mor_expert_rows(d.tokens, d.adapters, kRows) : up(d.tokens, kRows);
    f.wide = up(d.n_out, 8);
    f.natural = static_cast<bf16*>(parts.take((size_t)rows * 2 * pad * 2));
    f.turned = static_cast<bf16*>(parts.take((size_t)rows * 2 * pad * 2));
    f.at = static_cast<bf16*>(parts.take((size_t)d.adapters * d.n_in * pad * 2));
    f.bt = static_cast<bf16*>(parts.take((size_t)d.adapters * pad * f.wide * 2));
    f.bytes = parts.used;
    return f;
}
bool small_call(const mor_adapter_desc_t& d, bool train) { return !train && d.tokens <= kSmallTokens && d.rank <= 64; }

template <typename F> cudaError_t by_rank(int padded, F&& f)
{
    return padded == 16 ? f(std::integral_constant<int, 16>{}) : padded == 32 ? f(std::integral_constant<int, 32>{}) : f(std::integral_constant<int, 64>{});
}

// Rows of few tokens leave most of the GPU without work, so their warps share the reduction axis instead of standing one below the other: from
// 2048 rows on there are enough of 128 (with 8 CTAs each 128 clusters' worth of warps).
cudaError_t shrink(const ShrinkParams& p, bool any, cudaStream_t st)
{
    const bool tall = p.s.rows >= 2048;
    const int64_t steps = (p.n + 31) / 32;
    uint32_t cluster = kMaxCluster;
    while (cluster > 1 && steps < 2 * cluster) cluster /= 2;
    return by_rank(p.padded > 64 ? 64 : p.padded, [&](auto r) {
        constexpr int R = decltype(r)::value;
        const dim3 grid((uint32_t)(up(p.s.rows, tall ? 4 * kRows : kRows) / (tall ? 4 * kRows : kRows)) * cluster, (uint32_t)(p.padded / R));
        if (tall) return any ? launch_clusters(adapter_shrink_kernel<R, 4, true>, grid, cluster, 128, st, p) : launch_clusters(adapter_shrink_kernel<R, 4, false>, grid, cluster, 128, st, p);
        return any ? launch_clusters(adapter_shrink_kernel<R, 1, true>, grid, cluster, 128, st, p) : launch_clusters(adapter_shrink_kernel<R, 1, false>, grid, cluster, 128, st, p);
    });
}
cudaError_t expand(ExpandParams p, int dtype, cudaStream_t st)
{
    p.row_ctas = (uint32_t)(up(p.s.rows, 4 * kRows) / (4 * kRows));
    const int64_t steps = (p.n + 31) / 32;
    // about eight CTAs an SM, and no fewer than four steps for the fragments of h that each loads
    int64_t across = std::max<int64_t>(1, std::min<int64_t>(steps / 4, 148 * 8 / std::max<uint32_t>(1, p.row_ctas)));
    p.share = (int32_t)((steps + across - 1) / across);
    across = (steps + p.share - 1) / p.share;
    const uint32_t copies = p.s.starts != nullptr ? (uint32_t)(up(p.s.tokens, 32) / 32) : 0;
    const dim3 grid(p.row_ctas + copies, (uint32_t)across);
    return by_rank(p.padded > 64 ? 64 : p.padded, [&](auto r) {
        constexpr int R = decltype(r)::value;
        return dtype == MOR_DTYPE_BF16 ? launch_clusters(adapter_expand_kernel<R, bf16>, grid, 0, 128, st, p) : launch_clusters(adapter_expand_kernel<R, float>, grid, 0, 128, st, p);
    });
}
cudaError_t outer(const OuterParams& p, bool any, cudaStream_t st)
{
    // as many CTAs as have two turns of 128 rows each, going by the adapters' mean
    const int64_t mean = p.s.rows / p.s.adapters;
    uint32_t cluster = kMaxCluster;
    while (cluster > 1 && mean < 256 * (int64_t)cluster) cluster /= 2;
    return by_rank(p.padded > 64 ? 64 : p.padded, [&](auto r) {
        constexpr int R = decltype(r)::value;
        const dim3 grid(cluster, (uint32_t)((p.n + 63) / 64), (uint32_t)(p.s.adapters * (p.padded / R)));
        return any ? launch_clusters(adapter_outer_kernel<R, true>, grid, cluster, 128, st, p) : launch_clusters(adapter_outer_kernel<R, false>, grid, cluster, 128, st, p);
    });
}

mor_status_t check_adapter(const mor_adapter_desc_t* d)
{
    if (d == nullptr || d->tokens < 0 || d->tokens >= (1ll << 30) || d->n_in < 1 || d->n_out < 1 || d->n_in > kMaxWidth || d->n_out > kMaxWidth) return MOR_ERR_INVALID_ARG;
    if (d->adapters < 1 || d->adapters >= MOR_MAX_GROUPS || d->rank < 1 || d->rank > MOR_MAX_RANK) return MOR_ERR_INVALID_ARG;
    if (d->a == nullptr || d->b == nullptr) return MOR_ERR_INVALID_ARG;
    if (d->ids != nullptr && mor_expert_rows(d->tokens, d->adapters, kRows) < 0) return MOR_ERR_INVALID_ARG;
    if (!is_aligned(d->a, 2) || !is_aligned(d->b, 2) || !is_aligned(d->ids, 4) || !is_aligned(d->scale, 4)) return MOR_ERR_ALIGNMENT;
    return MOR_OK;
}
// A token matrix: `whole` if 8 elements of it may be taken at once.
mor_status_t check_tokens(const void* m, int64_t tokens, int64_t n, int64_t ld, int dtype, bool& whole)
{
    const int es = (int)dtype_bytes(dtype);
    if (ld < n || (tokens > 0 && m == nullptr)) return MOR_ERR_INVALID_ARG;
    if (!is_aligned(m, es)) return MOR_ERR_ALIGNMENT;
    whole = n % 8 == 0 && access_bytes(m, tokens > 1 ? ld * es : 0, 0, es) >= 16;
    return MOR_OK;
}
bool rank_whole(const void* b, int rank) { return rank <= 16 ? rank % 4 == 0 && is_aligned(b, 8) : rank % 8 == 0 && is_aligned(b, 16); }
mor_status_t status(cudaError_t e) { return e == cudaSuccess ? MOR_OK : MOR_ERR_CUDA; }

}  // namespace
}  // namespace mor

using namespace mor;

extern "C" {

size_t mor_adapter_workspace_bytes(const mor_adapter_desc_t* d, int train)
{
    if (check_adapter(d) != MOR_OK || small_call(*d, train != 0)) return 0;
    return forward_parts(*d, train != 0, nullptr).bytes;
}

mor_status_t mor_adapter_add(const mor_adapter_desc_t* d, const void* x, int64_t ldx, const void* base, int64_t ldb, void* out, int64_t ldo, int dtype, int train,
                             void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    mor_status_t st = check_adapter(d);
    if (st != MOR_OK) return st;
    if (!is_dtype(dtype)) return MOR_ERR_INVALID_ARG;
    bool x_whole, base_whole, out_whole;
    if ((st = check_tokens(x, d->tokens, d->n_in, ldx, MOR_DTYPE_BF16, x_whole)) != MOR_OK) return st;
    if ((st = check_tokens(base, d->tokens, d->n_out, ldb, dtype, base_whole)) != MOR_OK) return st;
    if ((st = check_tokens(out, d->tokens, d->n_out, ldo, dtype, out_whole)) != MOR_OK) return st;
    // pieces of the result that a row ends in are stored element by element
    out_whole = access_bytes(out, d->tokens > 1 ? ldo * (int64_t)dtype_bytes(dtype) : 0, 0, 1) >= 16;
    const bool a_whole = d->n_in % 8 == 0 && is_aligned(d->a, 16), any = !(x_whole && a_whole);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (d->tokens == 0) return MOR_OK;
    if (small_call(*d, train != 0)) {
        SmallParams p = {static_cast<const bf16*>(x), static_cast<const bf16*>(d->a), static_cast<const bf16*>(d->b), d->ids, d->scale, d->factor, d->adapters, d->rank,
                         (int32_t)d->tokens, ldx, d->n_in, d->n_out, base, out, ldb, ldo, rank_whole(d->b, d->rank), base_whole, out_whole};
        const dim3 grid((uint32_t)(d->ids != nullptr ? d->tokens : ceil_div(d->tokens, kSmallRows)) * kMaxCluster);
        return status(by_rank(padded_rank(d->rank), [&](auto r) {
            constexpr int R = decltype(r)::value;
            if (dtype == MOR_DTYPE_BF16)
                return any ? launch_clusters(adapter_small_kernel<R, bf16, true>, grid, 0, kSmallWarps * 32, stream, p)
                           : launch_clusters(adapter_small_kernel<R, bf16, false>, grid, 0, kSmallWarps * 32, stream, p);
            return any ? launch_clusters(adapter_small_kernel<R, float, true>, grid, 0, kSmallWarps * 32, stream, p)
                       : launch_clusters(adapter_small_kernel<R, float, false>, grid, 0, kSmallWarps * 32, stream, p);
        }));
    }
    if (workspace == nullptr || workspace_bytes < mor_adapter_workspace_bytes(d, train)) return MOR_ERR_WORKSPACE;
    if (!is_aligned(workspace, 256)) return MOR_ERR_ALIGNMENT;
    const Forward f = forward_parts(*d, train != 0, workspace);
    if (d->ids != nullptr) {
        st = mor_expert_sort(d->ids, d->tokens, d->adapters, kRows, const_cast<int32_t*>(f.s.starts), const_cast<int32_t*>(f.s.row_of_token),
                             const_cast<int32_t*>(f.s.token_of_row), f.sort, f.sort_bytes, cuda_stream);
        if (st != MOR_OK) return st;
    }
    const int padded = padded_rank(d->rank);
    ShrinkParams sp = {f.s, static_cast<const bf16*>(x), static_cast<const bf16*>(d->a), d->scale, d->factor, ldx, d->n_in, d->n_in, (int64_t)d->rank * d->n_in, d->rank, padded,
                       f.natural, f.turned};
    if (shrink(sp, any, stream) != cudaSuccess) return MOR_ERR_CUDA;
    ExpandParams ep = {f.s, f.natural, static_cast<const bf16*>(d->b), d->n_out, d->rank, (int64_t)d->n_out * d->rank, d->rank, padded, base, out, ldb, ldo, 0, 0,
                       rank_whole(d->b, d->rank), base_whole, out_whole};
    return status(expand(ep, dtype, stream));
}

size_t mor_adapter_grad_workspace_bytes(const mor_adapter_desc_t* d) { return check_adapter(d) != MOR_OK ? 0 : backward_parts(*d, nullptr).bytes; }

mor_status_t mor_adapter_grad(const mor_adapter_desc_t* d, const void* x, int64_t ldx, const void* dy, int64_t lddy, const void* base, int64_t ldb, void* dx, int64_t lddx,
                              void* da, void* db, const void* saved, size_t saved_bytes, void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    mor_status_t st = check_adapter(d);
    if (st != MOR_OK) return st;
    bool x_whole = true, dy_whole, base_whole = true, dx_whole = true;
    if (da != nullptr && (st = check_tokens(x, d->tokens, d->n_in, ldx, MOR_DTYPE_BF16, x_whole)) != MOR_OK) return st;
    if ((st = check_tokens(dy, d->tokens, d->n_out, lddy, MOR_DTYPE_BF16, dy_whole)) != MOR_OK) return st;
    if (dx != nullptr && base != nullptr && (st = check_tokens(base, d->tokens, d->n_in, ldb, MOR_DTYPE_BF16, base_whole)) != MOR_OK) return st;
    if (dx != nullptr && (st = check_tokens(dx, d->tokens, d->n_in, lddx, MOR_DTYPE_BF16, dx_whole)) != MOR_OK) return st;
    if (!is_aligned(da, 2) || !is_aligned(db, 2)) return MOR_ERR_ALIGNMENT;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (d->tokens == 0) {                                          // sums over nothing
        if (da != nullptr && cudaMemsetAsync(da, 0, (size_t)d->adapters * d->rank * d->n_in * 2, stream) != cudaSuccess) return MOR_ERR_CUDA;
        if (db != nullptr && cudaMemsetAsync(db, 0, (size_t)d->adapters * d->rank * d->n_out * 2, stream) != cudaSuccess) return MOR_ERR_CUDA;
        return MOR_OK;
    }
    if (saved == nullptr || saved_bytes < mor_adapter_workspace_bytes(d, 1)) return MOR_ERR_WORKSPACE;
    if (workspace == nullptr || workspace_bytes < mor_adapter_grad_workspace_bytes(d)) return MOR_ERR_WORKSPACE;
    if (!is_aligned(saved, 256) || !is_aligned(workspace, 256)) return MOR_ERR_ALIGNMENT;
    const Forward f = forward_parts(*d, true, const_cast<void*>(saved));
    const Backward w = backward_parts(*d, workspace);
    const int padded = padded_rank(d->rank);
    if (dx != nullptr || da != nullptr) {
        const uint32_t a_ctas = (uint32_t)(ceil_div(padded, 32) * ceil_div(d->n_in, 32)), b_ctas = (uint32_t)(ceil_div(w.wide, 32) * ceil_div(padded, 32));
        TurnParams tp = {static_cast<const bf16*>(d->a), static_cast<const bf16*>(d->b), w.at, w.bt, d->n_in, d->n_out, w.wide, d->rank, padded, a_ctas};
        if (launch_clusters(adapter_turn_kernel, dim3(a_ctas + b_ctas, (uint32_t)d->adapters), 0, 256, stream, tp) != cudaSuccess) return MOR_ERR_CUDA;
        ShrinkParams sp = {f.s, static_cast<const bf16*>(dy), w.bt, d->scale, d->factor, lddy, d->n_out, w.wide, (int64_t)padded * w.wide, padded, padded, w.natural,
                           da != nullptr ? w.turned : nullptr};
        if (shrink(sp, !dy_whole, stream) != cudaSuccess) return MOR_ERR_CUDA;
    }
    if (db != nullptr) {
        OuterParams op = {f.s, f.turned, static_cast<const bf16*>(dy), lddy, d->n_out, d->rank, padded, static_cast<bf16*>(db), 1};
        if (outer(op, !dy_whole, stream) != cudaSuccess) return MOR_ERR_CUDA;
    }
    if (da != nullptr) {
        OuterParams op = {f.s, w.turned, static_cast<const bf16*>(x), ldx, d->n_in, d->rank, padded, static_cast<bf16*>(da), 0};
        if (outer(op, !x_whole, stream) != cudaSuccess) return MOR_ERR_CUDA;
    }
    if (dx != nullptr) {
        dx_whole = access_bytes(dx, d->tokens > 1 ? lddx * 2 : 0, 0, 1) >= 16;
        ExpandParams ep = {f.s, w.natural, w.at, d->n_in, padded, (int64_t)d->n_in * padded, padded, padded, base, dx, ldb, lddx, 0, 0, true, base_whole, dx_whole};
        if (expand(ep, MOR_DTYPE_BF16, stream) != cudaSuccess) return MOR_ERR_CUDA;
    }
    return MOR_OK;
}

}  // extern "C"
