// Low-rank adapters beside a shared projection: out = base + s (x a^T) b^T with an adapter for every token, and the gradients.
//
// The ranks are small, so every product here moves far more than it multiplies: the wide matrices (x, base, out, dy) are read and written once, and
// what has to be kept in flight for that decides the shape of the kernels.  Tiles come by asynchronous copies of 16 bytes into rings of shared memory
// (rows lie wherever the tokens of an adapter are, so the copies are a thread's own and not a tensor map's), fragments from there to the registers of the
// tensor instructions (mma.sync, BF16 in, FP32 sums).
//
//   shrink   h = s x a^T              reduction over the width, cut over a cluster's CTAs and joined through distributed shared memory
//   expand   out = base + h b^T       h as the sum of two BF16 (16 bits and more), in registers while the columns pass
//   outer    db = dy^T h, da = u^T x  reduction over an adapter's tokens, cut and joined like shrink
//   small    shrink and expand of up to 16 tokens of an adapter by one cluster, in one launch, for few tokens
//
// More tokens are sorted by adapter first; each adapter's rows start at a multiple of a tile.  All sums run in an order that depends on the sizes and
// ids alone.
#include "mor_layers.cuh"

namespace mor {
namespace {

using bf16 = __nv_bfloat16;

constexpr int kRows = 32;                 // rows of a warp
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

// ---- tiles in shared memory: rows of ROW_BYTES (32, 64 or 128) whose 16-byte chunks are dealt out so that 8 rows of a chunk lie in distinct banks

template <int ROW_BYTES> __device__ __forceinline__ uint32_t chunk_at(int row, int chunk)
{
    const int turn = ROW_BYTES == 128 ? row & 7 : ROW_BYTES == 64 ? (row >> 1) & 3 : (row >> 2) & 1;
    return (uint32_t)(row * ROW_BYTES + ((chunk ^ turn) << 4));
}
// 16 bytes to shared memory, `bytes` of them from `from`, the others zero.
__device__ __forceinline__ void copy_async(uint32_t to, const void* from, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void store_chunk(uint32_t to, const uint32_t* w)
{
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
}
// 16 bytes of a row of n elements from `at` on (zero past its end, or where there is no row); ANY: the row starts anywhere, and the copy is not asynchronous.
template <typename T, bool ANY> __device__ __forceinline__ void fill_chunk(uint32_t to, const T* row, int64_t at, int64_t n, const void* valid)
{
    constexpr int kElems = 16 / (int)sizeof(T);
    if constexpr (ANY) {
        uint32_t w[4] = {0, 0, 0, 0};
        if (row != nullptr && at < n) load_any<T, 16>(w, row, at, n);
        store_chunk(to, w);
    } else {
        const int64_t left = row != nullptr ? n - at : 0;
        const int bytes = (int)sizeof(T) * (int)max((int64_t)0, min((int64_t)kElems, left));
        copy_async(to, bytes > 0 ? static_cast<const void*>(row + at) : valid, bytes);
    }
}
__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void load_matrices_turned(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t shared_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ float4 load_remote4(uint32_t own, uint32_t rank)
{
    float4 v;
    asm volatile("{ .reg .u32 a; mapa.shared::cluster.u32 a, %4, %5; ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a]; }"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(own), "r"(rank) : "memory");
    return v;
}
// Sum of four neighbouring values over the cluster's CTAs, in their order.
__device__ __forceinline__ float4 sum_remote4(uint32_t own, uint32_t ctas)
{
    float4 v[kMaxCluster];
#pragma unroll
    for (uint32_t c = 0; c < kMaxCluster; ++c) v[c] = c < ctas ? load_remote4(own, c) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (uint32_t c = 1; c < kMaxCluster; ++c) {
        v[0].x += v[c].x;
        v[0].y += v[c].y;
        v[0].z += v[c].z;
        v[0].w += v[c].w;
    }
    return v[0];
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
    int32_t padded;            // rank as the output has it
    bf16* h;                   // [rows][2][padded]
};

// A CTA of 4 warps takes ROWS rows of one adapter (a warp 32 of them, or of 32 rows a quarter of each step's 64 elements) and R of the ranks (blockIdx.y);
// a cluster's CTAs share the reduction axis.
constexpr int kShrinkStages = 4;
template <int R, int ROWS> constexpr int kShrinkSmem = kShrinkStages * (ROWS + R) * 128;

template <int R, int ROWS, bool ANY> __global__ void __launch_bounds__(128) adapter_shrink_kernel(const __grid_constant__ ShrinkParams p)
{
    constexpr int kStage = (ROWS + R) * 128, kTiles = R / 8, kParts = ROWS == kRows ? 4 : 1, kPitch = R + 4;
    static_assert(kParts * ROWS * kPitch * 4 <= kShrinkSmem<R, ROWS>, "the sums take the ring's place");
    extern __shared__ __align__(128) uint8_t ring[];
    wait_for_predecessor();
    const uint32_t rank = cluster_rank(), ctas = cluster_size();
    const int64_t first = (int64_t)(blockIdx.x / ctas) * ROWS;
    if (first >= used_rows(p.s)) return;                                          // the whole cluster
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    const int r0 = blockIdx.y * R, adapter = adapter_of(p.s, first, lane);
    const float scale = (p.scale != nullptr ? p.scale[adapter] : 1.f) * p.factor;
    const uint32_t smem = shared_at(ring);
    // what this thread copies: chunk tid % 8 of every 16th row
    const bf16* xr[ROWS / 16];
    const bf16* mr[R / 16];
#pragma unroll
    for (int i = 0; i < ROWS / 16; ++i) {
        const int32_t t = token_at(p.s, first + i * 16 + (tid >> 3));
        xr[i] = t >= 0 ? p.x + (int64_t)t * p.ldx : nullptr;
    }
#pragma unroll
    for (int i = 0; i < R / 16; ++i) {
        const int r = r0 + i * 16 + (tid >> 3);
        mr[i] = r < p.m_rows ? p.m + (int64_t)adapter * p.m_stride + (int64_t)r * p.ldm : nullptr;
    }
    const int64_t steps = (p.n + 63) / 64, share = (steps + ctas - 1) / ctas, begin = min((int64_t)rank * share, steps), end = min(begin + share, steps);
    auto fill = [&](int64_t step) {
        if (step < end) {
            const uint32_t stage = smem + (uint32_t)((step - begin) % kShrinkStages) * kStage;
            const int64_t at = step * 64 + (tid & 7) * 8;
#pragma unroll
            for (int i = 0; i < ROWS / 16; ++i) fill_chunk<bf16, ANY>(stage + chunk_at<128>(i * 16 + (tid >> 3), tid & 7), xr[i], at, p.n, p.x);
#pragma unroll
            for (int i = 0; i < R / 16; ++i) fill_chunk<bf16, ANY>(stage + ROWS * 128 + chunk_at<128>(i * 16 + (tid >> 3), tid & 7), mr[i], at, p.n, p.x);
        }
        copies_commit();
    };
    float acc[2][kTiles][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < kTiles; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[i][j][k] = 0.f;
#pragma unroll
    for (int s = 0; s < kShrinkStages - 1; ++s) fill(begin + s);
    const int a_row = (ROWS == kRows ? 0 : warp * kRows) + (lane & 15);
    for (int64_t step = begin; step < end; ++step) {
        copies_wait<kShrinkStages - 2>();
        __syncthreads();
        fill(step + kShrinkStages - 1);
        const uint32_t stage = smem + (uint32_t)((step - begin) % kShrinkStages) * kStage, ms = stage + ROWS * 128;
        if constexpr (ROWS == kRows) {
            uint32_t a[2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i) load_matrices(a[i], stage + chunk_at<128>(i * 16 + a_row, warp * 2 + (lane >> 4)));
#pragma unroll
            for (int j = 0; j < kTiles; j += 2) {
                uint32_t b[4];
                load_matrices(b, ms + chunk_at<128>(j * 8 + (lane & 7) + (lane >> 4) * 8, warp * 2 + ((lane >> 3) & 1)));
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    mma(acc[i][j], a[i][0], a[i][1], a[i][2], a[i][3], b[0], b[1]);
                    mma(acc[i][j + 1], a[i][0], a[i][1], a[i][2], a[i][3], b[2], b[3]);
                }
            }
        } else {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t a[2][2][4];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int k = 0; k < 2; ++k) load_matrices(a[i][k], stage + chunk_at<128>(i * 16 + a_row, half * 4 + k * 2 + (lane >> 4)));
#pragma unroll
                for (int j = 0; j < kTiles; ++j) {
                    uint32_t b[4];
                    load_matrices(b, ms + chunk_at<128>(j * 8 + (lane & 7), half * 4 + (lane >> 3)));
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        mma(acc[i][j], a[i][0][0], a[i][0][1], a[i][0][2], a[i][0][3], b[0], b[1]);
                        mma(acc[i][j], a[i][1][0], a[i][1][1], a[i][1][2], a[i][1][3], b[2], b[3]);
                    }
                }
            }
        }
    }
    copies_wait<0>();
    __syncthreads();
    float* part = reinterpret_cast<float*>(ring);                                 // [kParts][ROWS][kPitch]
    {
        float* to = part + (warp * kRows + g) * kPitch + 2 * q;                   // a part's or a warp's 32 rows
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < kTiles; ++j) {
                *reinterpret_cast<float2*>(to + i * 16 * kPitch + j * 8) = make_float2(acc[i][j][0], acc[i][j][1]);
                *reinterpret_cast<float2*>(to + (i * 16 + 8) * kPitch + j * 8) = make_float2(acc[i][j][2], acc[i][j][3]);
            }
    }
    __syncthreads();
    if constexpr (kParts > 1) {
        for (int at = tid; at < ROWS * R / 4; at += 128) {
            float4* to = reinterpret_cast<float4*>(part + at / (R / 4) * kPitch + at % (R / 4) * 4);
            float4 v = *to;
#pragma unroll
            for (int k = 1; k < kParts; ++k) {
                const float4 u = to[k * ROWS * kPitch / 4];
                v.x += u.x;
                v.y += u.y;
                v.z += u.z;
                v.w += u.w;
            }
            *to = v;
        }
    }
    cluster_arrive();
    cluster_wait();
    const int rows = ROWS / (int)ctas;                                            // of each CTA: 1, 2, 4 or 8 divide the tile
    for (int at = tid; at < rows * (R / 4); at += 128) {
        const int row = (int)rank * rows + at / (R / 4), col = at % (R / 4) * 4;
        const float4 v = sum_remote4(shared_at(part + row * kPitch + col), ctas);
        const float f[4] = {v.x * scale, v.y * scale, v.z * scale, v.w * scale};
        bf16 hi[4], lo[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) split(f[k], hi[k], lo[k]);
        uint16_t* to = reinterpret_cast<uint16_t*>(p.h) + (first + row) * 2 * p.padded + r0 + col;
        *reinterpret_cast<ushort4*>(to) = make_ushort4(bits_of(hi[0]), bits_of(hi[1]), bits_of(hi[2]), bits_of(hi[3]));
        *reinterpret_cast<ushort4*>(to + p.padded) = make_ushort4(bits_of(lo[0]), bits_of(lo[1]), bits_of(lo[2]), bits_of(lo[3]));
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
    int32_t share;             // steps of a CTA
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

template <typename T> __device__ void copy_row(const ExpandParams& p, int64_t token, int64_t from, int64_t to, int lane)
{
    const T* base = p.base != nullptr ? static_cast<const T*>(p.base) + token * p.ldb : nullptr;
    T* out = static_cast<T*>(p.out) + token * p.ldo;
    const bool whole = p.base_whole && p.n % kPer == 0;
    for (int64_t at = from + lane * kPer; at < to; at += 32 * kPer) {
        float v[kPer];
        load_base(v, base, at, p.n, whole);
        store_out(v, out, at, p.n, p.out_whole);
    }
}

// A CTA of 4 warps takes ROWS rows of one adapter and walks columns: 64 a step with a warp on 32 of 128 rows, 128 a step with a warp on 32 of them for 32
// rows.  h stays in registers.  The rows of m (a column of the result each) are laid down so that the 8 of an instruction's operand follow each other:
// column c of operand j is column 8 (c / 2) + 2 j + c % 2 of 32, and a thread's results are 8 neighbouring columns.
constexpr int kExpandStages = 3;
template <int ROWS> constexpr int kExpandCols = ROWS == kRows ? 128 : 64;
template <int R, int ROWS, typename T> constexpr int kExpandSmem = kExpandStages * kExpandCols<ROWS> * (ROWS * (int)sizeof(T) + R * 2);

template <int R, int ROWS, typename T, bool ANY> __global__ void __launch_bounds__(128) adapter_expand_kernel(const __grid_constant__ ExpandParams p)
{
    constexpr int kCols = kExpandCols<ROWS>, kBase = kCols * ROWS * (int)sizeof(T), kStage = kBase + kCols * R * 2;
    constexpr int kChunks = 64 * (int)sizeof(T) / 16, kUnits = kCols / 64 * (ROWS == kRows ? 1 : 2);     // of a row's 64 columns; of 32 columns for a warp
    static_assert(kCols == 64 || kUnits == 2, "");
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ int32_t tokens[ROWS];
    wait_for_predecessor();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    const int64_t steps = (p.n + kCols - 1) / kCols, begin = (int64_t)blockIdx.y * p.share, end = min(begin + (int64_t)p.share, steps);
    if (blockIdx.x >= p.row_ctas) {
        const int64_t t0 = (int64_t)(blockIdx.x - p.row_ctas) * 32;
        const uint32_t none = __ballot_sync(0xFFFFFFFFu, t0 + lane < p.s.tokens && p.s.row_of_token[t0 + lane] < 0);
        for (int i = warp; i < 32; i += 4)
            if (none >> i & 1) copy_row<T>(p, t0 + i, begin * kCols, min(end * kCols, p.n), lane);
        return;
    }
    const int64_t first = (int64_t)blockIdx.x * ROWS;
    if (first >= used_rows(p.s)) return;
    const int adapter = adapter_of(p.s, first, lane);
    const bf16* m = p.m + (int64_t)adapter * p.m_stride;
    if (tid < ROWS) tokens[tid] = token_at(p.s, first + tid);
    __syncthreads();
    const uint32_t smem = shared_at(ring);
    const int chunks = p.padded / R;                                              // of the ranks
    auto base_at = [&](int row, int col16) {                                      // a 16-byte piece of the tile: blocks of 64 columns one after the other
        const int block = col16 / kChunks, chunk = col16 % kChunks;
        return (uint32_t)((block * ROWS + row) * (kChunks * 16) + ((chunk ^ ((row & 1) * (kChunks / 2))) << 4));
    };
    auto fill = [&](int64_t turn) {                                               // turn: step and chunk of ranks
        const int64_t step = begin + turn / chunks;
        if (step < end) {
            const int r0 = (int)(turn % chunks) * R;
            const uint32_t stage = smem + (uint32_t)(turn % kExpandStages) * kStage;
            if (p.base != nullptr && r0 == 0) {
                constexpr int kPieces = kCols * (int)sizeof(T) / 16;
#pragma unroll 8
                for (int i = tid; i < ROWS * kPieces; i += 128) {
                    const int row = i / kPieces, c = i % kPieces;
                    const int32_t t = tokens[row];
                    fill_chunk<T, ANY>(stage + base_at(row, c), t >= 0 ? static_cast<const T*>(p.base) + (int64_t)t * p.ldb : nullptr, step * kCols + c * (16 / (int)sizeof(T)), p.n,
                                       p.base);
                }
            }
#pragma unroll 4
            for (int i = tid; i < kCols * R / 8; i += 128) {
                const int c = i / (R / 8), k = i % (R / 8), at = r0 + k * 8;
                const int64_t n = step * kCols + c;
                const int slot = (c & ~31) + ((c >> 1) & 3) * 8 + ((c >> 3) & 3) * 2 + (c & 1);
                const uint32_t to = stage + kBase + chunk_at<R * 2>(slot, k);
                const bf16* row = n < p.n ? m + n * p.ldm : nullptr;
                if (p.m_whole) {
                    fill_chunk<bf16, false>(to, row, at, p.m_cols, p.m);
                } else {
                    uint32_t w[4];
                    load_m<32>(w, row, at, p.m_cols, false);
                    store_chunk(to, w);
                }
            }
        }
        copies_commit();
    };
    const int64_t turns = (end - begin) * chunks;
#pragma unroll
    for (int s = 0; s < kExpandStages - 1; ++s) fill(s);
    const int row0 = ROWS == kRows ? 0 : warp * kRows;
    uint32_t hi[2][R / 16][4], lo[2][R / 16][4];
    auto load_h = [&](int r0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t* h = reinterpret_cast<const uint32_t*>(p.h + (first + row0 + i * 16 + g) * 2 * p.padded + r0) + q;
            const int64_t below = (int64_t)8 * p.padded;                          // 8 rows, in words
#pragma unroll
            for (int k = 0; k < R / 16; ++k) {
                hi[i][k][0] = h[k * 8];
                hi[i][k][1] = h[below + k * 8];
                hi[i][k][2] = h[k * 8 + 4];
                hi[i][k][3] = h[below + k * 8 + 4];
                const uint32_t* l = h + p.padded / 2;
                lo[i][k][0] = l[k * 8];
                lo[i][k][1] = l[below + k * 8];
                lo[i][k][2] = l[k * 8 + 4];
                lo[i][k][3] = l[below + k * 8 + 4];
            }
        }
    };
    if (chunks == 1) load_h(0);
    T* out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int32_t t = tokens[row0 + i * 8 + g];
        out[i] = t >= 0 ? static_cast<T*>(p.out) + (int64_t)t * p.ldo : nullptr;
    }
    float acc[kUnits / (kCols / 64)][2][4][4];                                    // [units of 32 columns of this warp][16 rows][operand]
    constexpr int kMine = kUnits / (kCols / 64);
    for (int64_t turn = 0; turn < turns; ++turn) {
        copies_wait<kExpandStages - 2>();
        __syncthreads();
        fill(turn + kExpandStages - 1);
        const uint32_t stage = smem + (uint32_t)(turn % kExpandStages) * kStage, ms = stage + kBase;
        const int r0 = (int)(turn % chunks) * R;
        const int64_t c0 = (begin + turn / chunks) * kCols;
        if (chunks > 1) load_h(r0);
        // base into the sums, from the first chunk of ranks on
        if (r0 == 0) {
#pragma unroll
            for (int u = 0; u < kMine; ++u) {
                const int c16 = (ROWS == kRows ? warp : u) * (32 * (int)sizeof(T) / 16) + q * (int)sizeof(T) / 2;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v[kPer];
                    if (p.base != nullptr) {
                        Piece<T, kPer * (int)sizeof(T), 16> piece;
#pragma unroll
                        for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
                            const uint4 w = *reinterpret_cast<const uint4*>(ring + (stage - smem) + base_at(row0 + i * 8 + g, c16 + k));
                            piece.w[4 * k] = w.x; piece.w[4 * k + 1] = w.y; piece.w[4 * k + 2] = w.z; piece.w[4 * k + 3] = w.w;
                        }
#pragma unroll
                        for (int k = 0; k < kPer; ++k) v[k] = piece.get(k);
                    } else {
#pragma unroll
                        for (int k = 0; k < kPer; ++k) v[k] = 0.f;
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        acc[u][i >> 1][j][(i & 1) * 2] = v[2 * j];
                        acc[u][i >> 1][j][(i & 1) * 2 + 1] = v[2 * j + 1];
                    }
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kMine; ++u) {
            const int unit = ROWS == kRows ? warp : u;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int slot = unit * 32 + j * 8;
                if constexpr (R == 16) {
                    // two operands of 16 ranks at once would cross j: one, its halves twice
                    uint32_t b[4];
                    load_matrices(b, ms + chunk_at<32>(slot + (lane & 7), (lane >> 3) & 1));
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        mma(acc[u][i][j], hi[i][0][0], hi[i][0][1], hi[i][0][2], hi[i][0][3], b[0], b[1]);
                        mma(acc[u][i][j], lo[i][0][0], lo[i][0][1], lo[i][0][2], lo[i][0][3], b[0], b[1]);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < R / 32; ++k) {
                        uint32_t b[4];
                        load_matrices(b, ms + chunk_at<R * 2>(slot + (lane & 7), k * 4 + (lane >> 3)));
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            mma(acc[u][i][j], hi[i][2 * k][0], hi[i][2 * k][1], hi[i][2 * k][2], hi[i][2 * k][3], b[0], b[1]);
                            mma(acc[u][i][j], hi[i][2 * k + 1][0], hi[i][2 * k + 1][1], hi[i][2 * k + 1][2], hi[i][2 * k + 1][3], b[2], b[3]);
                            mma(acc[u][i][j], lo[i][2 * k][0], lo[i][2 * k][1], lo[i][2 * k][2], lo[i][2 * k][3], b[0], b[1]);
                            mma(acc[u][i][j], lo[i][2 * k + 1][0], lo[i][2 * k + 1][1], lo[i][2 * k + 1][2], lo[i][2 * k + 1][3], b[2], b[3]);
                        }
                    }
                }
            }
        }
        if (r0 + R < p.padded) continue;
#pragma unroll
        for (int u = 0; u < kMine; ++u) {
            const int64_t at = c0 + (ROWS == kRows ? warp : u) * 32 + q * 8;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (out[i] == nullptr) continue;
                float v[kPer];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[2 * j] = acc[u][i >> 1][j][(i & 1) * 2];
                    v[2 * j + 1] = acc[u][i >> 1][j][(i & 1) * 2 + 1];
                }
                store_out(v, out[i], at, p.n, p.out_whole);
            }
        }
    }
    copies_wait<0>();
}

// Fragments of 16 rows of h in registers, for the slots that load_m() gives a thread.
template <int R> struct HFrags {
    uint32_t a[R / 16][4];
};
// 32 columns from c0 on of 16 rows, straight from memory: acc += h m^T.  Ranks are dealt to the instructions' slots so that a thread's are neighbours
// (both operands agree, which is all that a reduction asks for).
template <int R> struct Columns {
    uint32_t w[4][R / 8];
    __device__ __forceinline__ void load(const bf16* m, int64_t c0, int64_t n, int64_t ldm, int cols, bool whole, int g, int q)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t c = c0 + 8 * (g >> 1) + 2 * j + (g & 1);
            const bf16* row = c < n ? m + c * ldm : nullptr;
            if constexpr (R == 16) load_m<R>(w[j], row, q * 4, cols, whole);
            else
#pragma unroll
                for (int k = 0; k < R / 32; ++k) load_m<R>(w[j] + 4 * k, row, k * 32 + q * 8, cols, whole);
        }
    }
    __device__ __forceinline__ void add(float (&acc)[4][4], const HFrags<R>& hi, const HFrags<R>& lo) const
    {
#pragma unroll
        for (int k = 0; k < R / 16; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                mma(acc[j], hi.a[k][0], hi.a[k][1], hi.a[k][2], hi.a[k][3], w[j][2 * k], w[j][2 * k + 1]);
                mma(acc[j], lo.a[k][0], lo.a[k][1], lo.a[k][2], lo.a[k][3], w[j][2 * k], w[j][2 * k + 1]);
            }
    }
};

// -------------------------------------------------------------------------------------------- outer ----

struct OuterParams {
    Sorted s;
    const bf16* h;             // [rows][2][padded]
    const bf16* z;             // [tokens, ldz], n wide
    int64_t ldz, n;
    int32_t rank, padded;
    bf16* out;                 // [adapters][rank][n], or [adapters][n][rank]
};

// R ranks x 256 columns of an adapter by 8 warps, 64 columns each, half of them on the first 32 of each step's 64 rows, half on the others.  The reduction runs over
// the adapter's rows, cut over a cluster's CTAs.  Both operands have the reduction axis outside and are turned as they are read from shared memory.
constexpr int kOuterStages = 4, kOuterCols = 256, kOuterRows = 64;
template <int R> constexpr int kOuterStage = kOuterRows * (kOuterCols + 2 * R) * 2;
template <int R> constexpr int kOuterSmem = kOuterStages * kOuterStage<R>;

template <int R, bool BY_COLUMN, bool ANY> __global__ void __launch_bounds__(256) adapter_outer_kernel(const __grid_constant__ OuterParams p)
{
    constexpr int kTiles = R / 16, kHalf = kOuterRows * R * 2;                    // bytes of h's high parts
    constexpr int kPitch = (BY_COLUMN ? R : kOuterCols) + 4, kLines = BY_COLUMN ? kOuterCols : R, kLine = BY_COLUMN ? R : kOuterCols;
    static_assert(kLines * kPitch * 4 <= kOuterSmem<R>, "the sums take the ring's place");
    extern __shared__ __align__(128) uint8_t ring[];
    wait_for_predecessor();
    const uint32_t rank = cluster_rank(), ctas = cluster_size();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    const int chunks = p.padded / R, adapter = blockIdx.z / chunks, r0 = blockIdx.z % chunks * R;
    const int64_t c0 = (int64_t)blockIdx.y * kOuterCols;
    const int64_t from = p.s.starts != nullptr ? p.s.starts[adapter] : 0, to = p.s.starts != nullptr ? p.s.starts[adapter + 1] : adapter == 0 ? p.s.rows : 0;
    const uint32_t smem = shared_at(ring);
    const int64_t steps = (to - from + kOuterRows - 1) / kOuterRows, share = (steps + ctas - 1) / ctas, begin = min((int64_t)rank * share, steps), end = min(begin + share, steps);
    // a thread copies chunk lane of every 8th row; the tokens of a step's rows are looked up a step ahead
    int32_t ahead[8];
    auto look = [&](int64_t step) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t row = from + step * kOuterRows + i * 8 + warp;
            ahead[i] = step < end && row < to ? token_at(p.s, row) : -1;
        }
    };
    auto fill = [&](int64_t step) {
        if (step < end) {
            const uint32_t stage = smem + (uint32_t)((step - begin) % kOuterStages) * kOuterStage<R>;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                fill_chunk<bf16, ANY>(stage + (lane >> 3) * (kOuterRows * 128) + chunk_at<128>(i * 8 + warp, lane & 7), ahead[i] >= 0 ? p.z + (int64_t)ahead[i] * p.ldz : nullptr,
                                      c0 + lane * 8, p.n, p.z);
            const uint32_t hs = stage + kOuterRows * kOuterCols * 2;
#pragma unroll
            for (int i = tid; i < kOuterRows * R / 4; i += 256) {
                const int row = i / (R / 4), c = i % (R / 4), part = c / (R / 8), chunk = c % (R / 8);
                const int64_t at = from + step * kOuterRows + row;
                fill_chunk<bf16, false>(hs + part * kHalf + chunk_at<R * 2>(row, chunk), at < to ? p.h + at * 2 * p.padded + part * p.padded : nullptr, r0 + chunk * 8, p.padded, p.h);
            }
        }
        copies_commit();
        look(step + 1);
    };
    float acc[kTiles][8][4];
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[i][j][k] = 0.f;
    look(begin);
#pragma unroll
    for (int s = 0; s < kOuterStages - 1; ++s) fill(begin + s);
    const int block = warp & 3, row0 = (warp >> 2) * 32;
    for (int64_t step = begin; step < end; ++step) {
        copies_wait<kOuterStages - 2>();
        __syncthreads();
        fill(step + kOuterStages - 1);
        const uint32_t stage = smem + (uint32_t)((step - begin) % kOuterStages) * kOuterStage<R>, zs = stage + block * (kOuterRows * 128), hs = stage + kOuterRows * kOuterCols * 2;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint32_t b[4][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) load_matrices_turned(b[j], zs + chunk_at<128>(row0 + k * 16 + (lane & 15), j * 2 + (lane >> 4)));
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    uint32_t a[4];
                    load_matrices_turned(a, hs + part * kHalf + chunk_at<R * 2>(row0 + k * 16 + (lane & 7) + (lane >> 4) * 8, i * 2 + ((lane >> 3) & 1)));
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        mma(acc[i][2 * j], a[0], a[1], a[2], a[3], b[j][0], b[j][1]);
                        mma(acc[i][2 * j + 1], a[0], a[1], a[2], a[3], b[j][2], b[j][3]);
                    }
                }
        }
    }
    copies_wait<0>();
    __syncthreads();
    float* part = reinterpret_cast<float*>(ring);                                 // [kLines][kPitch]
#pragma unroll 1
    for (int turn = 0; turn < 2; ++turn) {
        if (warp >> 2 == turn) {
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int r = i * 16 + (k >> 1) * 8 + g, c = block * 64 + j * 8 + 2 * q + (k & 1);
                        float* at = part + (BY_COLUMN ? c * kPitch + r : r * kPitch + c);
                        *at = turn > 0 ? *at + acc[i][j][k] : acc[i][j][k];
                    }
        }
        __syncthreads();
    }
    cluster_arrive();
    cluster_wait();
    bf16* out = p.out + (int64_t)adapter * p.rank * p.n;
    const int lines = kLines / (int)ctas;
    for (int at = tid; at < lines * (kLine / 4); at += 256) {
        const int line = (int)rank * lines + at / (kLine / 4), e = at % (kLine / 4) * 4;
        const float4 v = sum_remote4(shared_at(part + line * kPitch + e), ctas);
        const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int r = r0 + (BY_COLUMN ? e + k : line);
            const int64_t c = c0 + (BY_COLUMN ? line : e + k);
            if (r < p.rank && c < p.n) out[BY_COLUMN ? c * p.rank + r : (int64_t)r * p.n + c] = __float2bfloat16(f[k]);
        }
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
    Columns<R> cols;
    float v0[kPer], v1[kPer];
    int64_t step = c_first + warp;
    auto fetch = [&] {
        if (step >= c_last) return;
        cols.load(b, step * 32, p.n_out, p.rank, p.rank, p.b_whole, g, q);
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
    HFrags<R> hi, lo;
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
            hi.a[k][i] = (uint32_t)bits_of(h0) | (uint32_t)bits_of(h1) << 16;
            lo.a[k][i] = (uint32_t)bits_of(l0) | (uint32_t)bits_of(l1) << 16;
        }
    while (step < c_last) {
        float sum[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[j][k] = 0.f;
        cols.add(sum, hi, lo);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v0[2 * j] += sum[j][0];
            v0[2 * j + 1] += sum[j][1];
            v1[2 * j] += sum[j][2];
            v1[2 * j + 1] += sum[j][3];
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
cudaError_t launch_clusters(void (*kernel)(P...), dim3 grid, uint32_t cluster, uint32_t block, size_t smem, cudaStream_t st, A&&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
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

// Rows of a tile.  128 where there are tokens for it: enough to fill the GPU with such tiles, and as many for an adapter that the rows left empty at its end (64 on
// average) cost less than what smaller tiles read again of the adapters.
int tile_rows(const mor_adapter_desc_t& d) { return d.tokens >= 2048 && d.tokens >= 256 * (int64_t)d.adapters ? 128 : kRows; }
int64_t sorted_rows(const mor_adapter_desc_t& d)
{
    return d.ids != nullptr ? mor_expert_rows(d.tokens, d.adapters, tile_rows(d)) : up(d.tokens, tile_rows(d));
}

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
    bf16* h;
    size_t bytes;
};
Forward forward_parts(const mor_adapter_desc_t& d, void* workspace)
{
    Forward f = {};
    Parts parts = {static_cast<uint8_t*>(workspace)};
    f.s.tokens = d.tokens;
    f.s.adapters = d.adapters;
    f.s.rows = sorted_rows(d);
    if (d.ids != nullptr) {
        f.s.starts = static_cast<int32_t*>(parts.take((size_t)(d.adapters + 1) * 4));
        f.s.row_of_token = static_cast<int32_t*>(parts.take((size_t)d.tokens * 4));
        f.s.token_of_row = static_cast<int32_t*>(parts.take((size_t)f.s.rows * 4));
        f.sort_bytes = mor_expert_workspace_bytes(d.tokens, d.adapters);
        f.sort = parts.take(f.sort_bytes);
    }
    f.h = static_cast<bf16*>(parts.take((size_t)f.s.rows * 2 * padded_rank(d.rank) * 2));
    f.bytes = parts.used;
    return f;
}
struct Backward {
    bf16 *u, *at, *bt;
    int64_t wide;
    size_t bytes;
};
Backward backward_parts(const mor_adapter_desc_t& d, void* workspace)
{
    Backward f = {};
    Parts parts = {static_cast<uint8_t*>(workspace)};
    const int pad = padded_rank(d.rank);
    f.wide = up(d.n_out, 8);
    f.u = static_cast<bf16*>(parts.take((size_t)sorted_rows(d) * 2 * pad * 2));
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

constexpr int64_t kResident = 148 * 2;       // CTAs that the GPU holds of the larger shapes

// Allows the kernel its shared memory and launches it.
template <typename K, typename P> cudaError_t launch_ring(K kernel, std::atomic<uint64_t>& done, int smem, dim3 grid, uint32_t cluster, uint32_t block, cudaStream_t st, const P& p)
{
    if (!allow_smem(kernel, smem, done)) return cudaErrorUnknown;
    return launch_clusters(kernel, grid, cluster, block, (size_t)smem, st, p);
}

template <int R, int ROWS, bool ANY> cudaError_t shrink_launch(const ShrinkParams& p, cudaStream_t st)
{
    static std::atomic<uint64_t> done{0};
    const int64_t tiles = p.s.rows / ROWS, steps = (p.n + 63) / 64;
    const uint32_t chunks = (uint32_t)(p.padded / R);
    uint32_t cluster = 1;                     // as many CTAs to a tile as the GPU holds at once, two steps each at least
    while (cluster < kMaxCluster && tiles * chunks * cluster * 2 <= kResident && steps >= 4 * cluster) cluster *= 2;
    return launch_ring(adapter_shrink_kernel<R, ROWS, ANY>, done, kShrinkSmem<R, ROWS>, dim3((uint32_t)tiles * cluster, chunks), cluster, 128, st, p);
}
cudaError_t shrink(const ShrinkParams& p, int rows, bool any, cudaStream_t st)
{
    return by_rank(p.padded > 64 ? 64 : p.padded, [&](auto r) {
        constexpr int R = decltype(r)::value;
        if (rows == kRows) return any ? shrink_launch<R, kRows, true>(p, st) : shrink_launch<R, kRows, false>(p, st);
        return any ? shrink_launch<R, 128, true>(p, st) : shrink_launch<R, 128, false>(p, st);
    });
}

template <int R, int ROWS, typename T, bool ANY> cudaError_t expand_launch(ExpandParams p, cudaStream_t st)
{
    static std::atomic<uint64_t> done{0};
    p.row_ctas = (uint32_t)(p.s.rows / ROWS);
    const int64_t steps = (p.n + kExpandCols<ROWS> - 1) / kExpandCols<ROWS>;
    // as many CTAs as the GPU holds at once
    int64_t across = std::max<int64_t>(1, std::min<int64_t>(steps, kResident / std::max<uint32_t>(1, p.row_ctas)));
    p.share = (int32_t)((steps + across - 1) / across);
    across = (steps + p.share - 1) / p.share;
    const uint32_t copies = p.s.starts != nullptr ? (uint32_t)(up(p.s.tokens, 32) / 32) : 0;
    return launch_ring(adapter_expand_kernel<R, ROWS, T, ANY>, done, kExpandSmem<R, ROWS, T>, dim3(p.row_ctas + copies, (uint32_t)across), 0, 128, st, p);
}
template <typename T> cudaError_t expand_rows(const ExpandParams& p, int rows, cudaStream_t st)
{
    const bool any = p.base != nullptr && !p.base_whole;
    return by_rank(p.padded > 64 ? 64 : p.padded, [&](auto r) {
        constexpr int R = decltype(r)::value;
        if (rows == kRows) return any ? expand_launch<R, kRows, T, true>(p, st) : expand_launch<R, kRows, T, false>(p, st);
        return any ? expand_launch<R, 128, T, true>(p, st) : expand_launch<R, 128, T, false>(p, st);
    });
}
cudaError_t expand(const ExpandParams& p, int rows, int dtype, cudaStream_t st)
{
    return dtype == MOR_DTYPE_BF16 ? expand_rows<bf16>(p, rows, st) : expand_rows<float>(p, rows, st);
}

template <int R, bool BY_COLUMN, bool ANY> cudaError_t outer_launch(const OuterParams& p, cudaStream_t st)
{
    static std::atomic<uint64_t> done{0};
    const uint32_t across = (uint32_t)((p.n + kOuterCols - 1) / kOuterCols), deep = (uint32_t)(p.s.adapters * (p.padded / R));
    const int64_t mean = p.s.rows / p.s.adapters;      // two steps each at least, going by the adapters' mean
    uint32_t cluster = 1;
    while (cluster < kMaxCluster && (int64_t)across * deep * cluster * 2 <= kResident && mean >= 4 * kOuterRows * (int64_t)cluster) cluster *= 2;
    return launch_ring(adapter_outer_kernel<R, BY_COLUMN, ANY>, done, kOuterSmem<R>, dim3(cluster, across, deep), cluster, 256, st, p);
}
cudaError_t outer(const OuterParams& p, bool by_column, bool any, cudaStream_t st)
{
    return by_rank(p.padded > 64 ? 64 : p.padded, [&](auto r) {
        constexpr int R = decltype(r)::value;
        if (by_column) return any ? outer_launch<R, true, true>(p, st) : outer_launch<R, true, false>(p, st);
        return any ? outer_launch<R, false, true>(p, st) : outer_launch<R, false, false>(p, st);
    });
}

mor_status_t check_adapter(const mor_adapter_desc_t* d)
{
    if (d == nullptr || d->tokens < 0 || d->tokens >= (1ll << 30) || d->n_in < 1 || d->n_out < 1 || d->n_in > kMaxWidth || d->n_out > kMaxWidth) return MOR_ERR_INVALID_ARG;
    if (d->adapters < 1 || d->adapters >= MOR_MAX_GROUPS || d->rank < 1 || d->rank > MOR_MAX_RANK) return MOR_ERR_INVALID_ARG;
    if (d->a == nullptr || d->b == nullptr) return MOR_ERR_INVALID_ARG;
    if (sorted_rows(*d) < 0) return MOR_ERR_INVALID_ARG;
    if (!is_aligned(d->a, 2) || !is_aligned(d->b, 2) || !is_aligned(d->ids, 4) || !is_aligned(d->scale, 4)) return MOR_ERR_ALIGNMENT;
    return MOR_OK;
}
// A token matrix: `whole` if its rows start on 16 bytes.
mor_status_t check_tokens(const void* m, int64_t tokens, int64_t n, int64_t ld, int dtype, bool& whole)
{
    const int es = (int)dtype_bytes(dtype);
    if (ld < n || (tokens > 0 && m == nullptr)) return MOR_ERR_INVALID_ARG;
    if (!is_aligned(m, es)) return MOR_ERR_ALIGNMENT;
    whole = access_bytes(m, tokens > 1 ? ld * es : 0, 0, es) >= 16;
    return MOR_OK;
}
mor_status_t status(cudaError_t e) { return e == cudaSuccess ? MOR_OK : MOR_ERR_CUDA; }

}  // namespace
}  // namespace mor

using namespace mor;

extern "C" {

size_t mor_adapter_workspace_bytes(const mor_adapter_desc_t* d, int train)
{
    if (check_adapter(d) != MOR_OK || small_call(*d, train != 0)) return 0;
    return forward_parts(*d, nullptr).bytes;
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
    const bool a_whole = d->n_in % 8 == 0 && is_aligned(d->a, 16), any = !(x_whole && a_whole);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (d->tokens == 0) return MOR_OK;
    if (small_call(*d, train != 0)) {
        SmallParams p = {static_cast<const bf16*>(x), static_cast<const bf16*>(d->a), static_cast<const bf16*>(d->b), d->ids, d->scale, d->factor, d->adapters, d->rank,
                         (int32_t)d->tokens, ldx, d->n_in, d->n_out, base, out, ldb, ldo, d->rank <= 16 ? d->rank % 4 == 0 && is_aligned(d->b, 8) : d->rank % 8 == 0 && is_aligned(d->b, 16),
                         base_whole && d->n_out % kPer == 0, out_whole};
        const dim3 grid((uint32_t)(d->ids != nullptr ? d->tokens : ceil_div(d->tokens, kSmallRows)) * kMaxCluster);
        return status(by_rank(padded_rank(d->rank), [&](auto r) {
            constexpr int R = decltype(r)::value;
            if (dtype == MOR_DTYPE_BF16)
                return any ? launch_clusters(adapter_small_kernel<R, bf16, true>, grid, 0, kSmallWarps * 32, 0, stream, p)
                           : launch_clusters(adapter_small_kernel<R, bf16, false>, grid, 0, kSmallWarps * 32, 0, stream, p);
            return any ? launch_clusters(adapter_small_kernel<R, float, true>, grid, 0, kSmallWarps * 32, 0, stream, p)
                       : launch_clusters(adapter_small_kernel<R, float, false>, grid, 0, kSmallWarps * 32, 0, stream, p);
        }));
    }
    if (workspace == nullptr || workspace_bytes < mor_adapter_workspace_bytes(d, train)) return MOR_ERR_WORKSPACE;
    if (!is_aligned(workspace, 256)) return MOR_ERR_ALIGNMENT;
    const Forward f = forward_parts(*d, workspace);
    const int rows = tile_rows(*d);
    if (d->ids != nullptr) {
        st = mor_expert_sort(d->ids, d->tokens, d->adapters, rows, const_cast<int32_t*>(f.s.starts), const_cast<int32_t*>(f.s.row_of_token),
                             const_cast<int32_t*>(f.s.token_of_row), f.sort, f.sort_bytes, cuda_stream);
        if (st != MOR_OK) return st;
    }
    const int padded = padded_rank(d->rank);
    ShrinkParams sp = {f.s, static_cast<const bf16*>(x), static_cast<const bf16*>(d->a), d->scale, d->factor, ldx, d->n_in, d->n_in, (int64_t)d->rank * d->n_in, d->rank, padded, f.h};
    if (shrink(sp, rows, any, stream) != cudaSuccess) return MOR_ERR_CUDA;
    ExpandParams ep = {f.s, f.h, static_cast<const bf16*>(d->b), d->n_out, d->rank, (int64_t)d->n_out * d->rank, d->rank, padded, base, out, ldb, ldo, 0, 0,
                       d->rank % 8 == 0 && is_aligned(d->b, 16), base_whole, out_whole};
    return status(expand(ep, rows, dtype, stream));
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
    const Forward f = forward_parts(*d, const_cast<void*>(saved));
    const int rows = tile_rows(*d);
    const Backward w = backward_parts(*d, workspace);
    const int padded = padded_rank(d->rank);
    if (dx != nullptr || da != nullptr) {
        const uint32_t a_ctas = (uint32_t)(ceil_div(padded, 32) * ceil_div(d->n_in, 32)), b_ctas = (uint32_t)(ceil_div(w.wide, 32) * ceil_div(padded, 32));
        TurnParams tp = {static_cast<const bf16*>(d->a), static_cast<const bf16*>(d->b), w.at, w.bt, d->n_in, d->n_out, w.wide, d->rank, padded, a_ctas};
        if (launch_clusters(adapter_turn_kernel, dim3(a_ctas + b_ctas, (uint32_t)d->adapters), 0, 256, 0, stream, tp) != cudaSuccess) return MOR_ERR_CUDA;
        ShrinkParams sp = {f.s, static_cast<const bf16*>(dy), w.bt, d->scale, d->factor, lddy, d->n_out, w.wide, (int64_t)padded * w.wide, padded, padded, w.u};
        if (shrink(sp, rows, !dy_whole, stream) != cudaSuccess) return MOR_ERR_CUDA;
    }
    if (db != nullptr) {
        OuterParams op = {f.s, f.h, static_cast<const bf16*>(dy), lddy, d->n_out, d->rank, padded, static_cast<bf16*>(db)};
        if (outer(op, true, !dy_whole, stream) != cudaSuccess) return MOR_ERR_CUDA;
    }
    if (da != nullptr) {
        OuterParams op = {f.s, w.u, static_cast<const bf16*>(x), ldx, d->n_in, d->rank, padded, static_cast<bf16*>(da)};
        if (outer(op, false, !x_whole, stream) != cudaSuccess) return MOR_ERR_CUDA;
    }
    if (dx != nullptr) {
        ExpandParams ep = {f.s, w.u, w.at, d->n_in, padded, (int64_t)d->n_in * padded, padded, padded, base, dx, ldb, lddx, 0, 0, true, base_whole, dx_whole};
        if (expand(ep, rows, MOR_DTYPE_BF16, stream) != cudaSuccess) return MOR_ERR_CUDA;
    }
    return MOR_OK;
}

}  // extern "C"
