// Low-rank adapters beside a shared projection: out = base + s (x a^T) b^T with an adapter for every token, and the gradients.
//
// The ranks are small, so every product here moves far more than it multiplies: the wide matrices (x, base, out, dy) are read and written once by each
// kernel, and what has to be kept in flight for that decides the shape of the kernels.  Tiles come by asynchronous copies of 16 bytes into rings of shared memory
// (rows lie wherever the tokens of an adapter are, so the copies are a thread's own and not a tensor map's).
//
// Tiles of 128 rows (and every `outer`) go through the fifth-generation tensor cores, whose operands stay in shared memory and whose sums are in tensor
// memory: by mma.sync the products of 64 ranks took longer than the memory does (8192 tokens, 4096 -> 4096, rank 64, training: 308 us, 141 now, of which the bytes
// take 53).  Where an adapter has few rows, tiles of 32 by mma.sync (BF16 in, FP32 sums) leave less empty.
//
//   shrink   h = s x a^T              reduction over the width, cut over a cluster's CTAs and joined through distributed shared memory
//   expand   out = base + h b^T       h as the sum of two BF16 (16 bits and more), kept while the columns pass
//   outer    db = dy^T h, da = u^T x  reduction over an adapter's tokens, cut and joined like shrink
//   small    shrink and expand of up to 16 tokens of an adapter by one cluster, in one launch, for few tokens
//
// More tokens are sorted by adapter first; each adapter's rows start at a multiple of a tile.  All sums run in an order that depends on the sizes and
// ids alone.
#include "../fp4/mor_tcgen05.cuh"
#include "../mor_internal.h"
#include "mor_layers.cuh"

namespace mor {
namespace {

using bf16 = __nv_bfloat16;

constexpr int kRows = 32;                 // rows of a warp
constexpr int kMaxCluster = 8;
constexpr int kSmallRows = 16;            // tokens of a cluster in the small kernel
constexpr int kSmallWarps = 8;
constexpr int64_t kMaxWidth = 1 << 21;    // of the token matrices: what the grids hold
constexpr int64_t kSmallTokens = 256;     // most tokens that the small kernel could take

// d += a b for 16 x 16 by 16 x 8.
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t a0, const uint32_t a1, const uint32_t a2, const uint32_t a3, const uint32_t b0, const uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
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
// v as the sum of two BF16; a value that is not finite is the first alone.  An infinite factor of both gives NaN where the second is zero or of the other sign: kept so,
// since a second part that always has the first's sign would be a bit shorter for all values.
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
// 16 bytes each of N rows that start anywhere, `at` elements on, of rows of n elements (zero past their ends, or where there is no row): all loads are on their
// way before the first is put in place.  What reaches past a row's ends goes element by element.
template <typename T, int N, typename Row, typename Place> __device__ __forceinline__ void fill_shifted(Row row, int64_t at, int64_t n, Place place)
{
    constexpr int kElems = 16 / (int)sizeof(T);
    uint4 lo[N], hi[N];
    uint32_t inside = 0;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const T* r = row(k);
        lo[k] = hi[k] = make_uint4(0, 0, 0, 0);
        const int phase = phase_of(r + at);
        if (r != nullptr && at >= phase && at - phase + kElems + (phase != 0 ? kElems : 0) <= n) {
            inside |= 1u << k;
            const uint4* from = reinterpret_cast<const uint4*>(r + at - phase);
            lo[k] = from[0];
            if (phase != 0) hi[k] = from[1];
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const T* r = row(k);
        uint32_t w[4] = {0, 0, 0, 0};
        if (inside >> k & 1) {
            const uint32_t bytes = (uint32_t)phase_of(r + at) * (uint32_t)sizeof(T);
            uint32_t v[8] = {lo[k].x, lo[k].y, lo[k].z, lo[k].w, hi[k].x, hi[k].y, hi[k].z, hi[k].w};
#pragma unroll
            for (int i = 0; i < 6; ++i) v[i] = bytes & 8u ? v[i + 2] : v[i];
#pragma unroll
            for (int i = 0; i < 5; ++i) v[i] = bytes & 4u ? v[i + 1] : v[i];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = sizeof(T) == 4 ? v[i] : __funnelshift_r(v[i], v[i + 1], (bytes & 2u) * 8u);
        } else if (r != nullptr && at < n) {
            load_any<T, 16>(w, r, at, n);
        }
        store_chunk(place(k), w);
    }
}
// The same chunk of N rows, N of them a thread's, copied step by step along the rows: what does not change from step to step is worked out once (the copies
// of a tile are most of a step's instructions, and few warps run them).
template <typename T, int N, bool ANY> struct RowCopies {
    const T* row[N];           // from the thread's chunk on
    uint32_t present;
    __device__ __forceinline__ void set(int k, const T* r, int64_t at, const void* valid)
    {
        if (k == 0) present = 0;
        if (r != nullptr) present |= 1u << k;
        row[k] = r != nullptr ? r + at : static_cast<const T*>(valid);
    }
    // To `to` and every `apart` bytes from there.  `at`: elements since the first step; `left`: from the chunk's place now to the row's end; `first`: from where the
    // rows start to the chunk
    __device__ __forceinline__ void copy(uint32_t to, uint32_t apart, int64_t at, int left, int first) const
    {
        constexpr int kElems = 16 / (int)sizeof(T);
        if constexpr (ANY) {
            fill_shifted<T, N>([&](int k) { return (present >> k & 1) && left > 0 ? row[k] - first : nullptr; }, first + at, first + at + left, [&](int k) { return to + k * apart; });
        } else {
            const int bytes = (int)sizeof(T) * max(0, min(kElems, left));
#pragma unroll
            for (int k = 0; k < N; ++k) copy_async(to + k * apart, row[k] + at, (present >> k & 1) ? bytes : 0);
        }
    }
};
__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
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

// ---- the fifth-generation tensor cores, BF16

// Bounds of the waits: one that takes longer is given up, and the status word says so.  A test makes one run out: the CTA `skip` does not announce its first
// products.
struct Waits {
    uint32_t* status;
    long long cycles;
    uint32_t skip;
};

// Rows of ROW_BYTES laid down by chunk_at<ROW_BYTES>(), the reduction axis along the rows (K) or across them.  Groups of 8 rows are one after the
// other; `next`: bytes between pieces of 64 columns (operands whose rows are the reduction axis and that are wider than that).
template <int ROW_BYTES> __device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t next = 16)
{
    constexpr uint64_t kSwizzle = ROW_BYTES == 128 ? 2 : ROW_BYTES == 64 ? 4 : 6;
    return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)(next >> 4) << 16) | ((uint64_t)(ROW_BYTES * 8 >> 4) << 32) | (1ull << 46) | (kSwizzle << 61);
}
// BF16 x BF16 into FP32, 128 x n; across: the reduction axis runs across both operands' rows.
__host__ __device__ constexpr uint32_t product(int n, bool across) { return (1u << 4) | (1u << 7) | (1u << 10) | (across ? 3u << 15 : 0u) | ((uint32_t)(n >> 3) << 17) | (8u << 24); }
__device__ __forceinline__ void mma_bf16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate)
{
    const uint32_t acc = accumulate;
    asm volatile("{ .reg .pred p; setp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
// Lanes 16 i .. 16 i + 15 of a warp's and 32 columns, as the results of mma.sync lie: r[4 j + k] is row lane / 4 + 8 (k / 2), column 8 j + 2 (lane % 4) + k % 2.
__device__ __forceinline__ void tmem_load_frags(float (&r)[4][4], uint32_t addr)
{
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=f"(r[0][0]), "=f"(r[0][1]), "=f"(r[0][2]), "=f"(r[0][3]), "=f"(r[1][0]), "=f"(r[1][1]), "=f"(r[1][2]), "=f"(r[1][3]), "=f"(r[2][0]), "=f"(r[2][1]), "=f"(r[2][2]),
                   "=f"(r[2][3]), "=f"(r[3][0]), "=f"(r[3][1]), "=f"(r[3][2]), "=f"(r[3][3])
                 : "r"(addr));
}
struct Products {
    uint64_t done[8];          // a stage's (or an accumulator set's) products are through
    uint32_t tmem;
};
// Before wait_for_predecessor(), which lets the next kernel start: that one may then take what is left of tensor memory, but nothing that this one still needs.
__device__ __forceinline__ void products_begin(Products& c, uint32_t columns)
{
    if (threadIdx.x == 0) {
        for (int i = 0; i < 8; ++i) mbar_init(&c.done[i], 1);
        fence_mbar_init();
    }
    if (threadIdx.x < 32) tmem_alloc<1>(&c.tmem, columns);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
}
__device__ __forceinline__ void products_end(const Products& c, uint32_t columns, bool given_up = false)
{
    if (given_up)                                     // whatever still runs in tensor memory: long enough for all of it
        for (const long long t0 = clock64(); clock64() - t0 < 400000;) {}
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x < 32) {
        tc_fence_after();
        tmem_free<1>(c.tmem, columns);
    }
}
// For all threads: the products that were the n-th to be committed to this barrier (from 0) are through.
__device__ __forceinline__ void products_wait(Products& c, int which, uint32_t n, const Waits& w, bool& given_up)
{
    if (given_up) return;
    if (!mbar_wait(&c.done[which], n & 1u, nullptr, w.cycles)) {
        given_up = true;
        if (w.status != nullptr) atomicExch(w.status, (uint32_t)MOR_ERR_TIMEOUT);
    }
}
// For the thread that issued them: the products so far are the step's.
__device__ __forceinline__ void products_commit(Products& c, int which, int32_t step, const Waits& w)
{
    if (step > 0 || blockIdx.x != w.skip) tc_commit<1>(shared_at(&c.done[which]));
}

// Joins the rows' sums over the cluster's CTAs and stores them as pairs of BF16.  part: [rows][R + 4], of this CTA; there: a bit for every row that has a token.
// What is past the ranks that there are, and rows without a token, are zero whatever x and m hold (zero times infinity).
template <int R>
__device__ __forceinline__ void join_rows(float* part, const uint32_t* there, int rows, int64_t first, int r0, float scale, bf16* h, int padded, int ranks, uint32_t rank, uint32_t ctas)
{
    constexpr int kPitch = R + 4;
    cluster_arrive();
    cluster_wait();
    rows /= (int)ctas;                                                            // of each CTA: 1, 2, 4 or 8 divide the tile
    for (int at = threadIdx.x; at < rows * (R / 4); at += blockDim.x) {
        const int row = (int)rank * rows + at / (R / 4), col = at % (R / 4) * 4;
        const float4 v = sum_remote4(shared_at(part + row * kPitch + col), ctas);
        const float f[4] = {v.x * scale, v.y * scale, v.z * scale, v.w * scale};
        bf16 hi[4], lo[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) split((there[row >> 5] >> (row & 31) & 1u) != 0 && r0 + col + k < ranks ? f[k] : 0.f, hi[k], lo[k]);
        uint16_t* to = reinterpret_cast<uint16_t*>(h) + (first + row) * 2 * padded + r0 + col;
        *reinterpret_cast<ushort4*>(to) = make_ushort4(bits_of(hi[0]), bits_of(hi[1]), bits_of(hi[2]), bits_of(hi[3]));
        *reinterpret_cast<ushort4*>(to + padded) = make_ushort4(bits_of(lo[0]), bits_of(lo[1]), bits_of(lo[2]), bits_of(lo[3]));
    }
    cluster_arrive();                    // nobody leaves while its sums are read
    cluster_wait();
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
    int32_t rank, padded;      // and as the output has it
    bf16* h;                   // [rows][2][padded]
    Waits waits;
};

constexpr int kShrinkStages = 4;
template <int R, int ROWS> constexpr int kShrinkSmem = kShrinkStages * (ROWS + R) * 128 + 1024;

// The copies of a CTA: steps of 64 elements of ROWS rows of x and R of m; a thread's are chunk tid % 8 of every THREADS / 8th row.  The cluster's CTAs take the
// steps in turn, so that what they read at the same time lies side by side in memory.
template <int R, int ROWS, int THREADS, bool ANY> struct ShrinkCopies {
    static constexpr int kStage = (ROWS + R) * 128, kStep = THREADS / 8, kX = ROWS / kStep, kM = R > kStep ? R / kStep : 1;
    RowCopies<bf16, kX, ANY> x;
    RowCopies<bf16, kM, ANY> m;
    int32_t n, first, stride, count;   // elements: the row's, to the thread's chunk of the first step, from step to step; steps
    uint32_t ring, place;
    __device__ __forceinline__ ShrinkCopies(const ShrinkParams& p, int64_t row0, int r0, int adapter, uint32_t rank, uint32_t ctas, uint32_t smem) : n((int32_t)p.n), ring(smem)
    {
        const int line = threadIdx.x >> 3, chunk = threadIdx.x & 7;
        const int32_t steps = (n + 63) / 64;
        first = (int32_t)rank * 64 + chunk * 8;
        stride = (int32_t)ctas * 64;
        count = (steps - (int32_t)rank + (int32_t)ctas - 1) / (int32_t)ctas;
#pragma unroll
        for (int i = 0; i < kX; ++i) {
            const int32_t t = token_at(p.s, row0 + i * kStep + line);
            x.set(i, t >= 0 ? p.x + (int64_t)t * p.ldx : nullptr, first, p.x);
        }
#pragma unroll
        for (int i = 0; i < kM; ++i) {
            const int r = r0 + i * kStep + line;
            m.set(i, r < p.m_rows ? p.m + (int64_t)adapter * p.m_stride + (int64_t)r * p.ldm : nullptr, first, p.x);
        }
        place = chunk_at<128>(line, chunk);                                       // 8 rows further a chunk's place repeats
    }
    __device__ __forceinline__ uint32_t stage(int32_t i) const { return ring + (uint32_t)i % kShrinkStages * kStage; }
    __device__ __forceinline__ void fill(int32_t step) const
    {
        if (step < count) {
            const uint32_t to = stage(step) + place;
            const int at = step * stride, left = n - first - at;
            x.copy(to, kStep * 128, at, left, first);
            if (R >= kStep || (int)threadIdx.x < R * 8) m.copy(to + ROWS * 128, kStep * 128, at, left, first);
        }
        copies_commit();
    }
};

// A CTA takes 128 rows of one adapter and all ranks; a cluster's CTAs share the reduction axis.  Bound by latency: 8192 rows of 4096, rank 64, take 19-21 us, 10 of
// them for the 67 MB at the copy rate, the others launch, first loads and join.
template <int R, bool ANY> __global__ void __launch_bounds__(256) adapter_shrink_kernel(const __grid_constant__ ShrinkParams p)
{
    constexpr int kColumns = R < 32 ? 32 : R;
    extern __shared__ uint8_t smem_raw[];
    __shared__ Products c;
    __shared__ uint32_t there[4];
    products_begin(c, kColumns);
    wait_for_predecessor();
    const uint32_t rank = cluster_rank(), ctas = cluster_size(), smem = (shared_at(smem_raw) + 1023u) & ~1023u;
    const int64_t first = (int64_t)(blockIdx.x / ctas) * 128;
    if (first >= used_rows(p.s)) {                                                // the whole cluster
        products_end(c, kColumns);
        return;
    }
    const int warp = warp_number(), lane = threadIdx.x & 31;
    const int adapter = adapter_of(p.s, first, lane);
    const ShrinkCopies<R, 128, 256, ANY> copies(p, first, 0, adapter, rank, ctas, smem);
    bool given_up = false;
#pragma unroll
    for (int s = 0; s < kShrinkStages - 1; ++s) copies.fill(s);
    if (warp < 4) {
        const uint32_t mask = __ballot_sync(0xFFFFFFFFu, token_at(p.s, first + warp * 32 + lane) >= 0);
        if (lane == 0) there[warp] = mask;
    }
    for (int32_t n = 0; n < copies.count; ++n) {
        copies_wait<kShrinkStages - 2>();
        fence_async_smem();
        __syncthreads();
        if (warp == 0 && elect_one()) {
            const uint64_t x = operand<128>(copies.stage(n)), m = operand<128>(copies.stage(n) + 128 * 128);
#pragma unroll
            for (int k = 0; k < 4; ++k) mma_bf16(c.tmem, x + 2 * k, m + 2 * k, product(R, false), n > 0 || k > 0);
            products_commit(c, n % kShrinkStages, n, p.waits);
        }
        // the next step's tile goes where the last one's products read from
        if (n > 0) products_wait(c, (n - 1) % kShrinkStages, (uint32_t)((n - 1) / kShrinkStages), p.waits, given_up);
        copies.fill(n + kShrinkStages - 1);
    }
    const int32_t count = copies.count;
    if (count > 0) products_wait(c, (count - 1) % kShrinkStages, (uint32_t)((count - 1) / kShrinkStages), p.waits, given_up);
    copies_wait<0>();
    tc_fence_after();
    __syncthreads();
    float* part = reinterpret_cast<float*>(smem_raw + (smem - shared_at(smem_raw)));              // [128][R + 4]
    const uint32_t lanes = c.tmem + ((uint32_t)(warp & 3) << 21);                 // warps w and w + 4 take turns at 16 columns
#pragma unroll
    for (int r = 0; r < R; r += 16) {
        if ((r >> 4 & 1) != warp >> 2) continue;
        uint32_t v[16] = {};
        if (count > 0) {
            tmem_load16(v, lanes + r);
            tc_wait_ld();
        }
#pragma unroll
        for (int k = 0; k < 16; k += 4) *reinterpret_cast<uint4*>(part + ((warp & 3) * 32 + lane) * (R + 4) + r + k) = make_uint4(v[k], v[k + 1], v[k + 2], v[k + 3]);
    }
    products_end(c, kColumns, given_up);
    join_rows<R>(part, there, 128, first, 0, (p.scale != nullptr ? p.scale[adapter] : 1.f) * p.factor, p.h, p.padded, p.rank, rank, ctas);
}

// A CTA takes 32 rows of one adapter and R of the ranks (blockIdx.y); a warp works on a quarter of each step.  1187 tokens of 1500, rank 24: 12 us, latency.
template <int R, bool ANY> __global__ void __launch_bounds__(128) adapter_shrink32_kernel(const __grid_constant__ ShrinkParams p)
{
    constexpr int kTiles = R / 8, kPitch = R + 4;
    static_assert(4 * kRows * kPitch * 4 <= kShrinkSmem<R, kRows> - 1024, "the sums take the ring's place");
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t there[1];
    wait_for_predecessor();
    const uint32_t rank = cluster_rank(), ctas = cluster_size(), smem = (shared_at(smem_raw) + 1023u) & ~1023u;
    const int64_t first = (int64_t)(blockIdx.x / ctas) * kRows;
    if (first >= used_rows(p.s)) return;                                          // the whole cluster
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    const int r0 = blockIdx.y * R, adapter = adapter_of(p.s, first, lane);
    const ShrinkCopies<R, kRows, 128, ANY> copies(p, first, r0, adapter, rank, ctas, smem);
    float acc[2][kTiles][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < kTiles; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[i][j][k] = 0.f;
#pragma unroll
    for (int s = 0; s < kShrinkStages - 1; ++s) copies.fill(s);
    if (warp == 0) {
        const uint32_t mask = __ballot_sync(0xFFFFFFFFu, token_at(p.s, first + lane) >= 0);
        if (lane == 0) there[0] = mask;
    }
    for (int32_t step = 0; step < copies.count; ++step) {
        copies_wait<kShrinkStages - 2>();
        __syncthreads();
        copies.fill(step + kShrinkStages - 1);
        const uint32_t xs = copies.stage(step), ms = xs + kRows * 128;
        uint32_t a[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) load_matrices(a[i], xs + chunk_at<128>(i * 16 + (lane & 15), warp * 2 + (lane >> 4)));
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
    }
    copies_wait<0>();
    __syncthreads();
    float* part = reinterpret_cast<float*>(smem_raw + (smem - shared_at(smem_raw)));              // [4][32][kPitch]
    {
        float* to = part + (warp * kRows + g) * kPitch + 2 * q;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < kTiles; ++j) {
                *reinterpret_cast<float2*>(to + i * 16 * kPitch + j * 8) = make_float2(acc[i][j][0], acc[i][j][1]);
                *reinterpret_cast<float2*>(to + (i * 16 + 8) * kPitch + j * 8) = make_float2(acc[i][j][2], acc[i][j][3]);
            }
    }
    __syncthreads();
    for (int at = tid; at < kRows * R / 4; at += 128) {
        float4* to = reinterpret_cast<float4*>(part + at / (R / 4) * kPitch + at % (R / 4) * 4);
        float4 v = *to;
#pragma unroll
        for (int k = 1; k < 4; ++k) {
            const float4 u = to[k * kRows * kPitch / 4];
            v.x += u.x;
            v.y += u.y;
            v.z += u.z;
            v.w += u.w;
        }
        *to = v;
    }
    join_rows<R>(part, there, kRows, first, r0, (p.scale != nullptr ? p.scale[adapter] : 1.f) * p.factor, p.h, p.padded, p.rank, rank, ctas);
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
    uint32_t tiles, across;    // CTAs: across for each tile of rows
    bool m_whole, base_whole, out_whole;
    Waits waits;
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
// To the columns from `at` on of a row of n, counted from anywhere.
template <typename T, typename I> __device__ __forceinline__ void store_out(const float* v, T* row, I at, I n, bool whole)
{
    if (at >= n) return;
    if (whole && at + kPer <= n) {
        Piece<T, kPer * (int)sizeof(T)> piece;
        piece.set_all(v);
#pragma unroll
        for (int i = 0; i < Piece<T, kPer * (int)sizeof(T)>::kWords; i += 4)
            *reinterpret_cast<uint4*>(reinterpret_cast<uint32_t*>(row + at) + i) = make_uint4(piece.w[i], piece.w[i + 1], piece.w[i + 2], piece.w[i + 3]);
    } else {
        store8(v, row + at, (int)min((I)kPer, n - at), false);
    }
}

template <int ROWS> constexpr int kExpandCols = ROWS == kRows ? 128 : 64;

// The copies of a CTA: kExpandCols columns of the base of ROWS rows, in blocks of 64, and the rows of m that make them, R of the ranks.  The rows of m
// are laid down so that column c of block j of 8 is column 8 (c / 2) + 2 j + c % 2 of 32: a thread's results, as the tensor instructions deal them
// out, are then 8 neighbouring columns.
enum Base : int { NO_BASE, WHOLE_BASE, ANY_BASE };      // none; rows that start on 16 bytes; rows that start anywhere
template <int R, int ROWS, int THREADS, typename T, int BASE> struct ExpandCopies {
    static constexpr bool ANY = BASE == ANY_BASE, kHas = BASE != NO_BASE;
    static constexpr int kCols = kExpandCols<ROWS>, kBase = kHas ? kCols * ROWS * (int)sizeof(T) : 0, kStage = kBase + kCols * R * 2;
    static constexpr int kChunks = 64 * (int)sizeof(T) / 16;                      // of a row's 64 columns
    static constexpr int kPieces = kCols * (int)sizeof(T) / 16, kStep = THREADS / kPieces, kB = ROWS / kStep;      // of a row; rows apart; a thread's
    static constexpr int kMChunks = R / 8, kMStep = THREADS / kMChunks, kM = kCols > kMStep ? kCols / kMStep : 1;
    static_assert(kStep % 2 == 0, "a piece's place repeats from row to row");
    RowCopies<T, kB, ANY> base;
    const bf16* m;
    int32_t n, m_cols;
    int64_t m_ld;
    uint32_t base_place, m_place;
    bool m_whole;
    // A 16-byte piece of the base: rows alternate between the halves of a line, for threads that read four neighbouring pieces of eight rows.
    static __device__ __forceinline__ uint32_t base_at(int row, int col16)
    {
        const int block = col16 / kChunks, chunk = col16 % kChunks;
        return (uint32_t)((block * ROWS + row) * (kChunks * 16) + ((chunk ^ ((row & 1) * (kChunks / 2))) << 4));
    }
    // c0: the first step's first column
    __device__ __forceinline__ ExpandCopies(const ExpandParams& p, const int32_t* tokens, int adapter, int64_t c0)
        : n((int32_t)(p.n - c0)), m_cols(p.m_cols), m_ld(p.ldm), m_whole(p.m_whole)
    {
        const int row = threadIdx.x / kPieces, c = threadIdx.x % kPieces, line = threadIdx.x / kMChunks, k = threadIdx.x % kMChunks;
        if constexpr (kHas) {
#pragma unroll
            for (int i = 0; i < kB; ++i) {
                const int32_t t = tokens[row + i * kStep];
                base.set(i, t >= 0 ? static_cast<const T*>(p.base) + (int64_t)t * p.ldb : nullptr, c0 + c * (16 / (int)sizeof(T)), p.base);
            }
        }
        first = (int32_t)c0 + c * (16 / (int)sizeof(T));
        base_place = base_at(row, c);
        m = p.m + (int64_t)adapter * p.m_stride + (c0 + line) * p.ldm + k * 8;
        m_place = m_at(line, k);
    }
    static __device__ __forceinline__ uint32_t m_at(int c, int k)
    {
        const int slot = (c & ~31) + ((c >> 1) & 3) * 8 + ((c >> 3) & 3) * 2 + (c & 1);
        return (uint32_t)kBase + chunk_at<R * 2>(slot, k);
    }
    int32_t first;
    // Columns from `at` on (since c0), ranks from r0 on, and the base if it is wanted.  A row's CTAs take the steps in turn: what they read and write at the
    // same time lies side by side in memory.
    __device__ __forceinline__ void fill(uint32_t stage, int at, int r0, bool with_base) const
    {
        if (kHas && with_base) {
            const int c = (int)threadIdx.x % kPieces * (16 / (int)sizeof(T));
            base.copy(stage + base_place, kStep * (kChunks * 16), at, n - at - c, first);
        }
        const int k = (int)threadIdx.x % kMChunks * 8 + r0, line = (int)threadIdx.x / kMChunks;
#pragma unroll
        for (int i = 0; i < kM; ++i) {
            if (kMStep > kCols && line >= kCols) break;
            const uint32_t to = stage + (kMStep % 32 == 0 ? m_place + i * kMStep * (R * 2) : m_at(line + i * kMStep, (int)threadIdx.x % kMChunks));
            const bf16* from = m + (int64_t)(at + i * kMStep) * m_ld + r0;
            const int left = at + line + i * kMStep < n ? m_cols - k : 0;
            if (m_whole) {
                copy_async(to, left > 0 ? from : m, 2 * max(0, min(8, left)));
            } else {
                uint32_t w[4];
                load_m<32>(w, left > 0 ? from : nullptr, 0, left, false);
                store_chunk(to, w);
            }
        }
    }
    // 8 columns of a row, q's of a block of 32.
    static __device__ __forceinline__ void read_base(float* v, const uint8_t* stage, int row, int block32, int q)
    {
        const int c16 = block32 * (32 * (int)sizeof(T) / 16) + q * (int)sizeof(T) / 2;
        Piece<T, kPer * (int)sizeof(T), 16> piece;
#pragma unroll
        for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
            const uint4 w = *reinterpret_cast<const uint4*>(stage + base_at(row, c16 + k));
            piece.w[4 * k] = w.x; piece.w[4 * k + 1] = w.y; piece.w[4 * k + 2] = w.z; piece.w[4 * k + 3] = w.w;
        }
#pragma unroll
        for (int k = 0; k < kPer; ++k) v[k] = piece.get(k);
    }
};

// Tokens without an adapter: every CTA of the grid takes some, the next token the next CTA's (those of a request lie side by side, and CTAs of their own for
// neighbouring tokens had all the work: 200 us for 480 of 8192 tokens).
template <typename T> __device__ __forceinline__ void copy_tokens(const ExpandParams& p)
{
    if (p.s.starts == nullptr) return;
    const bool whole = p.base_whole && p.n % kPer == 0;
    const int64_t step = (int64_t)blockDim.x * kPer;
    for (int64_t t0 = 0; t0 < p.s.tokens; t0 += 32 * (int64_t)gridDim.x) {
        const int64_t mine = t0 + blockIdx.x + (int64_t)(threadIdx.x & 31) * gridDim.x;
        for (uint32_t none = __ballot_sync(0xFFFFFFFFu, mine < p.s.tokens && p.s.row_of_token[mine] < 0); none != 0; none &= none - 1) {
            const int64_t token = t0 + blockIdx.x + (int64_t)(__ffs(none) - 1) * gridDim.x;
            const T* base = p.base != nullptr ? static_cast<const T*>(p.base) + token * p.ldb : nullptr;
            T* out = static_cast<T*>(p.out) + token * p.ldo;
            for (int64_t at = threadIdx.x * kPer; at < p.n; at += 2 * step) {
                float v[2][kPer];
#pragma unroll
                for (int k = 0; k < 2; ++k) load_base(v[k], base, at + k * step, p.n, whole);
#pragma unroll
                for (int k = 0; k < 2; ++k) store_out(v[k], out, at + k * step, p.n, p.out_whole);
            }
        }
    }
}

// A CTA takes 128 rows of one adapter and walks columns, 64 a step, with h in shared memory.  The products of a step run while the step before is read out
// of the other set of accumulators, added to its base and stored.  4096 -> 14336, rank 32, 8192 tokens: 94 us, 4.9 TB/s (a copy: 6.5) with
// 42 % of the issue slots and no byte read twice.  A tile's CTAs side by side in the grid, more and shorter CTAs, streaming stores: no difference.
// Three stages where a fourth would leave room for one CTA an SM only (two are worth more).
template <int R, typename T, int BASE> constexpr int kExpandStage = 64 * ((BASE != NO_BASE ? 128 * (int)sizeof(T) : 0) + R * 2);
template <int R, typename T, int BASE> constexpr int kExpandRest = 2 * 128 * R * 2 + 1024;
template <int R, typename T, int BASE> constexpr int kExpandStages = 4 * kExpandStage<R, T, BASE> + kExpandRest<R, T, BASE> <= 111 * 1024 ? 4 : 3;
template <int R, typename T, int BASE> constexpr int kExpandSmem = kExpandStages<R, T, BASE> * kExpandStage<R, T, BASE> + kExpandRest<R, T, BASE>;

template <int R, typename T, int BASE> __global__ void __launch_bounds__(256, BASE == NO_BASE ? 3 : 2) adapter_expand_kernel(const __grid_constant__ ExpandParams p)
{
    using C = ExpandCopies<R, 128, 256, T, BASE>;
    constexpr int kColumns = 128, kStages = kExpandStages<R, T, BASE>;
    static_assert(C::kStage == kExpandStage<R, T, BASE>, "");
    extern __shared__ uint8_t smem_raw[];
    __shared__ Products c;
    __shared__ int32_t tokens[128];
    products_begin(c, kColumns);
    wait_for_predecessor();
    const int tid = threadIdx.x, warp = warp_number(), lane = tid & 31, g = lane >> 2, q = lane & 3;
    const int32_t part = (int32_t)(blockIdx.x / p.tiles), count = ((int32_t)((p.n + 63) / 64) - part + (int32_t)p.across - 1) / (int32_t)p.across, stride = (int32_t)p.across * 64;
    const int64_t first = (int64_t)(blockIdx.x % p.tiles) * 128;
    if (first >= used_rows(p.s)) {
        products_end(c, kColumns);
        copy_tokens<T>(p);
        return;
    }
    const int adapter = adapter_of(p.s, first, lane);
    if (tid < 128) tokens[tid] = token_at(p.s, first + tid);
    __syncthreads();
    const uint32_t smem = (shared_at(smem_raw) + 1023u) & ~1023u, hs = smem + kStages * C::kStage;
    const uint8_t* const ring = smem_raw + (smem - shared_at(smem_raw));
    const C copies(p, tokens, adapter, (int64_t)part * 64);
    auto stage = [&](int32_t i) { return (uint32_t)i % kStages * C::kStage; };
    auto fill = [&](int32_t i) {
        if (i < count) copies.fill(smem + stage(i), i * stride, 0, true);
        copies_commit();
    };
#pragma unroll
    for (int i = tid; i < 128 * R / 4; i += 256) {
        const int row = i / (R / 4), half = i % (R / 4) / (R / 8), k = i % (R / 8);
        copy_async(hs + half * (128 * R * 2) + chunk_at<R * 2>(row, k), p.h + (first + row) * 2 * p.padded + half * p.padded + k * 8, 16);
    }
#pragma unroll
    for (int i = 0; i < kStages; ++i) fill(i);                                    // h with the first
    // warps w and w + 4 read the same 32 rows, 32 of the 64 columns each
    const int row0 = (warp & 3) * 32, block = warp >> 2;
    T* out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int32_t t = tokens[row0 + i * 8 + g];
        out[i] = t >= 0 ? static_cast<T*>(p.out) + (int64_t)t * p.ldo + (int64_t)part * 64 + block * 32 + q * 8 : nullptr;
    }
    const int width = (int)p.n - part * 64 - block * 32 - q * 8;               // columns from the thread's first on
    bool given_up = false;
    for (int32_t n = 0; n <= count; ++n) {
        if (n < count) {
            copies_wait<kStages - 2>();
            fence_async_smem();
        }
        __syncthreads();                                                          // step n is there
        if (n < count && warp == 0 && elect_one()) {
            tc_fence_after();
            const uint64_t h = operand<R * 2>(hs), w = operand<R * 2>(smem + stage(n) + C::kBase);
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int k = 0; k < R / 16; ++k)
                    mma_bf16(c.tmem + (n & 1) * 64, h + half * (128 * R * 2 / 16) + 2 * k, w + 2 * k, product(64, false), half > 0 || k > 0);
            products_commit(c, n & 1, n, p.waits);
        }
        if (n == 0) continue;
        const int32_t i0 = n - 1;
        products_wait(c, i0 & 1, (uint32_t)(i0 >> 1), p.waits, given_up);
        tc_fence_after();
        const uint32_t lanes = c.tmem + ((uint32_t)row0 << 16) + (i0 & 1) * 64 + block * 32;
        float acc[2][4][4];
        tmem_load_frags(acc[0], lanes);
        tmem_load_frags(acc[1], lanes + (16u << 16));
        tc_wait_ld();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float v[kPer] = {};
            if constexpr (C::kHas) C::read_base(v, ring + stage(i0), row0 + i * 8 + g, block, q);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[2 * j] += acc[i >> 1][j][(i & 1) * 2];
                v[2 * j + 1] += acc[i >> 1][j][(i & 1) * 2 + 1];
            }
            if (out[i] != nullptr) store_out(v, out[i], i0 * stride, width, p.out_whole);
        }
        tc_fence_before();
        __syncthreads();                                                          // step n - 1 is read: its place and its sums are free
        fill(n - 1 + kStages);
    }
    copies_wait<0>();
    products_end(c, kColumns, given_up);
    copy_tokens<T>(p);
}

// A CTA takes 32 rows of one adapter and walks columns, 128 a step and 32 of them a warp; h is in registers.  1187 tokens, rank 24, 1500 -> 2731: 15 us, latency.
constexpr int kExpand32Stages = 3;
template <int R, typename T, int BASE> constexpr int kExpand32Smem = kExpand32Stages * 128 * ((BASE != NO_BASE ? kRows * (int)sizeof(T) : 0) + R * 2) + 128;

template <int R, typename T, int BASE> __global__ void __launch_bounds__(128) adapter_expand32_kernel(const __grid_constant__ ExpandParams p)
{
    using C = ExpandCopies<R, kRows, 128, T, BASE>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ int32_t tokens[kRows];
    wait_for_predecessor();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    const int32_t part = (int32_t)(blockIdx.x / p.tiles), count = ((int32_t)((p.n + C::kCols - 1) / C::kCols) - part + (int32_t)p.across - 1) / (int32_t)p.across;
    const int32_t stride = (int32_t)p.across * C::kCols;
    const int64_t first = (int64_t)(blockIdx.x % p.tiles) * kRows;
    if (first >= used_rows(p.s)) {
        copy_tokens<T>(p);
        return;
    }
    const int adapter = adapter_of(p.s, first, lane);
    if (tid < kRows) tokens[tid] = token_at(p.s, first + tid);
    __syncthreads();
    const C copies(p, tokens, adapter, (int64_t)part * C::kCols);
    const uint32_t smem = (shared_at(smem_raw) + 127u) & ~127u;
    const uint8_t* const ring = smem_raw + (smem - shared_at(smem_raw));
    const int chunks = p.padded / R;                                              // of the ranks
    const int32_t turns = count * chunks;
    auto stage = [&](int32_t i) { return (uint32_t)i % kExpand32Stages * C::kStage; };
    auto fill = [&](int32_t i) {                                                  // a turn is a step and a chunk of the ranks
        if (i < turns) copies.fill(smem + stage(i), i / chunks * stride, i % chunks * R, i % chunks == chunks - 1);
        copies_commit();
    };
#pragma unroll
    for (int i = 0; i < kExpand32Stages - 1; ++i) fill(i);
    uint32_t hi[2][R / 16][4], lo[2][R / 16][4];
    auto load_h = [&](int r0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t* h = reinterpret_cast<const uint32_t*>(p.h + (first + i * 16 + g) * 2 * p.padded + r0) + q;
            const int64_t below = (int64_t)8 * p.padded;                          // 8 rows, in words
#pragma unroll
            for (int k = 0; k < R / 16; ++k) {
                const uint32_t* l = h + p.padded / 2;
                hi[i][k][0] = h[k * 8];
                hi[i][k][1] = h[below + k * 8];
                hi[i][k][2] = h[k * 8 + 4];
                hi[i][k][3] = h[below + k * 8 + 4];
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
        const int32_t t = tokens[i * 8 + g];
        out[i] = t >= 0 ? static_cast<T*>(p.out) + (int64_t)t * p.ldo : nullptr;
    }
    float acc[2][4][4];
    for (int32_t turn = 0; turn < turns; ++turn) {
        copies_wait<kExpand32Stages - 2>();
        __syncthreads();
        fill(turn + kExpand32Stages - 1);
        const uint32_t ms = smem + stage(turn) + C::kBase;
        const int r0 = turn % chunks * R;
        if (chunks > 1) load_h(r0);
        if (r0 == 0) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[i][j][k] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int slot = warp * 32 + j * 8 + (lane & 7);
#pragma unroll
            for (int k = 0; k < (R + 31) / 32; ++k) {
                uint32_t b[4];                                                    // 32 ranks, or 16 of them twice
                load_matrices(b, ms + chunk_at<R * 2>(slot, R == 16 ? (lane >> 3) & 1 : k * 4 + (lane >> 3)));
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    mma(acc[i][j], hi[i][2 * k][0], hi[i][2 * k][1], hi[i][2 * k][2], hi[i][2 * k][3], b[0], b[1]);
                    mma(acc[i][j], lo[i][2 * k][0], lo[i][2 * k][1], lo[i][2 * k][2], lo[i][2 * k][3], b[0], b[1]);
                    if constexpr (R > 16) {
                        mma(acc[i][j], hi[i][2 * k + 1][0], hi[i][2 * k + 1][1], hi[i][2 * k + 1][2], hi[i][2 * k + 1][3], b[2], b[3]);
                        mma(acc[i][j], lo[i][2 * k + 1][0], lo[i][2 * k + 1][1], lo[i][2 * k + 1][2], lo[i][2 * k + 1][3], b[2], b[3]);
                    }
                }
            }
        }
        if (r0 + R < p.padded) continue;
        const int64_t at = (int64_t)part * C::kCols + turn / chunks * stride + warp * 32 + q * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (out[i] == nullptr) continue;
            // the base last, in one addition: the tensor instructions cut what they add to, and sums that began with an FP32 base lost its last digits (64 ranks: 14 units)
            float v[kPer] = {};
            if constexpr (C::kHas) C::read_base(v, ring + stage(turn), i * 8 + g, warp, q);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[2 * j] += acc[i >> 1][j][(i & 1) * 2];
                v[2 * j + 1] += acc[i >> 1][j][(i & 1) * 2 + 1];
            }
            store_out(v, out[i], at, p.n, p.out_whole);
        }
    }
    copies_wait<0>();
    copy_tokens<T>(p);
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
    Waits waits;
};

// 128 columns x R ranks of an adapter: the reduction runs over its rows, 64 a step, cut over a cluster's CTAs.  Both operands have the reduction axis across
// their rows, as they lie in memory.  Bound by the latency of its steps: 8192 rows, 4096 columns and rank 64, db and da
// together, take 42 us (138 MB; steps of 32 rows or fewer of them in flight: 53).
constexpr int kOuterStages = 3, kOuterCols = 128, kOuterRows = 64;
template <int R> constexpr int kOuterStage = kOuterRows * (kOuterCols + 2 * R) * 2;
template <int R> constexpr uint32_t kOuterColumns = R < 32 ? 32 : R;
template <int R> constexpr int kOuterSmem = kOuterStages * kOuterStage<R> + 1024;

template <int R, bool BY_COLUMN, bool ANY> __device__ __forceinline__ void outer_part(const OuterParams& p, uint32_t z_block, Products& c, uint8_t* smem_raw)
{
    constexpr int kHalf = kOuterRows * R * 2, kColumns = kOuterColumns<R>;        // bytes of h's high parts; of tensor memory
    constexpr int kLines = BY_COLUMN ? kOuterCols : R, kLine = BY_COLUMN ? R : kOuterCols, kPitch = kLine + 4;
    static_assert(kLines * kPitch * 4 <= kOuterSmem<R> - 1024, "the sums take the ring's place");
    const uint32_t rank = cluster_rank(), ctas = cluster_size(), smem = (shared_at(smem_raw) + 1023u) & ~1023u;
    const int tid = threadIdx.x, warp = warp_number();
    const int chunks = p.padded / R, adapter = z_block / chunks, r0 = z_block % chunks * R;
    const int64_t c0 = (int64_t)blockIdx.y * kOuterCols;
    const int64_t from = p.s.starts != nullptr ? p.s.starts[adapter] : 0, to = p.s.starts != nullptr ? p.s.starts[adapter + 1] : adapter == 0 ? p.s.rows : 0;
    const int32_t steps = (int32_t)((to - from + kOuterRows - 1) / kOuterRows), share = (steps + (int32_t)ctas - 1) / (int32_t)ctas;
    const int32_t begin = min((int32_t)rank * share, steps), count = min(begin + share, steps) - begin;
    // a thread copies chunk tid % 16 of every 16th row; the tokens of a step's rows are looked up a step ahead
    const int line = tid >> 4;
    int32_t ahead[4];
    auto look = [&](int32_t i) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t row = from + (int64_t)(begin + i) * kOuterRows + k * 16 + line;
            ahead[k] = i < count && row < to ? token_at(p.s, row) : -1;
        }
    };
    auto stage = [&](int32_t i) { return smem + (uint32_t)i % kOuterStages * kOuterStage<R>; };
    const bf16* const z = p.z + c0 + (tid & 15) * 8;
    const int left = (int)min((int64_t)8, p.n - c0 - (tid & 15) * 8);             // elements of the thread's chunk
    const uint32_t z_place = ((tid & 15) >> 3) * (kOuterRows * 128) + chunk_at<128>(line, tid & 7);
    constexpr int kHChunks = R / 4, kHStep = 256 / kHChunks, kH = kOuterRows / kHStep;             // of a row, high and low; rows apart; a thread's
    const int h_line = tid / kHChunks, h_part = tid % kHChunks / (R / 8), h_chunk = tid % (R / 8);
    const bf16* const h = p.h + (from + (int64_t)begin * kOuterRows + h_line) * 2 * p.padded + h_part * p.padded + r0 + h_chunk * 8;
    const uint32_t h_place = kOuterRows * kOuterCols * 2 + h_part * kHalf + chunk_at<R * 2>(h_line, h_chunk);
    const int32_t rows = (int32_t)min(to - from - (int64_t)begin * kOuterRows, (int64_t)count * kOuterRows);
    auto fill = [&](int32_t i) {
        if (i < count) {
            const uint32_t zs = stage(i) + z_place;
            if constexpr (ANY) {
                fill_shifted<bf16, 4>([&](int k) { return ahead[k] >= 0 ? p.z + (int64_t)ahead[k] * p.ldz : nullptr; }, c0 + (tid & 15) * 8, p.n,
                                      [&](int k) { return zs + k * 16 * 128; });
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    copy_async(zs + k * 16 * 128, ahead[k] >= 0 && left > 0 ? z + (int64_t)ahead[k] * p.ldz : p.z, ahead[k] >= 0 ? 2 * max(0, left) : 0);
            }
#pragma unroll
            for (int k = 0; k < kH; ++k) {
                const int row = i * kOuterRows + k * kHStep;
                const bool there = row + h_line < rows;
                copy_async(stage(i) + h_place + k * kHStep * (R * 2), there ? h + (int64_t)row * 2 * p.padded : p.h, there ? 16 : 0);
            }
        }
        copies_commit();
        look(i + 1);
    };
    bool given_up = false;
    look(0);
#pragma unroll
    for (int i = 0; i < kOuterStages - 1; ++i) fill(i);
    for (int32_t n = 0; n < count; ++n) {
        copies_wait<kOuterStages - 2>();
        fence_async_smem();
        __syncthreads();
        if (warp == 0 && elect_one()) {
            const uint64_t zs = operand<128>(stage(n), kOuterRows * 128), hs = operand<R * 2>(stage(n) + kOuterRows * kOuterCols * 2);
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
                for (int k = 0; k < kOuterRows / 16; ++k)                          // 16 rows of either further
                    mma_bf16(c.tmem, zs + k * (16 * 128 / 16), hs + part * (kHalf / 16) + k * (16 * R * 2 / 16), product(R, true), n > 0 || part > 0 || k > 0);
            products_commit(c, n % kOuterStages, n, p.waits);
        }
        if (n > 0) products_wait(c, (n - 1) % kOuterStages, (uint32_t)((n - 1) / kOuterStages), p.waits, given_up);
        fill(n + kOuterStages - 1);
    }
    if (count > 0) products_wait(c, (count - 1) % kOuterStages, (uint32_t)((count - 1) / kOuterStages), p.waits, given_up);
    copies_wait<0>();
    tc_fence_after();
    __syncthreads();
    float* part = reinterpret_cast<float*>(smem_raw + (smem - shared_at(smem_raw)));              // [kLines][kPitch]
    const uint32_t lanes = c.tmem + ((uint32_t)(warp & 3) << 21);                 // warps w and w + 4 take turns at 16 ranks; a thread has a column
    const int col = tid & 127;
#pragma unroll
    for (int r = 0; r < R; r += 16) {
        if ((r >> 4 & 1) != warp >> 2) continue;
        uint32_t v[16] = {};
        if (count > 0) {
            tmem_load16(v, lanes + r);
            tc_wait_ld();
        }
        if constexpr (BY_COLUMN) {
#pragma unroll
            for (int k = 0; k < 16; k += 4) *reinterpret_cast<uint4*>(part + col * kPitch + r + k) = make_uint4(v[k], v[k + 1], v[k + 2], v[k + 3]);
        } else {
#pragma unroll
            for (int k = 0; k < 16; ++k) part[(r + k) * kPitch + col] = __uint_as_float(v[k]);
        }
    }
    products_end(c, kColumns, given_up);
    cluster_arrive();
    cluster_wait();
    bf16* out = p.out + (int64_t)adapter * p.rank * p.n;
    const int lines = kLines / (int)ctas;
    for (int at = tid; at < lines * (kLine / 4); at += 256) {
        const int l = (int)rank * lines + at / (kLine / 4), e = at % (kLine / 4) * 4;
        const float4 v = sum_remote4(shared_at(part + l * kPitch + e), ctas);
        const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int r = r0 + (BY_COLUMN ? e + k : l);
            const int64_t n = c0 + (BY_COLUMN ? l : e + k);
            if (r < p.rank && n < p.n) out[BY_COLUMN ? n * p.rank + r : (int64_t)r * p.n + n] = __float2bfloat16(f[k]);
        }
    }
    cluster_arrive();
    cluster_wait();
}

// Both gradients in one launch, db = dy^T h for the first `split` of blockIdx.z, da = u^T x for the others: with half as many CTAs for each, the ramps are paid once (one launch each: 25-27 us).
struct OuterPair {
    OuterParams b, a;
    uint32_t split;
};
template <int R, bool ANY> __global__ void __launch_bounds__(256) adapter_outer_kernel(const __grid_constant__ OuterPair p)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ Products c;
    const bool of_b = blockIdx.z < p.split;
    if ((int64_t)blockIdx.y * kOuterCols >= (of_b ? p.b.n : p.a.n)) return;       // the whole cluster
    products_begin(c, kOuterColumns<R>);
    wait_for_predecessor();
    if (of_b) outer_part<R, true, ANY>(p.b, blockIdx.z, c, smem_raw);
    else outer_part<R, false, ANY>(p.a, blockIdx.z - p.split, c, smem_raw);
}

// ---------------------------------------------------------------------------------------- transposes ----

struct TurnParams {
    const bf16 *a, *b;
    bf16 *at, *bt;             // [adapters][n_in][padded] and [adapters][padded][wide], zero where there is no element
    int64_t n_in, n_out, wide;
    int32_t rank, padded;
    uint32_t a_ctas;           // CTAs of a for one adapter
};

// Both matrices of the adapters with their axes swapped, for the gradients' products: tiles of 32 x 32.  Rank 64, 4096 and 4096: 3.6 us, a launch's latency.
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
// memories, and each CTA makes an eighth of the columns (or less: where tiles are few and columns many, several clusters do the first part alike and
// share the columns).  Bound by the latency of four dependent reads (ids, x and a, b and base, and the exchange): one token, rank 16, 4096 -> 14336 4.8 us in a graph,
// 48 tokens of 24 adapters, rank 32, 4096 -> 4096 7.7.
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
    const int64_t parts = (int64_t)gridDim.y * kMaxCluster, steps = (p.n_out + 31) / 32, share = (steps + parts - 1) / parts;
    const int64_t c_first = min((int64_t)(blockIdx.y * kMaxCluster + rank) * share, steps), c_last = min(c_first + share, steps);
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
        if (members[i / R] >= 0 && i % R < p.rank)
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
// average) cost less than what smaller tiles read again of the adapters.  Ranks above 64 come in pieces, which only the small tiles take.
int tile_rows(const mor_adapter_desc_t& d) { return d.rank <= 64 && d.tokens >= 2048 && d.tokens >= 256 * (int64_t)d.adapters ? 128 : kRows; }
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
// One launch by clusters of 16 tokens, or sorted tokens and two more launches.  Measured, 8 adapters, 4096 -> 4096, small and sorted: rank 16, 192 tokens 10.2 and
// 12.1 us, 256 tokens 12.7 and 12.4; rank 64, 96 tokens 11.4 and 17.1, 128 tokens 17.6 and 17.0; 4096 -> 14336, rank 16, 128 tokens 13.6 and 13.8, 256 tokens 18.4
// and 14.6.
bool small_call(const mor_adapter_desc_t& d, bool train)
{
    return !train && d.rank <= 64 && d.tokens <= (d.rank > 32 ? 96 : 224) && d.tokens * d.n_out <= 1 << 21;
}

template <typename F> cudaError_t by_rank(int padded, F&& f)
{
    return padded == 16 ? f(std::integral_constant<int, 16>{}) : padded == 32 ? f(std::integral_constant<int, 32>{}) : f(std::integral_constant<int, 64>{});
}

// CTAs that the GPU holds at once of a kernel with that much shared memory.
constexpr int64_t resident(int smem) { return 148 * std::min(227 * 1024 / (smem + 2048), 4); }

// Allows the kernel its shared memory and launches it.
template <typename K, typename P> cudaError_t launch_ring(K kernel, std::atomic<uint64_t>& done, int smem, dim3 grid, uint32_t cluster, uint32_t block, cudaStream_t st, const P& p)
{
    if (!allow_smem(kernel, smem, done)) return cudaErrorUnknown;
    return launch_clusters(kernel, grid, cluster, block, (size_t)smem, st, p);
}

// Tiles that are expected to hold tokens: of the rows that there may be, about half a tile of each adapter is empty.
int64_t filled_tiles(const Sorted& s, int rows)
{
    return std::max<int64_t>(1, s.starts != nullptr ? std::min(s.rows / rows, ceil_div(s.tokens, rows) + s.adapters / 2) : s.rows / rows);
}

template <int R, int ROWS, bool ANY> cudaError_t shrink_launch(const ShrinkParams& p, cudaStream_t st)
{
    static std::atomic<uint64_t> done{0};
    const int64_t tiles = p.s.rows / ROWS, steps = (p.n + 63) / 64;
    const int64_t filled = filled_tiles(p.s, ROWS);
    const uint32_t chunks = (uint32_t)(p.padded / R);
    uint32_t cluster = 1;                     // as many CTAs to a tile as the GPU holds at once (clusters do not fill it quite), two steps each at least
    while (cluster < kMaxCluster && filled * chunks * cluster * 20 <= resident(kShrinkSmem<R, ROWS>) * 9 && steps >= 4 * cluster) cluster *= 2;
    const dim3 grid((uint32_t)tiles * cluster, chunks);
    if constexpr (ROWS == 128) return launch_ring(adapter_shrink_kernel<R, ANY>, done, kShrinkSmem<R, ROWS>, grid, cluster, 256, st, p);
    else return launch_ring(adapter_shrink32_kernel<R, ANY>, done, kShrinkSmem<R, ROWS>, grid, cluster, 128, st, p);
}
cudaError_t shrink(const ShrinkParams& p, int rows, bool any, cudaStream_t st)
{
    return by_rank(p.padded > 64 ? 64 : p.padded, [&](auto r) {
        constexpr int R = decltype(r)::value;
        if (rows == kRows) return any ? shrink_launch<R, kRows, true>(p, st) : shrink_launch<R, kRows, false>(p, st);
        return any ? shrink_launch<R, 128, true>(p, st) : shrink_launch<R, 128, false>(p, st);
    });
}

template <int R, int ROWS, typename T, int BASE> cudaError_t expand_launch(ExpandParams p, cudaStream_t st)
{
    static std::atomic<uint64_t> done{0};
    p.tiles = (uint32_t)(p.s.rows / ROWS);
    const int64_t steps = (p.n + kExpandCols<ROWS> - 1) / kExpandCols<ROWS>;
    // as many CTAs as the GPU holds at once
    constexpr int kSmem = ROWS == 128 ? kExpandSmem<R, T, BASE> : kExpand32Smem<R, T, BASE>;
    p.across = (uint32_t)std::max<int64_t>(1, std::min<int64_t>(steps, resident(kSmem) / filled_tiles(p.s, ROWS)));
    const dim3 grid(p.tiles * p.across);
    if constexpr (ROWS == 128) return launch_ring(adapter_expand_kernel<R, T, BASE>, done, kSmem, grid, 0, 256, st, p);
    else return launch_ring(adapter_expand32_kernel<R, T, BASE>, done, kSmem, grid, 0, 128, st, p);
}
template <typename T, int BASE> cudaError_t expand_rows(const ExpandParams& p, int rows, cudaStream_t st)
{
    return by_rank(p.padded > 64 ? 64 : p.padded, [&](auto r) {
        constexpr int R = decltype(r)::value;
        return rows == kRows ? expand_launch<R, kRows, T, BASE>(p, st) : expand_launch<R, 128, T, BASE>(p, st);
    });
}
cudaError_t expand(const ExpandParams& p, int rows, int dtype, cudaStream_t st)
{
    if (p.base == nullptr) return expand_rows<bf16, NO_BASE>(p, rows, st);       // a gradient, BF16
    if (dtype == MOR_DTYPE_BF16) return p.base_whole ? expand_rows<bf16, WHOLE_BASE>(p, rows, st) : expand_rows<bf16, ANY_BASE>(p, rows, st);
    return p.base_whole ? expand_rows<float, WHOLE_BASE>(p, rows, st) : expand_rows<float, ANY_BASE>(p, rows, st);
}

template <int R, bool ANY> cudaError_t outer_launch(const OuterPair& p, uint32_t deep, cudaStream_t st)
{
    static std::atomic<uint64_t> done{0};
    const int64_t nb = p.split > 0 ? ceil_div(p.b.n, kOuterCols) : 0, na = deep > p.split ? ceil_div(p.a.n, kOuterCols) : 0;
    const Sorted& s = p.split > 0 ? p.b.s : p.a.s;
    const int64_t mean = s.rows / s.adapters, all = nb * p.split + na * (deep - p.split);      // two steps each at least, going by the adapters' mean
    uint32_t cluster = 1;
    while (cluster < kMaxCluster && all * cluster * 2 <= resident(kOuterSmem<R>) && mean >= 4 * kOuterRows * (int64_t)cluster) cluster *= 2;
    return launch_ring(adapter_outer_kernel<R, ANY>, done, kOuterSmem<R>, dim3(cluster, (uint32_t)std::max(na, nb), deep), cluster, 256, st, p);
}
// Of b, of a or of both; the other's `out` is null.
cudaError_t outer(const OuterParams& b, const OuterParams& a, bool any, cudaStream_t st)
{
    const OuterParams& one = b.out != nullptr ? b : a;
    return by_rank(one.padded > 64 ? 64 : one.padded, [&](auto r) {
        constexpr int R = decltype(r)::value;
        const uint32_t each = (uint32_t)(one.s.adapters * (one.padded / R)), deep = (b.out != nullptr ? each : 0) + (a.out != nullptr ? each : 0);
        const OuterPair p = {b, a, b.out != nullptr ? each : 0};
        return any ? outer_launch<R, true>(p, deep, st) : outer_launch<R, false>(p, deep, st);
    });
}

Waits waits_of(const mor_adapter_desc_t& d)
{
    Waits w = {d.status, 0, 0};
    test_hook_main(w.skip, w.cycles);
    return w;
}

mor_status_t check_adapter(const mor_adapter_desc_t* d)
{
    if (d == nullptr || d->tokens < 0 || d->tokens >= (1ll << 30) || d->n_in < 1 || d->n_out < 1 || d->n_in > kMaxWidth || d->n_out > kMaxWidth) return MOR_ERR_INVALID_ARG;
    if (d->adapters < 1 || d->adapters >= MOR_MAX_GROUPS || d->rank < 1 || d->rank > MOR_MAX_RANK) return MOR_ERR_INVALID_ARG;
    if (d->a == nullptr || d->b == nullptr) return MOR_ERR_INVALID_ARG;
    if (sorted_rows(*d) < 0) return MOR_ERR_INVALID_ARG;
    if (!is_aligned(d->a, 2) || !is_aligned(d->b, 2) || !is_aligned(d->ids, 4) || !is_aligned(d->scale, 4) || !is_aligned(d->status, 4)) return MOR_ERR_ALIGNMENT;
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
        // no more than two clusters' CTAs an SM, and a step of 32 columns for every warp
        const int64_t tiles = d->ids != nullptr ? d->tokens : ceil_div(d->tokens, kSmallRows);
        const int64_t across = std::max<int64_t>(1, std::min(ceil_div(d->n_out, 32 * kSmallWarps * kMaxCluster), 2 * 148 / kMaxCluster / tiles));
        const dim3 grid((uint32_t)tiles * kMaxCluster, (uint32_t)across);
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
    ShrinkParams sp = {f.s, static_cast<const bf16*>(x), static_cast<const bf16*>(d->a), d->scale, d->factor, ldx, d->n_in, d->n_in, (int64_t)d->rank * d->n_in, d->rank, d->rank, padded, f.h, waits_of(*d)};
    if (shrink(sp, rows, any, stream) != cudaSuccess) return MOR_ERR_CUDA;
    ExpandParams ep = {f.s, f.h, static_cast<const bf16*>(d->b), d->n_out, d->rank, (int64_t)d->n_out * d->rank, d->rank, padded, base, out, ldb, ldo, 0, 0,
                       d->rank % 8 == 0 && is_aligned(d->b, 16), base_whole, out_whole, waits_of(*d)};
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
        ShrinkParams sp = {f.s, static_cast<const bf16*>(dy), w.bt, d->scale, d->factor, lddy, d->n_out, w.wide, (int64_t)padded * w.wide, padded, d->rank, padded, w.u, waits_of(*d)};
        if (shrink(sp, rows, !dy_whole, stream) != cudaSuccess) return MOR_ERR_CUDA;
    }
    if (da != nullptr || db != nullptr) {
        const OuterParams b = {f.s, f.h, static_cast<const bf16*>(dy), lddy, d->n_out, d->rank, padded, static_cast<bf16*>(db), waits_of(*d)};
        const OuterParams a = {f.s, w.u, static_cast<const bf16*>(x), ldx, d->n_in, d->rank, padded, static_cast<bf16*>(da), waits_of(*d)};
        if (outer(b, a, (db != nullptr && !dy_whole) || (da != nullptr && !x_whole), stream) != cudaSuccess) return MOR_ERR_CUDA;
    }
    if (dx != nullptr) {
        ExpandParams ep = {f.s, w.u, w.at, d->n_in, padded, (int64_t)d->n_in * padded, padded, padded, base, dx, ldb, lddx, 0, 0, true, base_whole, dx_whole, waits_of(*d)};
        if (expand(ep, rows, MOR_DTYPE_BF16, stream) != cudaSuccess) return MOR_ERR_CUDA;
    }
    return MOR_OK;
}

}  // extern "C"
