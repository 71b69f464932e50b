// Products of microscaled 4-bit operands on the tensor cores: out[m, n] = ta tb sum_k (ca sa)(cb sb).
//
// Two kernels share the pipeline: a thread copies 256 elements of the reduction axis at a time (128 bytes of codes per row,
// swizzled, and the scale tiles) into a ring of stages, a thread moves a stage's scales to tensor memory and issues the
// matrix instructions (64 elements each), other warps read the accumulators out.  Block scales are applied by the tensor cores;
// the two tensor scales are one factor at the end.
//   wide    tiles of 256 x 256 by a pair of CTAs (each holds half of both operands' rows) or 128 x 256 by one; persistent
//   narrow  128 rows of b (a weight's outputs) x 16..128 rows of a (tokens): the product is taken transposed, so that the
//           instruction's 128 rows are all weights; the reduction axis is split over a cluster, whose partial sums are added in rank
//           order through distributed shared memory.
#include "mor_fp4.cuh"
#include "mor_internal.h"
#include "mor_tcgen05.cuh"

namespace mor {
namespace {

constexpr int kStageElems = 256;                     // of the reduction axis per stage: 128 bytes of codes, the swizzle's width
constexpr uint32_t kFull = 0xFFFFFFFFu;
constexpr int kCtrlBytes = 1024;
constexpr int kFewRows = 32;                         // a group's tile with no more rows than these is fetched by them alone
constexpr int kMaxSmem = 227 * 1024;

struct GemmParams {
    CUtensorMap a, b, sa, sb, a_few;     // a_few (ROWS): a in boxes of kFewRows rows
    int64_t m, n, k, ldo;
    int32_t a_row_tiles, b_row_tiles, a_ktiles, b_ktiles;
    const float *ta, *tb;
    const int32_t *starts, *slot_of_row;
    int32_t groups, grouping;
    int32_t m_tiles, n_tiles;        // of the whole output (REDUCE: of one group's)
    void* out;
    uint32_t* status;
    uint32_t skip_tile;              // test hook: this tile's first load is left out
    long long wait_cycles;
};

// After a wait ran out: report, and leave copies and matrix instructions in flight the time to end before shared and tensor
// memory go away (they take microseconds).
__device__ __noinline__ void give_up(volatile uint32_t* abort_flag, uint32_t* status)
{
    *abort_flag = 1;
    if (status != nullptr) atomicExch(status, (uint32_t)MOR_ERR_TIMEOUT);
}
__device__ __noinline__ void drain()
{
    const long long t0 = clock64();
    while (clock64() - t0 < 400000) {}
}

// A whole warp's bounded wait; false (and everything is told to stop) when it ran out for any lane.
template <typename Ctl> __device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, Ctl& C, const GemmParams& p)
{
    const bool ok = __all_sync(kFull, mbar_wait(bar, parity, &C.abort, p.wait_cycles));
    if (!ok) give_up(&C.abort, p.status);
    return ok;
}

template <int CG, int NT, int FMT> struct Wide {
    static constexpr bool kNv = FMT == MOR_FP4_E4M3_16;
    static constexpr int kSf = kNv ? 4 : 2;                          // scale tiles per stage and 128 rows
    static constexpr int kGroupsB = NT / 128;
    static constexpr int kBytesA = 128 * 128, kBytesB = NT / CG * 128;
    static constexpr int kBytesSa = kSf * kScaleTile, kBytesSb = kGroupsB * kSf * kScaleTile;
    static constexpr int kStage = kBytesA + kBytesB + kBytesSa + kBytesSb;
    static constexpr int kSfCols = kSf * 4 * (1 + kGroupsB);         // tensor memory columns of a stage's scales
    static constexpr int kFit = (kMaxSmem - kCtrlBytes - 1024) / kStage, kFitTmem = (512 - NT) / kSfCols;
    static constexpr int kStages = kFit < kFitTmem ? kFit : kFitTmem;
    static constexpr int kSmem = kStages * kStage + kCtrlBytes + 1024;
};
constexpr int kWideThreads = 384;      // copy, issue, tensor memory, idle; eight warps that read the accumulators out

struct WideCtrl {
    uint64_t full[8], empty[8], acc_full, acc_empty;
    uint32_t tmem, abort;
};
static_assert(sizeof(WideCtrl) <= kCtrlBytes, "control block");

// One output tile and the part of the reduction axis that it sums over.
struct TileAt {
    int row, row_end;       // first row of the tile; rows from row_end on belong to another group
    int n, group;           // tile column; matrix of b (ROWS) or of out (REDUCE)
    int k0, len;
};

// Tiles are walked in bands of eight tile rows, column by column inside a band, so that the CTAs that run at the same time share
// rows of both operands in L2.
__device__ __forceinline__ void in_bands(int t, int m_tiles, int n_tiles, int& m, int& n)
{
    const int band = t / (8 * n_tiles), in = t - band * 8 * n_tiles, height = min(8, m_tiles - band * 8);
    n = in / height;
    m = band * 8 + in % height;
}

// The groups in shared memory: where they start, and (ROWS) the number of tile rows before each (a group has whole tiles of its
// own; the last may reach past it).
template <int GROUP> struct Groups {
    int32_t starts[GROUP == MOR_GROUP_NONE ? 1 : MOR_MAX_GROUPS + 1];
    int32_t before[GROUP == MOR_GROUP_ROWS ? MOR_MAX_GROUPS + 1 : 1];
};
template <int CG, int GROUP> __device__ __forceinline__ void fill_table(const GemmParams& p, Groups<GROUP>& table)
{
    if constexpr (GROUP == MOR_GROUP_NONE) return;
    // copies and stores have to start on whole tiles inside the matrix whatever the array holds
    const int most = (int)(GROUP == MOR_GROUP_ROWS ? p.m : p.k);
    for (int i = threadIdx.x; i <= p.groups; i += blockDim.x) table.starts[i] = min(max(p.starts[i], 0) & ~127, most);
    if constexpr (GROUP == MOR_GROUP_ROWS) {
        __syncthreads();
        if (threadIdx.x < 32) {
            int before = 0;
            for (int g0 = 0; g0 < p.groups; g0 += 32) {
                const int g = g0 + (int)threadIdx.x;
                const int v = g < p.groups ? max(0, (table.starts[g + 1] - table.starts[g] + 128 * CG - 1) / (128 * CG)) : 0;
                int sum = v;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int u = __shfl_up_sync(kFull, sum, o);
                    if ((int)threadIdx.x >= o) sum += u;
                }
                if (g < p.groups) table.before[g] = before + sum - v;
                before += __shfl_sync(kFull, sum, 31);
            }
            if (threadIdx.x == 0) table.before[p.groups] = before;
        }
    }
}

template <int CG, int GROUP> __device__ __forceinline__ bool tile_at(const GemmParams& p, const Groups<GROUP>& table, int t, TileAt& at)
{
    int m;
    at.group = 0;
    at.k0 = 0;
    at.len = (int)p.k;
    at.row_end = (int)p.m;
    if constexpr (GROUP == MOR_GROUP_NONE) {
        if (t >= p.m_tiles * p.n_tiles) return false;
        in_bands(t, p.m_tiles, p.n_tiles, m, at.n);
        at.row = m * 128 * CG;
    } else if constexpr (GROUP == MOR_GROUP_ROWS) {
        if (t >= table.before[p.groups] * p.n_tiles) return false;
        const int tile_row = t / p.n_tiles;
        int lo = 0, hi = p.groups - 1;                  // the last group with no more tile rows before it
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (table.before[mid] <= tile_row) lo = mid;
            else hi = mid - 1;
        }
        at.group = lo;
        const int in = t - table.before[lo] * p.n_tiles, height = table.before[lo + 1] - table.before[lo];
        at.n = in / height;
        at.row = table.starts[lo] + in % height * 128 * CG;
        at.row_end = table.starts[lo + 1];
    } else {
        const int per = p.m_tiles * p.n_tiles;
        if (t >= per * p.groups) return false;
        at.group = t / per;
        in_bands(t - at.group * per, p.m_tiles, p.n_tiles, m, at.n);
        at.row = m * 128 * CG;
        at.k0 = table.starts[at.group];
        at.len = table.starts[at.group + 1] - at.k0;
    }
    return true;
}

// Both tensor scales, as two factors of a sum.  Where their product is a normal number it is the one factor.  Operands of small values would
// lose its digits (each scale may be 2^-99) though the results are normal numbers, and those of large ones would make sums of zero NaN; there
// the scales are applied one after the other, the smaller first: E4M3_16 sums are multiples of 2^-20 below 2^55, so that this step neither overflows
// before the result does nor reaches the subnormal numbers.
struct OutScale {
    float first, then;
    __device__ __forceinline__ OutScale() : first(0.f), then(1.f) {}
    __device__ __forceinline__ OutScale(float a, float b) : first(a * b), then(1.f)
    {
        const float size = fabsf(first);
        if (size < 0x1p-126f || size == INFINITY) {
            const bool order = fabsf(a) <= fabsf(b);
            first = order ? a : b;
            then = order ? b : a;
        }
    }
    __device__ __forceinline__ float of(float sum) const { return sum * first * then; }
    __device__ __forceinline__ float of(uint32_t sum) const { return of(__uint_as_float(sum)); }
};

template <typename T> __device__ __forceinline__ uint32_t out_word(const uint32_t* acc, const OutScale& scale, int j)
{
    if constexpr (sizeof(T) == 2) return bf16x2_of(scale.of(acc[2 * j]), scale.of(acc[2 * j + 1]));
    else return __float_as_uint(scale.of(acc[j]));
}
// 32 neighbouring values of one output row, or the first n of them.
template <typename T> __device__ __forceinline__ void store_row32(T* to, const uint32_t* acc, const OutScale& scale, int n)
{
    constexpr int kWords = 32 * sizeof(T) / 4;
    uint32_t w[kWords];
#pragma unroll
    for (int j = 0; j < kWords; ++j) w[j] = out_word<T>(acc, scale, j);
    if (n >= 32 && (reinterpret_cast<uintptr_t>(to) & 31) == 0) {
#pragma unroll
        for (int j = 0; j < kWords; j += 8) stg256(reinterpret_cast<uint32_t*>(to) + j, w + j);
    } else if (n >= 32) {
#pragma unroll
        for (int j = 0; j < kWords; j += 4) *reinterpret_cast<uint4*>(reinterpret_cast<uint32_t*>(to) + j) = make_uint4(w[j], w[j + 1], w[j + 2], w[j + 3]);
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            if (j >= n) break;
            if constexpr (sizeof(T) == 2) reinterpret_cast<uint16_t*>(to)[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
            else reinterpret_cast<uint32_t*>(to)[j] = w[j];
        }
    }
}
// COLS values of a row that starts 16 bytes past a sector of 32: half a sector at both ends, whole ones between, where 16-byte stores alone
// would write every sector in two parts (8192 x 14328 x 4096 BF16: 196 us, 223 by 16 bytes; 3000 x 7004 x 1000 FP32: 27 us, 40).
template <typename T, int COLS> __device__ __forceinline__ void store_row_off16(T* to, const uint32_t* acc, const OutScale& scale)
{
    constexpr int kWords = COLS * sizeof(T) / 4;
    uint32_t* const out = reinterpret_cast<uint32_t*>(to);
    auto four = [&](int j) {
        return make_uint4(out_word<T>(acc, scale, j), out_word<T>(acc, scale, j + 1), out_word<T>(acc, scale, j + 2), out_word<T>(acc, scale, j + 3));
    };
    *reinterpret_cast<uint4*>(out) = four(0);
#pragma unroll
    for (int j = 4; j < kWords - 4; j += 8) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = out_word<T>(acc, scale, j + i);
        stg256(out + j, w);
    }
    *reinterpret_cast<uint4*>(out + kWords - 4) = four(kWords - 4);
}

// Wide.  A pair's tile of 256 x 256 fetches 2 x 128 rows of either operand per CTA, the least per product that tensor memory holds
// with a stage's scales; one accumulator set, handed over after its registers are filled, so that the stores run under the next tile's
// products.  8192 x 14336 x 4096 E4M3_16 -> BF16: 190-200 us (4.8-5.0 PFLOP/s) in a short run, 226 us at the 1000 W cap (1.4 GHz);
// 8192 x 4096 x 8192: 100 us (5.5 PFLOP/s).  Its copies alone take 142 us (54 bytes a clock and SM from L2), its products alone 157 us,
// and without the result's stores it is 30 us faster.  256 x 192 tiles with two accumulator sets: 215 us.
// Groups of rows, 28,956 rows over 32 groups, E8M0_32: 2048 -> 1024 40 us, 1024 -> 2048 54 us, 29 us each without the stores (64 and 127 MB); with FP32
// results 51 and 78 us.  Groups of the reduction axis, 32 results of 1024 x 2048: 63 us, FP32 87.  The tensor pipe is 18-42 % active and DRAM at
// 24-35 % of its peak: with 4 to 8 stages a tile, what bounds them is that products and reading out take turns at the one accumulator set.
template <int CG, int NT, int FMT, typename T, int GROUP>
__global__ void __launch_bounds__(kWideThreads, 1) fp4_wide_kernel(const __grid_constant__ GemmParams p)
{
    using W = Wide<CG, NT, FMT>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ Groups<GROUP> table;
    uint8_t* smem = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    WideCtrl& C = *reinterpret_cast<WideCtrl*>(smem + W::kStages * W::kStage);
    const int warp = warp_number(), lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;

    if (threadIdx.x == 0) {
        for (int s = 0; s < W::kStages; ++s) {
            mbar_init(&C.full[s], 1);
            mbar_init(&C.empty[s], 1);
        }
        mbar_init(&C.acc_full, 1);
        mbar_init(&C.acc_empty, 8 * CG);
        C.abort = 0;
        fence_mbar_init();
        if (p.k > 0) {
            prefetch_map(&p.a);
            prefetch_map(&p.b);
            prefetch_map(&p.sa);
            prefetch_map(&p.sb);
        }
    }
    if (warp == 2) tmem_alloc<CG>(&C.tmem, 512);
    tc_fence_before();
    wait_for_predecessor();
    fill_table<CG, GROUP>(p, table);
    if constexpr (CG == 2) cluster_sync();
    else __syncthreads();
    tc_fence_after();
    const uint32_t tmem = C.tmem;
    const int first = blockIdx.x / CG, step = gridDim.x / CG;
    TileAt at;

    if (warp == 0) {                                                // ---- copies
        uint32_t slot = 0, lap = 0;
        bool ok = true;
        for (int t = first; ok && tile_at<CG, GROUP>(p, table, t, at); t += step) {
            const int stages = (at.len + kStageElems - 1) / kStageElems;
            const int row_a = at.row + (int)rank * 128, row_b = at.n * NT + (int)rank * (NT / CG);
            const int za = 0, zb = GROUP == MOR_GROUP_ROWS ? at.group : 0;
            // rows past the group's last slot are not needed: what an earlier stage left there enters rows that are not stored
            bool few = false;
            if constexpr (GROUP == MOR_GROUP_ROWS)
                few = p.slot_of_row != nullptr && row_a + kFewRows < (int)p.m && p.slot_of_row[row_a + kFewRows] < 0;
            const uint32_t bytes = CG * (W::kStage - (few ? W::kBytesA - kFewRows * 128 : 0));
            const int sa = (za * p.a_row_tiles + row_a / 128) * p.a_ktiles, sb = (zb * p.b_row_tiles + at.n * (NT / 128)) * p.b_ktiles;
            for (int s = 0; s < stages; ++s) {
                if (lap > 0 && !wait_warp(&C.empty[slot], (lap - 1u) & 1u, C, p)) {
                    ok = false;
                    break;
                }
                if (elect_one()) {
                    const uint32_t base = smem_addr(smem) + slot * W::kStage;
                    uint32_t bar = smem_addr(&C.full[slot]);
                    if (rank == 0) mbar_arrive_expect_tx(&C.full[slot], bytes);
                    if constexpr (CG == 2) bar = map_rank(bar, 0);
                    const int k = at.k0 + s * kStageElems, ktile = k / (W::kNv ? 64 : 128);
                    if (!(t == (int)p.skip_tile && s == 0)) load_tile_3d<CG>(base, few ? &p.a_few : &p.a, k / 2, row_a, za, bar);
                    load_tile_3d<CG>(base + W::kBytesA, &p.b, k / 2, row_b, zb, bar);
                    const uint32_t sf = base + W::kBytesA + W::kBytesB;
                    load_tile_2d<CG>(sf, &p.sa, 0, sa + ktile, bar);
#pragma unroll
                    for (int g = 0; g < W::kGroupsB; ++g)
                        load_tile_2d<CG>(sf + W::kBytesSa + g * W::kSf * kScaleTile, &p.sb, 0, sb + g * p.b_ktiles + ktile, bar);
                }
                __syncwarp();
                if (++slot == W::kStages) { slot = 0; ++lap; }
            }
        }
    } else if (warp == 1 && rank == 0) {                            // ---- matrix instructions
        uint32_t slot = 0, lap = 0, done = 0;
        bool ok = true;
        for (int t = first; ok && tile_at<CG, GROUP>(p, table, t, at); t += step) {
            const int stages = (at.len + kStageElems - 1) / kStageElems;
            if (stages <= 0) continue;
            if (done > 0) ok = wait_warp(&C.acc_empty, (done - 1u) & 1u, C, p);
            tc_fence_after();
            for (int s = 0; ok && s < stages; ++s) {
                if (!wait_warp(&C.full[slot], lap & 1u, C, p)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const int steps = min(4, (at.len - s * kStageElems + 63) / 64);
                if (elect_one()) {
                    const uint32_t base = smem_addr(smem) + slot * W::kStage, sf = base + W::kBytesA + W::kBytesB;
                    const uint32_t tsa = tmem + NT + slot * W::kSfCols, tsb = tsa + 4 * W::kSf;
                    const uint64_t da = codes_desc(base), db = codes_desc(base + W::kBytesA), ds = scales_desc(sf);
#pragma unroll
                    for (int j = 0; j < W::kSf; ++j) {
                        copy_scales<CG>(tsa + 4 * j, ds + j * (kScaleTile >> 4));
#pragma unroll
                        for (int g = 0; g < W::kGroupsB; ++g)
                            copy_scales<CG>(tsb + (j * W::kGroupsB + g) * 4, ds + ((W::kBytesSa + (g * W::kSf + j) * kScaleTile) >> 4));
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (j >= steps) break;
                        const int tile = W::kNv ? j : j >> 1, byte = W::kNv ? 0 : 2 * (j & 1);
                        mma_fp4<CG, W::kNv>(tmem, da + 2 * j, db + 2 * j, fp4_idesc(128 * CG, NT, W::kNv, byte), tsa + 4 * tile,
                                            tsb + 4 * W::kGroupsB * tile, s > 0 || j > 0);
                    }
                    tc_commit<CG>(smem_addr(&C.empty[slot]));
                    if (s == stages - 1) tc_commit<CG>(smem_addr(&C.acc_full));
                }
                __syncwarp();
                if (++slot == W::kStages) { slot = 0; ++lap; }
            }
            ++done;
        }
    } else if (warp >= 4) {                                         // ---- accumulators out
        const int half = (warp - 4) >> 2;
        const OutScale scale = p.k > 0 ? OutScale(*p.ta, *p.tb) : OutScale();
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        constexpr int kCols = NT / 2;
        uint32_t acc[kCols], done = 0;
        bool ok = true;
        for (int t = first; ok && tile_at<CG, GROUP>(p, table, t, at); t += step) {
            const int64_t row = (int64_t)at.row + rank * 128 + (warp & 3) * 32 + lane;
            const int64_t col = (int64_t)at.n * NT + half * kCols;
            bool wanted = row < at.row_end;
            if (GROUP == MOR_GROUP_ROWS && p.slot_of_row != nullptr) wanted = wanted && p.slot_of_row[row] >= 0;
            if (at.len > 0) {
                ok = wait_warp(&C.acc_full, done & 1u, C, p);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int j = 0; j < kCols; j += 32) tmem_load32(acc + j, tmem + lanes + half * kCols + j);
                tc_wait_ld();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (CG == 2) mbar_arrive_cluster(map_rank(smem_addr(&C.acc_empty), 0));
                    else mbar_arrive(&C.acc_empty);
                }
                ++done;
            } else {
#pragma unroll
                for (uint32_t& v : acc) v = 0;
            }
            if (wanted) {
                T* out = static_cast<T*>(p.out) + ((GROUP == MOR_GROUP_REDUCE ? (int64_t)at.group * p.m : 0) + row) * p.ldo + col;
                const OutScale f = at.len > 0 ? scale : OutScale();
                if ((reinterpret_cast<uintptr_t>(out) & 31) != 0 && col + kCols <= p.n) {
                    store_row_off16<T, kCols>(out, acc, f);
                } else {
#pragma unroll
                    for (int j = 0; j < kCols; j += 32)
                        if (col + j < p.n) store_row32<T>(out + j, acc + j, f, (int)min((int64_t)32, p.n - col - j));
                }
            }
            __syncwarp();
        }
    }
    __syncwarp();
    __syncthreads();
    if (*(volatile uint32_t*)&C.abort) drain();
    if constexpr (CG == 2) cluster_sync();
    if (warp == 2) {
        tc_fence_after();
        tmem_free<CG>(tmem, 512);
    }
}

// ---- narrow

template <int NT, int FMT> struct Narrow {
    static constexpr bool kNv = FMT == MOR_FP4_E4M3_16;
    static constexpr int kSf = kNv ? 4 : 2;
    static constexpr int kBytesA = 128 * 128, kBytesB = NT * 128;
    static constexpr int kBytesSf = kSf * kScaleTile;
    static constexpr int kStage = kBytesA + kBytesB + 2 * kBytesSf;
    static constexpr int kSfCols = 8 * kSf;
    static constexpr int kAcc = NT < 32 ? 32 : NT;
    static constexpr int kTmem = 256;                               // two CTAs share an SM
    static constexpr int kFit = (kMaxSmem / 2 - kCtrlBytes - 2048) / kStage, kFitTmem = (kTmem - kAcc) / kSfCols;
    static constexpr int kStages = kFit < kFitTmem ? kFit : kFitTmem;
    static constexpr int kSmem = kStages * kStage + kCtrlBytes + 1024;
    static_assert(NT * 512 <= kStages * kStage, "the partial sums fit the ring");
};
constexpr int kNarrowThreads = 192;    // copy, issue, four warps that read the accumulators out
constexpr int kMaxSplit = 8;

// Bound by the read of the weights: 3.2 us and then 6.5 TB/s (14336 rows of b, K from 4096 to 65536).  Two CTAs an SM keep a ring of copies in
// flight each; the split over a cluster fills the SMs where there are few tiles (16 x 14336 x 4096: 7.0 us with its launch), and adding
// the parts in rank order keeps the result the same from run to run.
template <int NT, int FMT, typename T> __global__ void __launch_bounds__(kNarrowThreads, 2) fp4_narrow_kernel(const __grid_constant__ GemmParams p)
{
    using W = Narrow<NT, FMT>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    WideCtrl& C = *reinterpret_cast<WideCtrl*>(smem + W::kStages * W::kStage);
    const int warp = warp_number(), lane = threadIdx.x & 31;
    uint32_t split;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(split));
    const uint32_t rank = cluster_rank();
    const int tile = blockIdx.x / split, feature0 = tile % p.n_tiles * 128, token0 = tile / p.n_tiles * NT;
    const int all = (int)((p.k + kStageElems - 1) / kStageElems);
    const int begin = (int)((int64_t)all * rank / split), end = (int)((int64_t)all * (rank + 1) / split);

    if (threadIdx.x == 0) {
        for (int s = 0; s < W::kStages; ++s) {
            mbar_init(&C.full[s], 1);
            mbar_init(&C.empty[s], 1);
        }
        mbar_init(&C.acc_full, 1);
        C.abort = 0;
        fence_mbar_init();
        if (p.k > 0) {
            prefetch_map(&p.a);
            prefetch_map(&p.b);
            prefetch_map(&p.sa);
            prefetch_map(&p.sb);
        }
    }
    if (warp == 1) tmem_alloc<1>(&C.tmem, W::kTmem);
    tc_fence_before();
    wait_for_predecessor();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = C.tmem;

    if (warp == 0) {
        uint32_t slot = 0, lap = 0;
        for (int s = begin; s < end; ++s) {
            if (lap > 0 && !wait_warp(&C.empty[slot], (lap - 1u) & 1u, C, p)) break;
            if (elect_one()) {
                const uint32_t base = smem_addr(smem) + slot * W::kStage, bar = smem_addr(&C.full[slot]);
                mbar_arrive_expect_tx(&C.full[slot], W::kStage);
                const int k = s * kStageElems, ktile = k / (W::kNv ? 64 : 128);
                if (!(tile == (int)p.skip_tile && s == begin)) load_tile_3d<1>(base, &p.b, k / 2, feature0, 0, bar);
                load_tile_3d<1>(base + W::kBytesA, &p.a, k / 2, token0, 0, bar);
                load_tile_2d<1>(base + W::kBytesA + W::kBytesB, &p.sb, 0, feature0 / 128 * p.b_ktiles + ktile, bar);
                load_tile_2d<1>(base + W::kBytesA + W::kBytesB + W::kBytesSf, &p.sa, 0, token0 / 128 * p.a_ktiles + ktile, bar);
            }
            __syncwarp();
            if (++slot == W::kStages) { slot = 0; ++lap; }
        }
    } else if (warp == 1) {
        uint32_t slot = 0, lap = 0;
        for (int s = begin; s < end; ++s) {
            if (!wait_warp(&C.full[slot], lap & 1u, C, p)) break;
            tc_fence_after();
            const int steps = (int)min((int64_t)4, (p.k - (int64_t)s * kStageElems + 63) / 64);
            if (elect_one()) {
                const uint32_t base = smem_addr(smem) + slot * W::kStage, sf = base + W::kBytesA + W::kBytesB;
                const uint32_t tsa = tmem + W::kAcc + slot * W::kSfCols, tsb = tsa + 4 * W::kSf;
                const uint64_t da = codes_desc(base), db = codes_desc(base + W::kBytesA), ds = scales_desc(sf);
#pragma unroll
                for (int j = 0; j < W::kSf; ++j) {
                    copy_scales<1>(tsa + 4 * j, ds + j * (kScaleTile >> 4));
                    copy_scales<1>(tsb + 4 * j, ds + ((W::kBytesSf + j * kScaleTile) >> 4));
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (j >= steps) break;
                    const int t = W::kNv ? j : j >> 1, byte = W::kNv ? 0 : 2 * (j & 1);
                    mma_fp4<1, W::kNv>(tmem, da + 2 * j, db + 2 * j, fp4_idesc(128, NT, W::kNv, byte), tsa + 4 * t, tsb + 4 * t, s > begin || j > 0);
                }
                tc_commit<1>(smem_addr(&C.empty[slot]));
                if (s == end - 1) tc_commit<1>(smem_addr(&C.acc_full));
            }
            __syncwarp();
            if (++slot == W::kStages) { slot = 0; ++lap; }
        }
    }
    __syncwarp();
    const int part = warp & 3, feature = part * 32 + lane;            // a warp reads the 32 lanes of its number modulo 4
    float* sums = reinterpret_cast<float*>(smem);
    bool ok = true;
    if (warp >= 2) {
        if (begin < end) {
            ok = wait_warp(&C.acc_full, 0, C, p);
            tc_fence_after();
        }
        if (ok) {
            const uint32_t lanes = (uint32_t)part << 21;
#pragma unroll
            for (int j = 0; j < NT; j += 16) {
                uint32_t acc[16];
                if (begin < end) {
                    tmem_load16(acc, tmem + lanes + j);
                    tc_wait_ld();
                } else {
#pragma unroll
                    for (uint32_t& v : acc) v = 0;
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) sums[(j + i) * 128 + feature] = __uint_as_float(acc[i]);
            }
        }
    }
    tc_fence_before();
    cluster_sync();
    if (warp >= 2 && ok) {
        const OutScale scale = p.k > 0 ? OutScale(*p.ta, *p.tb) : OutScale();
        const int64_t f = (int64_t)feature0 + feature;
        if (f < p.n)
            for (int j = (int)rank; j < NT && token0 + j < p.m; j += (int)split) {
                const uint32_t from = smem_addr(sums + j * 128 + feature);
                float s = 0.f;
                for (uint32_t r = 0; r < split; ++r) s += lds_cluster(map_rank(from, r));
                T* to = static_cast<T*>(p.out) + (int64_t)(token0 + j) * p.ldo + f;
                if constexpr (sizeof(T) == 2) *to = __float2bfloat16(scale.of(s));
                else *to = scale.of(s);
            }
    }
    __syncwarp();
    if (*(volatile uint32_t*)&C.abort) drain();
    cluster_sync();
    if (warp == 1) {
        tc_fence_after();
        tmem_free<1>(tmem, W::kTmem);
    }
}

// ---- host side

bool encode_codes(CUtensorMap& map, const mor_fp4_matrix_t& m, uint32_t box_rows, EncodeTiledFn enc)
{
    const cuuint64_t dims[3] = {(cuuint64_t)(ceil_div(m.cols, 32) * 16), (cuuint64_t)m.rows, (cuuint64_t)m.batch};
    const cuuint64_t strides[2] = {(cuuint64_t)m.ld, (cuuint64_t)m.ld * (cuuint64_t)m.rows};
    const cuuint32_t box[3] = {128, box_rows, 1}, estr[3] = {1, 1, 1};
    return enc(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, m.codes, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// The scale tiles of the whole stack as rows of 512 bytes.
bool encode_scales(CUtensorMap& map, const mor_fp4_matrix_t& m, uint32_t tiles, EncodeTiledFn enc)
{
    const cuuint64_t all = (cuuint64_t)(m.batch * ceil_div(m.rows, 128) * scale_ktiles(m.cols, m.format));
    const cuuint64_t dims[2] = {kScaleTile / 4, all}, strides[1] = {kScaleTile};
    const cuuint32_t box[2] = {kScaleTile / 4, tiles}, estr[2] = {1, 1};
    return enc(&map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, m.scales, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t launch_cluster(void (*kernel)(GemmParams), uint32_t grid, uint32_t block, size_t smem, uint32_t cluster, cudaStream_t st, const GemmParams& p)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <int CG, int NT, int FMT, typename T, int GROUP>
mor_status_t run_wide(GemmParams& p, const mor_fp4_matrix_t& a, const mor_fp4_matrix_t& b, EncodeTiledFn enc, cudaStream_t st)
{
    using W = Wide<CG, NT, FMT>;
    static_assert(W::kStages >= 2 && W::kStages <= 8, "ring");
    static std::atomic<uint64_t> done{0};
    if (p.k > 0 && !(encode_codes(p.a, a, 128, enc) && encode_codes(p.b, b, NT / CG, enc) && encode_scales(p.sa, a, W::kSf, enc) && encode_scales(p.sb, b, W::kSf, enc)))
        return MOR_ERR_CUDA;
    // ROWS: how many tile rows there are is known on the device alone; each group may leave one partly empty
    if (GROUP == MOR_GROUP_ROWS && p.k > 0 && !encode_codes(p.a_few, a, kFewRows, enc)) return MOR_ERR_CUDA;
    const int64_t mt = GROUP == MOR_GROUP_ROWS ? p.m / (128 * CG) + p.groups : ceil_div(p.m, 128 * CG);
    const int64_t nt = ceil_div(p.n, NT), groups = GROUP == MOR_GROUP_REDUCE ? p.groups : 1;
    if (mt * nt * groups >= (1ll << 31) - 1024) return MOR_ERR_UNSUPPORTED;
    p.m_tiles = (int32_t)mt;
    p.n_tiles = (int32_t)nt;
    auto* kernel = fp4_wide_kernel<CG, NT, FMT, T, GROUP>;
    if (!allow_smem(kernel, W::kSmem, done)) return MOR_ERR_CUDA;
    const int64_t tiles = mt * nt * groups, most = 148 / CG;
    const uint32_t grid = (uint32_t)((tiles < most ? tiles : most) * CG);
    return launch_cluster(kernel, grid, kWideThreads, W::kSmem, CG, st, p) == cudaSuccess ? MOR_OK : MOR_ERR_CUDA;
}

template <int NT, int FMT, typename T>
mor_status_t run_narrow(GemmParams& p, const mor_fp4_matrix_t& a, const mor_fp4_matrix_t& b, EncodeTiledFn enc, cudaStream_t st)
{
    using W = Narrow<NT, FMT>;
    static_assert(W::kStages >= 2 && W::kStages <= 8, "ring");
    static std::atomic<uint64_t> done{0};
    if (p.k > 0 && !(encode_codes(p.a, a, NT, enc) && encode_codes(p.b, b, 128, enc) && encode_scales(p.sa, a, W::kSf, enc) && encode_scales(p.sb, b, W::kSf, enc)))
        return MOR_ERR_CUDA;
    const int64_t nt = ceil_div(p.n, 128), mt = ceil_div(p.m, NT), stages = ceil_div(p.k, kStageElems);
    if (nt * mt >= (1ll << 31) / kMaxSplit) return MOR_ERR_UNSUPPORTED;
    p.n_tiles = (int32_t)nt;
    p.m_tiles = (int32_t)mt;
    int64_t split = 148 * 2 / (nt * mt);
    split = split > kMaxSplit ? kMaxSplit : split;
    split = split > stages ? stages : split;
    split = split >= 8 ? 8 : split >= 4 ? 4 : split >= 2 ? 2 : 1;      // clusters of other sizes leave places empty (6144 x 4096 by 6: 9.8 us, by 4: 5.5)
    auto* kernel = fp4_narrow_kernel<NT, FMT, T>;
    if (!allow_smem(kernel, W::kSmem, done)) return MOR_ERR_CUDA;
    return launch_cluster(kernel, (uint32_t)(nt * mt * split), kNarrowThreads, W::kSmem, (uint32_t)split, st, p) == cudaSuccess ? MOR_OK : MOR_ERR_CUDA;
}

template <int FMT, typename T> mor_status_t run_format(GemmParams& p, const mor_fp4_matrix_t& a, const mor_fp4_matrix_t& b, EncodeTiledFn enc, cudaStream_t st)
{
    // groups of rows by single CTAs: tiles of 128 rows waste less of a group's last one (28,700 rows over 32 groups, E8M0_32: 2048 ->
    // 1024 39.6 us against 41.2 by pairs, 1024 -> 2048 52.8 against 59.4)
    if (p.grouping == MOR_GROUP_ROWS) return run_wide<1, 256, FMT, T, MOR_GROUP_ROWS>(p, a, b, enc, st);
    if (p.grouping == MOR_GROUP_REDUCE) return run_wide<2, 256, FMT, T, MOR_GROUP_REDUCE>(p, a, b, enc, st);
    // The narrow kernel spreads few tokens over the whole GPU, the wide one fetches the weights once for 256.  E8M0_32, weights beyond L2, narrow and
    // wide by tokens: 4096 x 4096: 32 6.9 and 9.2 us, 64 8.4 and 9.7, 128 11.2 and 10.6, 256 14.9 and 10.7; 4096 outputs x 14336: 64 11.8 and
    // 21.2, 128 14.8 and 22.1, 256 20.3 and 22.2.  With 14336 outputs the wide kernel has tiles for 56 pairs and is ahead from 32 tokens on (12.7
    // and 11.8 us; 128: 24.6 and 12.4): the switch at 128 tokens is right for few outputs or a long reduction axis and gives that case away.
    if (p.m <= 16) return run_narrow<16, FMT, T>(p, a, b, enc, st);
    if (p.m <= 32) return run_narrow<32, FMT, T>(p, a, b, enc, st);
    if (p.m <= 64) return run_narrow<64, FMT, T>(p, a, b, enc, st);
    if (p.m <= 128) return run_narrow<128, FMT, T>(p, a, b, enc, st);
    return run_wide<2, 256, FMT, T, MOR_GROUP_NONE>(p, a, b, enc, st);
}

}  // namespace
}  // namespace mor

using namespace mor;

extern "C" mor_status_t mor_fp4_matmul(const mor_fp4_matmul_desc_t* host_desc, void* cuda_stream)
{
    if (host_desc == nullptr) return MOR_ERR_INVALID_ARG;
    const mor_fp4_matmul_desc_t& d = *host_desc;
    const bool rows = d.grouping == MOR_GROUP_ROWS, reduce = d.grouping == MOR_GROUP_REDUCE;
    if (!is_dtype(d.out_dtype) || (d.grouping != MOR_GROUP_NONE && !rows && !reduce)) return MOR_ERR_INVALID_ARG;
    mor_status_t s = check_matrix(d.a);
    if (s != MOR_OK) return s;
    if ((s = check_matrix(d.b)) != MOR_OK) return s;
    if (d.a.format != d.b.format || d.a.cols != d.b.cols || d.a.batch != 1) return MOR_ERR_INVALID_ARG;
    if (d.grouping != MOR_GROUP_NONE && (d.groups < 1 || d.groups > MOR_MAX_GROUPS || d.starts == nullptr)) return MOR_ERR_INVALID_ARG;
    if (d.b.batch != (rows ? d.groups : 1) || (d.slot_of_row != nullptr && !rows)) return MOR_ERR_INVALID_ARG;
    if (d.ldo < d.b.rows) return MOR_ERR_INVALID_ARG;
    const int es = (int)dtype_bytes(d.out_dtype);
    if (!is_aligned(d.out, 16) || d.ldo * es % 16 != 0 || !is_aligned(d.starts, 4) || !is_aligned(d.slot_of_row, 4) || !is_aligned(d.status, 4)) return MOR_ERR_ALIGNMENT;
    if (d.a.rows == 0 || d.b.rows == 0) return MOR_OK;
    if (d.out == nullptr) return MOR_ERR_INVALID_ARG;
    EncodeTiledFn enc = encode_tiled_fn();
    if (enc == nullptr) return MOR_ERR_CUDA;

    GemmParams p = {};
    p.m = d.a.rows;
    p.n = d.b.rows;
    p.k = d.a.cols;
    p.ldo = d.ldo;
    p.a_row_tiles = (int32_t)ceil_div(d.a.rows, 128);
    p.b_row_tiles = (int32_t)ceil_div(d.b.rows, 128);
    p.a_ktiles = p.b_ktiles = (int32_t)scale_ktiles(d.a.cols, d.a.format);
    p.ta = d.a.tensor_scale;
    p.tb = d.b.tensor_scale;
    p.starts = d.starts;
    p.groups = d.groups;
    p.slot_of_row = d.slot_of_row;
    p.grouping = d.grouping;
    p.out = d.out;
    p.status = d.status;
    test_hook_main(p.skip_tile, p.wait_cycles);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (d.a.format == MOR_FP4_E4M3_16)
        return d.out_dtype == MOR_DTYPE_BF16 ? run_format<MOR_FP4_E4M3_16, __nv_bfloat16>(p, d.a, d.b, enc, st) : run_format<MOR_FP4_E4M3_16, float>(p, d.a, d.b, enc, st);
    return d.out_dtype == MOR_DTYPE_BF16 ? run_format<MOR_FP4_E8M0_32, __nv_bfloat16>(p, d.a, d.b, enc, st) : run_format<MOR_FP4_E8M0_32, float>(p, d.a, d.b, enc, st);
}
