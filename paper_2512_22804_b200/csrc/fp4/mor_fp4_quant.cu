// Quantisation to microscaled 4-bit codes, along the rows, along the columns, or both from one read, and its inverse.
//
// Both directions are bound by memory: per element 2 (or 4) bytes in, 0.5 + 1/16 (or 1/32) out per direction; the tensor maximum
// of E4M3_16 costs one more read unless the caller has it.  A CTA takes tiles of 128 x 128 elements, so that the
// scale tiles it writes (128 rows x 4 blocks) are whole and leave as 16-byte stores, and in the column direction the codes of a
// transposed row leave 64 bytes at a time.  A thread takes units of 32 consecutive elements: one or two blocks, so a block's
// maximum needs no exchange between threads.  For the column direction the tile goes through shared memory once, in the
// input's own type where no weight is applied.
#include <type_traits>

#include "mor_fp4.cuh"

namespace mor {
namespace {

constexpr int kQThreads = 256;
constexpr int kAmaxMaxBlocks = MOR_FP4_WORKSPACE_BYTES / 4;
constexpr int64_t kSelfAmaxElems = 32768;     // up to here every CTA takes the maximum of the whole tensor by itself: one launch
                                              // instead of two (a CTA reads 32768 elements from L2 in about 1 us)

enum Mode : int { PLAIN = 0, GATHER = 1, WEIGHTED = 2 };

struct QuantParams {
    const void* x;
    int64_t ld, batch_stride;          // elements
    int64_t rows, cols;                // of the output matrix along the rows
    int64_t x_rows;                    // of x, over the whole stack when it is contiguous in rows
    uint32_t row_tiles, col_tiles;
    int32_t access;                    // bytes of a vector load: 32, 16, or one element
    const float* amax;
    const float* partial;              // maxima per CTA of the amax kernel
    uint32_t n_partial;                // 0 with partial == NULL and amax == NULL: the CTA takes the maximum itself
    int64_t batch;
    const int32_t* slot_of_row;
    const int32_t* row_of_slot;
    uint32_t top, inv_top;             // inv_top = floor((2^32 - 1) / top), see token_of()
    int32_t weight_dtype;
    const void* weight;
    uint8_t *r_codes, *r_scales, *c_codes, *c_scales;
    int64_t r_ld, c_ld;
    uint32_t r_ktiles, c_ktiles, c_row_tiles;
    float *r_t, *c_t;
};

// slot / top: the product with the rounded-down reciprocal is the quotient or one less.
__device__ __forceinline__ int64_t token_of(uint32_t slot, const QuantParams& p)
{
    const uint32_t q = __umulhi(slot, p.inv_top);
    return slot - q * p.top >= p.top ? q + 1 : q;
}

template <typename T> struct Raw;
template <> struct Raw<__nv_bfloat16> { uint32_t w[16]; };
template <> struct Raw<float> { uint32_t w[32]; };

// One unit from global memory; elements from n on are zero.
template <typename T> __device__ __forceinline__ void load_unit(Raw<T>& r, const T* p, int n, int access)
{
    constexpr int kWords = sizeof(Raw<T>) / 4;
    if (n >= kUnit && access == 32) {
#pragma unroll
        for (int i = 0; i < kWords; i += 8) ldg256(r.w + i, reinterpret_cast<const uint32_t*>(p) + i);
    } else if (n >= kUnit && access == 16) {
#pragma unroll
        for (int i = 0; i < kWords; i += 4) {
            const uint4 q = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint32_t*>(p) + i);
            r.w[i] = q.x; r.w[i + 1] = q.y; r.w[i + 2] = q.z; r.w[i + 3] = q.w;
        }
    } else if constexpr (sizeof(T) == 2) {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            const uint32_t lo = 2 * i < n ? h[2 * i] : 0, hi = 2 * i + 1 < n ? h[2 * i + 1] : 0;
            r.w[i] = lo | (hi << 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kWords; ++i) r.w[i] = i < n ? reinterpret_cast<const uint32_t*>(p)[i] : 0;
    }
}
template <typename T> __device__ __forceinline__ void unpack(const Raw<T>& r, float* v)
{
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 16; ++i) { v[2 * i] = bf16_low(r.w[i]); v[2 * i + 1] = bf16_high(r.w[i]); }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r.w[i]);
    }
}

__device__ __forceinline__ float block_max(float m, float* shared)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = m;
    __syncthreads();
    float r = shared[0];
#pragma unroll
    for (int i = 1; i < kQThreads / 32; ++i) r = fmaxf(r, shared[i]);
    __syncthreads();
    return r;
}

// Largest finite magnitude of a piece, times the weight of each slot that has a row.  The maximum over slots of fl(w x) is
// fl(max|w| * max|x|), since rounding is monotonic; only where that is not finite are the products looked at one by one.
template <typename T, int BYTES, int MODE> __device__ __noinline__ float piece_max_careful(const Piece<T, BYTES> v, const QuantParams& p, int64_t token)
{
    float m = 0.f;
    const int slots = MODE == PLAIN ? 1 : (int)p.top;
    for (int j = 0; j < slots; ++j) {
        if (MODE != PLAIN && p.row_of_slot[token * p.top + j] < 0) continue;
        const float w = MODE == WEIGHTED ? weight_at(p.weight, p.weight_dtype, token * p.top + j) : 1.f;
#pragma unroll
        for (int i = 0; i < Piece<T, BYTES>::kElems; ++i) {
            const float a = fabsf(v.get(i) * w);
            if (a < INFINITY) m = fmaxf(m, a);
        }
    }
    return m;
}
// Largest |weight| among the token's slots that have a row; -1 if none has.
template <int MODE> __device__ __forceinline__ float token_weight(const QuantParams& p, int64_t token)
{
    if constexpr (MODE == PLAIN) return 1.f;
    float w = -1.f;
    for (uint32_t j = 0; j < p.top; ++j)
        if (p.row_of_slot[token * p.top + j] >= 0) w = fmaxf(w, MODE == WEIGHTED ? fabsf(weight_at(p.weight, p.weight_dtype, token * p.top + j)) : 1.f);
    return w;
}
template <typename T, int BYTES, int MODE> __device__ __forceinline__ float piece_max(const Piece<T, BYTES>& v, const QuantParams& p, int64_t token)
{
    float a = 0.f;
    if constexpr (sizeof(T) == 2 && BYTES >= 4) {
        a = amax_of_pair(amax_of_words<BYTES / 4>(v.w));
    } else {
#pragma unroll
        for (int i = 0; i < Piece<T, BYTES>::kElems; ++i) a = max_nan(a, v.get(i));
    }
    const float w = token_weight<MODE>(p, token);
    if (MODE == GATHER && w < 0.f) return 0.f;
    const float m = a * w;
    return m >= 0.f && m < INFINITY ? m : piece_max_careful<T, BYTES, MODE>(v, p, token);
}

// The largest magnitude of the whole tensor, one part per CTA (they are joined by the kernel that quantises: no counter to
// clear, no atomics).  Bound by memory: a warp reads 1 KiB at a time (32 bytes a lane), a thread keeps four pieces in flight; the grid
// is resident as a whole.  8192 x 14336 BF16: 43 us (5.5 TB/s).
__host__ __device__ inline bool contiguous(const QuantParams& p) { return p.ld == p.cols && (p.batch == 1 || p.batch_stride == p.x_rows * p.ld); }
template <typename T, int BYTES, int MODE, bool ANY> __global__ void __launch_bounds__(kQThreads) fp4_amax_kernel(const __grid_constant__ QuantParams p, float* part)
{
    using P = Piece<T, BYTES>;
    constexpr int kFlight = 4;
    __shared__ float red[kQThreads / 32];
    wait_for_predecessor();
    const T* x = static_cast<const T*>(p.x);
    const bool flat = MODE == PLAIN && contiguous(p);
    const int64_t rows = flat ? 1 : p.x_rows * p.batch, cols = flat ? p.x_rows * p.batch * p.cols : p.cols;
    const int64_t per = ANY ? ceil_div(cols, P::kElems) : cols / P::kElems;     // whole pieces but for the end of a contiguous tensor
    const int64_t step = (int64_t)gridDim.x * kQThreads, div = per > 0 ? per : 1, drow = step / div, dpiece = step % div;
    const int64_t first = (int64_t)blockIdx.x * kQThreads + threadIdx.x;
    int64_t row = per > 0 ? first / div : rows, at = first % div;
    float m = 0.f;
    while (row < rows) {
        P v[kFlight];
        int64_t token[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            token[i] = row;
            v[i].clear();
            if (row < rows) {
                const T* from = x + (p.batch == 1 || flat ? row * p.ld : (row / p.x_rows) * p.batch_stride + (row % p.x_rows) * p.ld);
                if constexpr (ANY) load_any<T, BYTES>(v[i].w, from, at * P::kElems, cols);
                else v[i].load(from + at * P::kElems);
            }
            row += drow;
            at += dpiece;
            if (at >= per) { at -= per; ++row; }
        }
#pragma unroll
        for (int i = 0; i < kFlight; ++i)
            if (token[i] < rows) m = fmaxf(m, piece_max<T, BYTES, MODE>(v[i], p, token[i]));
    }
    if (!ANY && flat && blockIdx.x == 0 && per * P::kElems + threadIdx.x < cols) {
        Piece<T, (int)sizeof(T)> v;
        v.load(x + per * P::kElems + threadIdx.x);
        m = fmaxf(m, piece_max<T, (int)sizeof(T), PLAIN>(v, p, 0));
    }
    m = block_max(m, red);
    if (threadIdx.x == 0) part[blockIdx.x] = m;
}

// The tile in shared memory (COLS): rows of 128 elements without padding, their 16-byte chunks permuted, so that neither the
// threads that write units of two rows at a time nor those that walk down neighbouring columns meet bank conflicts: chunk c of
// row r is at c ^ (c / 8) ^ 2 (r & 1) for 16-bit elements (units of four chunks), c ^ (c / 8 + 4 (r & 1)) for 32-bit ones (eight).
template <bool NARROW> struct Tile {
    static constexpr int kPitch = 128 * (NARROW ? 2 : 4);
    static __device__ __forceinline__ int chunk(int row, int c) { return NARROW ? c ^ (c >> 3) ^ ((row & 1) << 1) : c ^ ((c >> 3) | ((row & 1) << 2)); }
};
// Codes of the transposed rows on their way out, 64 bytes each, permuted to the same end (even columns first).
__device__ __forceinline__ int stage_at(int lcol, int u) { return ((lcol >> 1) + 64 * (lcol & 1)) * 64 + ((u ^ ((lcol >> 2) & 3)) * 16); }

template <typename T, int FMT, bool ROWS, bool COLS, int MODE>
__global__ void __launch_bounds__(kQThreads, sizeof(T) == 2 && MODE != WEIGHTED ? 4 : 2) fp4_quant_kernel(const __grid_constant__ QuantParams p)
{
    constexpr bool kNarrow = sizeof(T) == 2 && MODE != WEIGHTED;          // the tile keeps the input's BF16 values
    using L = Tile<kNarrow>;
    constexpr int kPitch = L::kPitch;
    constexpr int kTiles = FMT == MOR_FP4_E4M3_16 ? 2 : 1;                // scale tiles per 128 elements
    constexpr int kPerUnit = Fp4<FMT>::kBlocksPerUnit;
    __shared__ float red[kQThreads / 32];
    __shared__ float factors[FMT == MOR_FP4_E4M3_16 ? 128 : 1];
    __shared__ __align__(16) uint8_t row_scales[ROWS ? kTiles * kScaleTile : 16];
    __shared__ __align__(16) uint8_t col_scales[COLS ? kTiles * kScaleTile : 16];
    extern __shared__ __align__(16) uint8_t dyn[];                        // COLS: tile, then the codes of the transposed rows
    const int tid = threadIdx.x;
    const uint32_t per = p.row_tiles * p.col_tiles, tiles = per * (uint32_t)p.batch;
    TensorScale ts = {1.f, 1.f, 1.f};
    for (uint64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const uint32_t batch = (uint32_t)tile / per, in_batch = (uint32_t)tile % per;
        const uint32_t row_tile = in_batch / p.col_tiles, col_tile = in_batch % p.col_tiles;
        const T* x = static_cast<const T*>(p.x) + (int64_t)batch * p.batch_stride;

        // both units' loads first: the tile is in flight while the tensor maximum is waited for (x is older than the kernel that takes it)
        const bool first = tile == blockIdx.x;
        if (first && (FMT != MOR_FP4_E4M3_16 || p.partial == nullptr)) wait_for_predecessor();
        Raw<T> raw[2];
        float weight[2] = {1.f, 1.f};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = tid + i * kQThreads;
            const int64_t row = (int64_t)row_tile * 128 + (at >> 2), col = (int64_t)col_tile * 128 + (at & 3) * kUnit;
            int64_t src = row;
            bool have = row < p.rows && col < p.cols;
            if constexpr (MODE != PLAIN) {
                const int32_t slot = row < p.rows ? p.slot_of_row[row] : -1;
                have = have && slot >= 0;
                src = have ? token_of((uint32_t)slot, p) : 0;
                if (MODE == WEIGHTED && have) weight[i] = weight_at(p.weight, p.weight_dtype, slot);
            }
            if (have && p.access < 16) load_any<T, (int)sizeof(Raw<T>)>(raw[i].w, x + src * p.ld, col, p.cols);
            else if (have) load_unit<T>(raw[i], x + src * p.ld + col, (int)min((int64_t)kUnit, p.cols - col), p.access);
            else
#pragma unroll
                for (uint32_t& w : raw[i].w) w = 0;
        }

        if (FMT == MOR_FP4_E4M3_16 && first) {
            float amax = 0.f;
            if (p.amax != nullptr) {
                amax = *p.amax;
            } else if (p.partial != nullptr) {
                wait_for_predecessor();
                for (uint32_t i = tid; i < p.n_partial; i += kQThreads) amax = fmaxf(amax, __ldcg(p.partial + i));
                amax = block_max(amax, red);
            } else {
                using P = Piece<T, 16>;
                const int64_t per = ceil_div(p.cols, P::kElems);
                for (int64_t i = tid; i < per * p.x_rows * p.batch; i += kQThreads) {
                    const int64_t r = i / per;
                    P v;
                    load_any<T, 16>(v.w, static_cast<const T*>(p.x) + (r / p.x_rows) * p.batch_stride + (r % p.x_rows) * p.ld, i % per * P::kElems, p.cols);
                    amax = fmaxf(amax, piece_max<T, 16, PLAIN>(v, p, 0));
                }
                amax = block_max(amax, red);
            }
            ts = tensor_scale_of(amax);
            fill_factors(factors, ts.t, tid);
            __syncthreads();
        }
        if (tile == 0 && tid == 0) {
            if (ROWS) *p.r_t = ts.t;
            if (COLS) *p.c_t = ts.t;
        }

#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = tid + i * kQThreads, lrow = at >> 2, u = at & 3;
            const int64_t row = (int64_t)row_tile * 128 + lrow, col = (int64_t)col_tile * 128 + u * kUnit;
            float v[kNarrow ? 1 : kUnit];                                       // FP32, or BF16 as it came
            if constexpr (!kNarrow) unpack<T>(raw[i], v);
            if constexpr (MODE == WEIGHTED) {
#pragma unroll
                for (float& e : v) e *= weight[i];
            }
            if constexpr (COLS) {
                uint8_t* to = dyn + lrow * kPitch;
                if constexpr (kNarrow) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        *reinterpret_cast<uint4*>(to + L::chunk(lrow, u * 4 + j) * 16) = make_uint4(raw[i].w[4 * j], raw[i].w[4 * j + 1], raw[i].w[4 * j + 2], raw[i].w[4 * j + 3]);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) *reinterpret_cast<float4*>(to + L::chunk(lrow, u * 8 + j) * 16) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                }
            }
            if constexpr (ROWS) {
                uint32_t scales;
                float a[kPerUnit];
#pragma unroll
                for (int k = 0; k < kPerUnit; ++k) {
                    if constexpr (kNarrow) a[k] = amax_of_pair(amax_of_words<16 / kPerUnit>(raw[i].w + k * (16 / kPerUnit)));
                    else a[k] = amax_of<kUnit / kPerUnit>(v + k * (kUnit / kPerUnit));
                }
                uint4 codes;
                if constexpr (kNarrow) codes = quantise_unit<FMT>(UnitBf16<PAIRS>{raw[i].w}, a, ts, factors, scales);
                else codes = quantise_unit<FMT>(UnitF32{v}, a, ts, factors, scales);
                if (row < p.rows && col < p.cols)
                    *reinterpret_cast<uint4*>(p.r_codes + ((int64_t)batch * p.rows + row) * p.r_ld + col / 2) = codes;
                uint8_t* s = row_scales + ((u * kPerUnit) >> 2) * kScaleTile + scale_at(lrow, u * kPerUnit);
                if constexpr (kPerUnit == 2) *reinterpret_cast<uint16_t*>(s) = row < p.rows && col < p.cols ? (uint16_t)scales : 0;
                else *s = row < p.rows && col < p.cols ? (uint8_t)scales : 0;
            }
        }
        __syncthreads();
        if constexpr (ROWS) {
            const uint32_t ktile = col_tile * kTiles + (tid >> 5);
            if (tid < kTiles * 32 && ktile < p.r_ktiles)
                *reinterpret_cast<uint4*>(p.r_scales + (((int64_t)batch * p.row_tiles + row_tile) * p.r_ktiles + ktile) * kScaleTile + (tid & 31) * 16) =
                    *reinterpret_cast<const uint4*>(row_scales + tid * 16);
        }
        if constexpr (COLS) {
            uint8_t* stage = dyn + 128 * kPitch;
            auto put = [&](int lcol, int u, const auto& unit, const float* a) {
                uint32_t scales;
                const uint4 codes = quantise_unit<FMT>(unit, a, ts, factors, scales);
                *reinterpret_cast<uint4*>(stage + stage_at(lcol, u)) = codes;
                const bool in = (int64_t)col_tile * 128 + lcol < p.cols && (int64_t)row_tile * 128 + u * kUnit < p.rows;
                uint8_t* s = col_scales + ((u * kPerUnit) >> 2) * kScaleTile + scale_at(lcol, u * kPerUnit);
                if constexpr (kPerUnit == 2) *reinterpret_cast<uint16_t*>(s) = in ? (uint16_t)scales : 0;
                else *s = in ? (uint8_t)scales : 0;
            };
            if constexpr (kNarrow) {             // two neighbouring columns (one word) over 32 rows
                const int pair = tid & 63, u = tid >> 6;
                const uint8_t* from[2] = {dyn + u * kUnit * kPitch + L::chunk(0, pair >> 2) * 16 + (pair & 3) * 4,
                                          dyn + u * kUnit * kPitch + L::chunk(1, pair >> 2) * 16 + (pair & 3) * 4};
                uint32_t w[kUnit], m[kPerUnit];
                float a[kPerUnit];
#pragma unroll
                for (int i = 0; i < kUnit; ++i) w[i] = *reinterpret_cast<const uint32_t*>(from[i & 1] + i * kPitch);
#pragma unroll
                for (int k = 0; k < kPerUnit; ++k) m[k] = amax_of_words<kUnit / kPerUnit>(w + k * (kUnit / kPerUnit));
#pragma unroll
                for (int k = 0; k < kPerUnit; ++k) a[k] = fabsf(bf16_low(m[k]));
                put(2 * pair, u, UnitBf16<LOW>{w}, a);
#pragma unroll
                for (int k = 0; k < kPerUnit; ++k) a[k] = fabsf(bf16_high(m[k]));
                put(2 * pair + 1, u, UnitBf16<HIGH>{w}, a);
            } else {
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    const int lcol = tid & 127, u = (tid >> 7) + 2 * half;
                    float v[kUnit], a[kPerUnit];
#pragma unroll
                    for (int i = 0; i < kUnit; ++i) v[i] = *reinterpret_cast<const float*>(dyn + (u * kUnit + i) * kPitch + L::chunk(i & 1, lcol >> 2) * 16 + (lcol & 3) * 4);
#pragma unroll
                    for (int k = 0; k < kPerUnit; ++k) a[k] = amax_of<kUnit / kPerUnit>(v + k * (kUnit / kPerUnit));
                    put(lcol, u, UnitF32{v}, a);
                }
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int at = tid + i * kQThreads, lcol = at >> 2, u = at & 3;
                const int64_t col = (int64_t)col_tile * 128 + lcol, row = (int64_t)row_tile * 128 + u * kUnit;
                if (col < p.cols && row < p.rows)
                    *reinterpret_cast<uint4*>(p.c_codes + ((int64_t)batch * p.cols + col) * p.c_ld + row / 2) =
                        *reinterpret_cast<const uint4*>(stage + stage_at(lcol, u));
            }
            const uint32_t ktile = row_tile * kTiles + (tid >> 5);
            if (tid < kTiles * 32 && ktile < p.c_ktiles)
                *reinterpret_cast<uint4*>(p.c_scales + (((int64_t)batch * p.c_row_tiles + col_tile) * p.c_ktiles + ktile) * kScaleTile + (tid & 31) * 16) =
                    *reinterpret_cast<const uint4*>(col_scales + tid * 16);
        }
        __syncthreads();
    }
}

// ---- large BF16 tensors in the column direction: the same tiles, streamed
//
// Persistent CTAs, two an SM.  While a tile is converted, the next one is on its way into the other half of the shared memory
// (asynchronous 16-byte copies to the permuted chunks, zero-filled past the edges), so loads never wait for arithmetic: with one
// tile per CTA the loads stood still for most of its life.  8192 x 14336, columns alone: E4M3_16 66 us with a CTA per tile, 49 us
// (6.1 TB/s) streamed; both directions 60 us, E8M0_32 62 us.  Three CTAs an SM have a third fewer registers and form their
// addresses anew all the time (64 and 68 us); a ring of three tiles in place of two gained nothing (63 us).
__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

constexpr int kStreamTile = 128 * Tile<true>::kPitch;
constexpr int kStreamSmem = 2 * kStreamTile + 128 * 64;
constexpr uint32_t kStreamTiles = 148 * 4;      // below, every tile has a CTA of its own and there is nothing to stream

// Where a CTA is in the grid of tiles; advanced by its stride without divisions.
struct TileWalk {
    uint32_t batch, row, col;
    __device__ __forceinline__ TileWalk(const QuantParams& p, uint32_t tile)
    {
        const uint32_t per = p.row_tiles * p.col_tiles;
        batch = tile / per;
        row = tile % per / p.col_tiles;
        col = tile % per % p.col_tiles;
    }
    __device__ __forceinline__ void advance(const QuantParams& p, const TileWalk& step)
    {
        batch += step.batch;
        row += step.row;
        col += step.col;
        if (col >= p.col_tiles) { col -= p.col_tiles; ++row; }
        if (row >= p.row_tiles) { row -= p.row_tiles; ++batch; }
    }
};

// The arithmetic of a tile is about five instructions per element; addresses are formed once per tile and thread and stepped
// by constants, since 64-bit products per access came to as much again.
template <int FMT, bool ROWS, int MODE>
__global__ void __launch_bounds__(kQThreads, 2) fp4_stream_kernel(const __grid_constant__ QuantParams p, uint32_t tiles)
{
    using L = Tile<true>;
    constexpr int kTiles = FMT == MOR_FP4_E4M3_16 ? 2 : 1;
    constexpr int kPerUnit = Fp4<FMT>::kBlocksPerUnit;
    // 16-byte chunks: chunk tid % 16 of every 16th row; gathered, four chunks of every 64th row, so that a thread looks up two
    // rows (a quarter of a row is still two whole sectors)
    constexpr int kRowsOf = MODE == PLAIN ? 8 : 2, kChunksOf = MODE == PLAIN ? 1 : 4, kRowStep = 128 / kRowsOf;
    __shared__ float red[kQThreads / 32];
    __shared__ float factors[FMT == MOR_FP4_E4M3_16 ? 128 : 1];
    __shared__ __align__(16) float weights[MODE == WEIGHTED ? 2 * 128 : 4];
    __shared__ __align__(16) uint8_t row_scales[ROWS ? kTiles * kScaleTile : 16];
    __shared__ __align__(16) uint8_t col_scales[kTiles * kScaleTile];
    extern __shared__ __align__(16) uint8_t dyn[];                        // two tiles, then the codes of the transposed rows
    const int tid = threadIdx.x;

    const int c_row = MODE == PLAIN ? tid >> 4 : tid >> 2, c_chunk = MODE == PLAIN ? tid & 15 : tid & 3;
    const uint32_t c_to = (uint32_t)__cvta_generic_to_shared(dyn) + c_row * L::kPitch;
    const int64_t c_step = 2 * kRowStep * p.ld;                           // bytes between this thread's rows
    int32_t slot[MODE == PLAIN ? 1 : kRowsOf];                            // of the next tile to fetch
    float weight[MODE == WEIGHTED ? kRowsOf : 1];
    auto look_up = [&](const TileWalk& t, bool have) {
        if constexpr (MODE != PLAIN) {
#pragma unroll
            for (int i = 0; i < kRowsOf; ++i) {
                const int64_t row = (int64_t)t.row * 128 + c_row + kRowStep * i;
                slot[i] = have && row < p.rows ? p.slot_of_row[row] : -1;
                if constexpr (MODE == WEIGHTED) weight[i] = slot[i] >= 0 ? weight_at(p.weight, p.weight_dtype, slot[i]) : 0.f;
            }
        }
    };
    auto fetch = [&](const TileWalk& t, bool have, uint32_t half) {
        if (have) {
            const int64_t col = (int64_t)t.col * 128 + c_chunk * 8, row = (int64_t)t.row * 128 + c_row;
            const char* x = static_cast<const char*>(p.x) + 2 * col;
            const int cols = (int)max((int64_t)-128, min((int64_t)128, p.cols - col));        // from the thread's first chunk on
            if constexpr (MODE == PLAIN) {
                const char* from = x + 2 * ((int64_t)t.batch * p.batch_stride + row * p.ld);
                const uint32_t to = c_to + half + L::chunk(c_row, c_chunk) * 16;              // all rows of one parity: one place
                const int room = max(0, min(8, cols)) * 2, left = (int)min((int64_t)128, p.rows - row);
                if (room == 16 && left > kRowStep * (kRowsOf - 1)) {
#pragma unroll
                    for (int i = 0; i < kRowsOf; ++i, from += c_step) copy_async16(to + i * kRowStep * L::kPitch, from, 16);
                } else {
#pragma unroll 1
                    for (int i = 0; i < kRowsOf; ++i, from += c_step) {
                        const bool in = kRowStep * i < left && room > 0;
                        copy_async16(to + i * kRowStep * L::kPitch, in ? from : static_cast<const char*>(p.x), in ? room : 0);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < kRowsOf; ++i) {
                    const bool in = slot[i] >= 0;
                    const char* from = x + 2 * ((in ? token_of((uint32_t)slot[i], p) : 0) * p.ld);
#pragma unroll
                    for (int j0 = 0; j0 < kChunksOf; ++j0) {
                        const int j = j0 ^ (c_row & 1);                                       // neighbouring rows in other banks
                        const int room = in ? max(0, min(8, cols - 32 * j)) * 2 : 0;
                        copy_async16(c_to + half + i * kRowStep * L::kPitch + L::chunk(c_row, c_chunk + 4 * j) * 16,
                                     room > 0 ? from + 64 * j : static_cast<const char*>(p.x), room);
                    }
                    if (MODE == WEIGHTED && c_chunk == 0) weights[(half ? 128 : 0) + c_row + kRowStep * i] = weight[i];
                }
            }
        }
        copy_async_commit();
    };
    const TileWalk step(p, gridDim.x);
    TileWalk now(p, blockIdx.x), next = now;
    uint32_t tile = blockIdx.x;
    if (FMT != MOR_FP4_E4M3_16 || p.partial == nullptr) wait_for_predecessor();     // else x is older than the predecessor
    look_up(now, tile < tiles);
    fetch(now, tile < tiles, 0);
    next.advance(p, step);
    look_up(next, tile + gridDim.x < tiles);

    TensorScale ts = {1.f, 1.f, 1.f};
    if constexpr (FMT == MOR_FP4_E4M3_16) {
        float amax = 0.f;
        if (p.amax != nullptr) {
            amax = *p.amax;
        } else {
            wait_for_predecessor();
            for (uint32_t i = tid; i < p.n_partial; i += kQThreads) amax = fmaxf(amax, __ldcg(p.partial + i));
            amax = block_max(amax, red);
        }
        ts = tensor_scale_of(amax);
        fill_factors(factors, ts.t, tid);                                  // read after the loop's first barrier
    }
    if (blockIdx.x == 0 && tid == 0) {
        if (ROWS) *p.r_t = ts.t;
        *p.c_t = ts.t;
    }

    // rows: unit tid % 4 of rows tid / 4 and 64 + tid / 4; columns: two neighbours (one word) over the 32 rows of unit tid / 64
    const int r_row = tid >> 2, r_unit = tid & 3, pair = tid & 63, unit = tid >> 6;
    uint8_t* const stage = dyn + 2 * kStreamTile;
    uint32_t half = 0;                                                     // byte offset of the tile at hand
    for (; tile < tiles; tile += gridDim.x) {
        fetch(next, tile + gridDim.x < tiles, half ^ kStreamTile);
        TileWalk after = next;
        after.advance(p, step);
        look_up(after, tile + 2 * (uint64_t)gridDim.x < tiles);
        copy_async_wait<1>();
        __syncthreads();
        const uint8_t* in = dyn + half;
        const float* of_rows = weights + (half ? 128 : 0);
        const int rows_left = (int)min((int64_t)128, p.rows - (int64_t)now.row * 128), cols_left = (int)min((int64_t)128, p.cols - (int64_t)now.col * 128);
        if constexpr (ROWS) {
            uint8_t* to = p.r_codes + ((int64_t)now.batch * p.rows + (int64_t)now.row * 128 + r_row) * p.r_ld + now.col * 64 + r_unit * 16;
            const uint8_t* from = in + r_row * L::kPitch;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t w[16], scales;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint4 q = *reinterpret_cast<const uint4*>(from + i * 64 * L::kPitch + L::chunk(r_row, r_unit * 4 + j) * 16);
                    w[4 * j] = q.x; w[4 * j + 1] = q.y; w[4 * j + 2] = q.z; w[4 * j + 3] = q.w;
                }
                float a[kPerUnit];
                uint4 codes;
                if constexpr (MODE == WEIGHTED) {
                    const float f = of_rows[r_row + 64 * i];
                    float v[kUnit];
#pragma unroll
                    for (int j = 0; j < 16; ++j) { v[2 * j] = bf16_low(w[j]) * f; v[2 * j + 1] = bf16_high(w[j]) * f; }
#pragma unroll
                    for (int k = 0; k < kPerUnit; ++k) a[k] = amax_of<kUnit / kPerUnit>(v + k * (kUnit / kPerUnit));
                    codes = quantise_unit<FMT>(UnitF32{v}, a, ts, factors, scales);
                } else {
#pragma unroll
                    for (int k = 0; k < kPerUnit; ++k) a[k] = amax_of_pair(amax_of_words<16 / kPerUnit>(w + k * (16 / kPerUnit)));
                    codes = quantise_unit<FMT>(UnitBf16<PAIRS>{w}, a, ts, factors, scales);
                }
                const bool inside = r_row + 64 * i < rows_left && r_unit * kUnit < cols_left;
                if (inside) *reinterpret_cast<uint4*>(to + i * 64 * p.r_ld) = codes;
                uint8_t* s = row_scales + ((r_unit * kPerUnit) >> 2) * kScaleTile + scale_at(r_row + 64 * i, r_unit * kPerUnit);
                if constexpr (kPerUnit == 2) *reinterpret_cast<uint16_t*>(s) = inside ? (uint16_t)scales : 0;
                else *s = inside ? (uint8_t)scales : 0;
            }
        }
        {
            const uint8_t* from[2] = {in + unit * kUnit * L::kPitch + L::chunk(0, pair >> 2) * 16 + (pair & 3) * 4,
                                      in + unit * kUnit * L::kPitch + L::chunk(1, pair >> 2) * 16 + (pair & 3) * 4};
            uint32_t w[kUnit];
#pragma unroll
            for (int i = 0; i < kUnit; ++i) w[i] = *reinterpret_cast<const uint32_t*>(from[i & 1] + i * L::kPitch);
            auto put = [&](int lcol, const auto& values, const float* a) {
                uint32_t scales;
                const uint4 codes = quantise_unit<FMT>(values, a, ts, factors, scales);
                *reinterpret_cast<uint4*>(stage + stage_at(lcol, unit)) = codes;
                const bool inside = lcol < cols_left && unit * kUnit < rows_left;
                uint8_t* s = col_scales + ((unit * kPerUnit) >> 2) * kScaleTile + scale_at(lcol, unit * kPerUnit);
                if constexpr (kPerUnit == 2) *reinterpret_cast<uint16_t*>(s) = inside ? (uint16_t)scales : 0;
                else *s = inside ? (uint8_t)scales : 0;
            };
            float a[kPerUnit];
            if constexpr (MODE == WEIGHTED) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float v[kUnit];
#pragma unroll
                    for (int i = 0; i < kUnit; i += 4) {
                        const float4 f = *reinterpret_cast<const float4*>(of_rows + unit * kUnit + i);
                        v[i] = (c ? bf16_high(w[i]) : bf16_low(w[i])) * f.x;
                        v[i + 1] = (c ? bf16_high(w[i + 1]) : bf16_low(w[i + 1])) * f.y;
                        v[i + 2] = (c ? bf16_high(w[i + 2]) : bf16_low(w[i + 2])) * f.z;
                        v[i + 3] = (c ? bf16_high(w[i + 3]) : bf16_low(w[i + 3])) * f.w;
                    }
#pragma unroll
                    for (int k = 0; k < kPerUnit; ++k) a[k] = amax_of<kUnit / kPerUnit>(v + k * (kUnit / kPerUnit));
                    put(2 * pair + c, UnitF32{v}, a);
                }
            } else {
                uint32_t m[kPerUnit];
#pragma unroll
                for (int k = 0; k < kPerUnit; ++k) m[k] = amax_of_words<kUnit / kPerUnit>(w + k * (kUnit / kPerUnit));
#pragma unroll
                for (int k = 0; k < kPerUnit; ++k) a[k] = fabsf(bf16_low(m[k]));
                put(2 * pair, UnitBf16<LOW>{w}, a);
#pragma unroll
                for (int k = 0; k < kPerUnit; ++k) a[k] = fabsf(bf16_high(m[k]));
                put(2 * pair + 1, UnitBf16<HIGH>{w}, a);
            }
        }
        __syncthreads();
        {
            uint8_t* to = p.c_codes + ((int64_t)now.batch * p.cols + (int64_t)now.col * 128 + r_row) * p.c_ld + now.row * 64 + r_unit * 16;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (r_row + 64 * i < cols_left && r_unit * kUnit < rows_left)
                    *reinterpret_cast<uint4*>(to + i * 64 * p.c_ld) = *reinterpret_cast<const uint4*>(stage + stage_at(r_row + 64 * i, r_unit));
        }
        if (ROWS && tid < kTiles * 32) {
            const uint32_t ktile = now.col * kTiles + (tid >> 5);
            if (ktile < p.r_ktiles)
                *reinterpret_cast<uint4*>(p.r_scales + (((int64_t)now.batch * p.row_tiles + now.row) * p.r_ktiles + ktile) * kScaleTile + (tid & 31) * 16) =
                    *reinterpret_cast<const uint4*>(row_scales + tid * 16);
        }
        if (tid >= 128 && tid < 128 + kTiles * 32) {
            const int t = tid - 128;
            const uint32_t ktile = now.row * kTiles + (t >> 5);
            if (ktile < p.c_ktiles)
                *reinterpret_cast<uint4*>(p.c_scales + (((int64_t)now.batch * p.c_row_tiles + now.col) * p.c_ktiles + ktile) * kScaleTile + (t & 31) * 16) =
                    *reinterpret_cast<const uint4*>(col_scales + t * 16);
        }
        now = next;
        next = after;
        half ^= kStreamTile;
    }
}

// A tensor without elements has no codes, but a tensor scale like any other.
__global__ void fp4_empty_kernel(int format, const float* amax, float* r_t, float* c_t)
{
    wait_for_predecessor();
    const float t = format == MOR_FP4_E4M3_16 ? tensor_scale_of(amax != nullptr ? *amax : 0.f).t : 1.f;
    if (r_t != nullptr) *r_t = t;
    if (c_t != nullptr) *c_t = t;
}

struct DequantParams {
    const uint8_t *codes, *scales;
    const float* t;
    int64_t rows, cols, ld, ldo;
    uint32_t row_tiles, col_tiles, ktiles;
    int32_t access;
    void* out;
};

// The inverse: 0.5 + 1/16 (1/32) bytes in, 2 (4) out per element; bound by memory (8192 x 14336 to BF16: 48 us, 6.2 TB/s).  The tile's scales come in whole scale tiles; a thread
// turns 16 bytes of codes into 32 values.
template <typename T, int FMT> __global__ void __launch_bounds__(kQThreads) fp4_dequant_kernel(const __grid_constant__ DequantParams p)
{
    constexpr int kTiles = FMT == MOR_FP4_E4M3_16 ? 2 : 1;
    constexpr int kPerUnit = Fp4<FMT>::kBlocksPerUnit;
    constexpr int kPitch = 128 * (int)sizeof(T) + 16;
    extern __shared__ __align__(16) uint8_t dyn[];                  // rows that start anywhere: the tile's values
    __shared__ __align__(16) uint8_t scales[kTiles * kScaleTile];
    const int tid = threadIdx.x;
    const uint32_t per = p.row_tiles * p.col_tiles;
    const uint32_t batch = blockIdx.x / per, in_batch = blockIdx.x % per;
    const uint32_t row_tile = in_batch / p.col_tiles, col_tile = in_batch % p.col_tiles;
    uint4 codes[2];
    wait_for_predecessor();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int at = tid + i * kQThreads;
        const int64_t row = (int64_t)row_tile * 128 + (at >> 2), col = (int64_t)col_tile * 128 + (at & 3) * kUnit;
        if (row < p.rows && col < p.cols) codes[i] = *reinterpret_cast<const uint4*>(p.codes + ((int64_t)batch * p.rows + row) * p.ld + col / 2);
    }
    const uint32_t ktile = col_tile * kTiles + (tid >> 5);
    if (tid < kTiles * 32 && ktile < p.ktiles)
        *reinterpret_cast<uint4*>(scales + tid * 16) =
            *reinterpret_cast<const uint4*>(p.scales + (((int64_t)batch * p.row_tiles + row_tile) * p.ktiles + ktile) * kScaleTile + (tid & 31) * 16);
    const float t = *p.t;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int at = tid + i * kQThreads, lrow = at >> 2, u = at & 3;
        const int64_t row = (int64_t)row_tile * 128 + lrow, col = (int64_t)col_tile * 128 + u * kUnit;
        if (row >= p.rows || col >= p.cols) continue;
        const uint8_t* s = scales + ((u * kPerUnit) >> 2) * kScaleTile + scale_at(lrow, u * kPerUnit);
        const float s0 = scale_value<FMT>(s[0]), s1 = kPerUnit == 2 ? scale_value<FMT>(s[kPerUnit - 1]) : s0;
        const uint32_t c[4] = {codes[i].x, codes[i].y, codes[i].z, codes[i].w};
        float v[kUnit];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float2 d = e2m1x2_value((c[j >> 2] >> (8 * (j & 3))) & 0xFFu);
            const float sc = j < 8 ? s0 : s1;
            v[2 * j] = (d.x * sc) * t;
            v[2 * j + 1] = (d.y * sc) * t;
        }
        T* to = static_cast<T*>(p.out) + ((int64_t)batch * p.rows + row) * p.ldo + col;
        const int n = (int)min((int64_t)kUnit, p.cols - col);
        constexpr int kWords = kUnit * sizeof(T) / 4;
        uint32_t w[kWords];
#pragma unroll
        for (int j = 0; j < kWords; ++j) {
            if constexpr (sizeof(T) == 2) w[j] = bf16x2_of(v[2 * j], v[2 * j + 1]);
            else w[j] = __float_as_uint(v[j]);
        }
        if (p.access < 16) {
#pragma unroll
            for (int j = 0; j < kWords; j += 4)
                *reinterpret_cast<uint4*>(dyn + lrow * kPitch + u * kUnit * sizeof(T) + 4 * j) = make_uint4(w[j], w[j + 1], w[j + 2], w[j + 3]);
        } else if (n == kUnit && p.access == 32) {
#pragma unroll
            for (int j = 0; j < kWords; j += 8) stg256(reinterpret_cast<uint32_t*>(to) + j, w + j);
        } else if (n == kUnit) {
#pragma unroll
            for (int j = 0; j < kWords; j += 4) *reinterpret_cast<uint4*>(reinterpret_cast<uint32_t*>(to) + j) = make_uint4(w[j], w[j + 1], w[j + 2], w[j + 3]);
        } else {
#pragma unroll
            for (int j = 0; j < kUnit; ++j) {
                if (j >= n) break;
                if constexpr (sizeof(T) == 2) reinterpret_cast<uint16_t*>(to)[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
                else reinterpret_cast<uint32_t*>(to)[j] = w[j];
            }
        }
    }
    if (p.access >= 16) return;
    __syncthreads();
    for (int r = tid >> 5; r < 128; r += kQThreads / 32) {
        const int64_t row = (int64_t)row_tile * 128 + r;
        if (row >= p.rows) break;
        const T* from = reinterpret_cast<const T*>(dyn + r * kPitch);
        T* to = static_cast<T*>(p.out) + ((int64_t)batch * p.rows + row) * p.ldo + (int64_t)col_tile * 128;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = j * 32 + (tid & 31);
            if ((int64_t)col_tile * 128 + c < p.cols) to[c] = from[c];
        }
    }
}

template <typename T, int FMT, bool ROWS, bool COLS, int MODE> cudaError_t quant_launch(const QuantParams& p, uint32_t grid, cudaStream_t st)
{
    if constexpr (sizeof(T) == 2 && COLS) {
        if (p.access >= 16 && grid >= kStreamTiles && (FMT == MOR_FP4_E8M0_32 || p.amax != nullptr || p.partial != nullptr)) {
            static std::atomic<uint64_t> stream_done{0};
            if (!allow_smem(fp4_stream_kernel<FMT, ROWS, MODE>, kStreamSmem, stream_done)) return cudaErrorInvalidValue;
            return launch(fp4_stream_kernel<FMT, ROWS, MODE>, grid < 148 * 2 ? grid : 148 * 2, kQThreads, kStreamSmem, st, true, p, grid);
        }
    }
    constexpr bool kNarrow = sizeof(T) == 2 && MODE != WEIGHTED;
    constexpr int smem = COLS ? 128 * Tile<kNarrow>::kPitch + 128 * 64 : 0;
    static std::atomic<uint64_t> done{0};
    if (smem > 0 && !allow_smem(fp4_quant_kernel<T, FMT, ROWS, COLS, MODE>, smem, done)) return cudaErrorInvalidValue;
    // As many CTAs as are resident, each walking its tiles: the tensor's scale and its table are made once a CTA (8192 x 14336 E4M3_16 rows
    // with the maximum 91 us, 104 with a CTA per tile; 4096 x 4096 15 and 18.5), and the kernel may start early (4096 x 4096 E8M0_32
    // 8.0 us and 10.3).  E8M0_32 has nothing to share, and a CTA per tile is ahead beyond 1024 tiles (rows alone, walked and not, in a graph: 512
    // tiles BF16 5.3 and 5.6 us, FP32 9.2 and 10.5; 1024: 8.6 and 8.7, 16.0 and 16.1; 2048: 15.8 and 15.2, 30.1 and 28.9; 7168: 47.6 and
    // 45.2, 97 and 89).
    constexpr uint32_t most = 148 * (kNarrow ? 4 : 2);
    const bool walk = FMT == MOR_FP4_E4M3_16 || grid <= 1024;
    return launch(fp4_quant_kernel<T, FMT, ROWS, COLS, MODE>, walk && grid > most ? most : grid, kQThreads, smem, st, walk, p);
}
template <typename T, int FMT, int MODE> cudaError_t quant_dirs(const QuantParams& p, uint32_t grid, cudaStream_t st)
{
    if (p.r_codes != nullptr && p.c_codes != nullptr) return quant_launch<T, FMT, true, true, MODE>(p, grid, st);
    if (p.r_codes != nullptr) return quant_launch<T, FMT, true, false, MODE>(p, grid, st);
    return quant_launch<T, FMT, false, true, MODE>(p, grid, st);
}
template <typename T, int MODE> cudaError_t quant_all(const QuantParams& p, int format, uint32_t amax_grid, uint32_t grid, float* part, cudaStream_t st)
{
    if (amax_grid > 0) {
        // rows that may be taken as one long one need no alignment but the first's
        const bool flat = MODE == PLAIN && contiguous(p);
        const int64_t width = flat ? 0 : p.cols * (int64_t)sizeof(T);
        const int access = flat ? access_bytes(p.x, 0, 0, (int)sizeof(T)) : p.access;
        const cudaError_t e = access == 32 && width % 32 == 0   ? launch(fp4_amax_kernel<T, 32, MODE, false>, amax_grid, kQThreads, 0, st, true, p, part)
                              : access >= 16 && width % 16 == 0 ? launch(fp4_amax_kernel<T, 16, MODE, false>, amax_grid, kQThreads, 0, st, true, p, part)
                                                                : launch(fp4_amax_kernel<T, 16, MODE, true>, amax_grid, kQThreads, 0, st, true, p, part);
        if (e != cudaSuccess) return e;
    }
    return format == MOR_FP4_E4M3_16 ? quant_dirs<T, MOR_FP4_E4M3_16, MODE>(p, grid, st) : quant_dirs<T, MOR_FP4_E8M0_32, MODE>(p, grid, st);
}
template <typename T> cudaError_t quant_mode(const QuantParams& p, int format, uint32_t amax_grid, uint32_t grid, float* part, cudaStream_t st)
{
    if (p.slot_of_row == nullptr) return quant_all<T, PLAIN>(p, format, amax_grid, grid, part, st);
    if (p.weight == nullptr) return quant_all<T, GATHER>(p, format, amax_grid, grid, part, st);
    return quant_all<T, WEIGHTED>(p, format, amax_grid, grid, part, st);
}

}  // namespace
}  // namespace mor

using namespace mor;

extern "C" {

size_t mor_fp4_scale_bytes(int64_t batch, int64_t rows, int64_t cols, int format)
{
    if (!shape_ok(batch, rows, cols) || (format != MOR_FP4_E4M3_16 && format != MOR_FP4_E8M0_32)) return 0;
    return (size_t)batch * ceil_div(rows, 128) * scale_ktiles(cols, format) * kScaleTile;
}

mor_status_t mor_fp4_quantize(const mor_fp4_quantize_desc_t* host_desc, const mor_fp4_matrix_t* host_rows,
                              const mor_fp4_matrix_t* host_cols, void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    if (host_desc == nullptr || (host_rows == nullptr && host_cols == nullptr)) return MOR_ERR_INVALID_ARG;
    const mor_fp4_quantize_desc_t& d = *host_desc;
    const bool gather = d.slot_of_row != nullptr;
    if (!is_dtype(d.dtype) || (d.format != MOR_FP4_E4M3_16 && d.format != MOR_FP4_E8M0_32)) return MOR_ERR_INVALID_ARG;
    if (!shape_ok(d.batch, d.rows, d.cols) || d.ld < d.cols || d.batch_stride < 0) return MOR_ERR_INVALID_ARG;
    if (gather && (d.batch != 1 || d.top < 1 || d.row_of_slot == nullptr || !shape_ok(1, d.out_rows, d.cols))) return MOR_ERR_INVALID_ARG;
    if (gather && d.weight != nullptr && !is_dtype(d.weight_dtype)) return MOR_ERR_INVALID_ARG;
    if (!gather && d.weight != nullptr) return MOR_ERR_INVALID_ARG;
    const int64_t rows = gather ? d.out_rows : d.rows;
    const bool empty = d.batch == 0 || rows == 0 || d.cols == 0;
    if (!empty && d.x == nullptr && d.rows > 0) return MOR_ERR_INVALID_ARG;
    const int es = (int)dtype_bytes(d.dtype);
    if (!is_aligned(d.x, es)) return MOR_ERR_ALIGNMENT;
    if (host_rows != nullptr) {
        const mor_status_t s = check_matrix(*host_rows);
        if (s != MOR_OK) return s;
        if (host_rows->batch != d.batch || host_rows->rows != rows || host_rows->cols != d.cols || host_rows->format != d.format) return MOR_ERR_INVALID_ARG;
    }
    if (host_cols != nullptr) {
        const mor_status_t s = check_matrix(*host_cols);
        if (s != MOR_OK) return s;
        if (host_cols->batch != d.batch || host_cols->rows != d.cols || host_cols->cols != rows || host_cols->format != d.format) return MOR_ERR_INVALID_ARG;
    }
    const int64_t elems = d.batch * d.rows * d.cols;
    const bool want_amax = d.format == MOR_FP4_E4M3_16 && d.amax == nullptr;
    const bool amax_kernel = want_amax && (gather || elems > kSelfAmaxElems);
    if (want_amax) {
        if (workspace == nullptr || workspace_bytes < MOR_FP4_WORKSPACE_BYTES) return MOR_ERR_WORKSPACE;
        if (!is_aligned(workspace, 16)) return MOR_ERR_ALIGNMENT;
    }
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (empty) {
        float *r_t = host_rows != nullptr ? host_rows->tensor_scale : nullptr, *c_t = host_cols != nullptr ? host_cols->tensor_scale : nullptr;
        return launch(fp4_empty_kernel, 1, 1, 0, st, true, d.format, d.amax, r_t, c_t) == cudaSuccess ? MOR_OK : MOR_ERR_CUDA;
    }

    QuantParams p = {};
    p.x = d.x;
    p.ld = d.ld;
    p.batch_stride = d.batch_stride;
    p.rows = rows;
    p.cols = d.cols;
    p.x_rows = d.rows;
    p.batch = d.batch;
    p.row_tiles = (uint32_t)ceil_div(rows, 128);
    p.col_tiles = (uint32_t)ceil_div(d.cols, 128);
    p.access = access_bytes(d.x, d.ld * es, d.batch > 1 ? d.batch_stride * es : 0, es);
    p.amax = d.format == MOR_FP4_E4M3_16 ? d.amax : nullptr;
    p.slot_of_row = d.slot_of_row;
    p.row_of_slot = d.row_of_slot;
    p.top = (uint32_t)(gather ? d.top : 1);
    p.inv_top = 0xFFFFFFFFu / p.top;
    p.weight = d.weight;
    p.weight_dtype = d.weight_dtype;
    if (host_rows != nullptr) {
        p.r_codes = host_rows->codes;
        p.r_scales = host_rows->scales;
        p.r_ld = host_rows->ld;
        p.r_t = host_rows->tensor_scale;
        p.r_ktiles = (uint32_t)scale_ktiles(d.cols, d.format);
    }
    if (host_cols != nullptr) {
        p.c_codes = host_cols->codes;
        p.c_scales = host_cols->scales;
        p.c_ld = host_cols->ld;
        p.c_t = host_cols->tensor_scale;
        p.c_ktiles = (uint32_t)scale_ktiles(rows, d.format);
        p.c_row_tiles = p.col_tiles;
    }
    uint32_t amax_grid = 0;
    if (amax_kernel) {
        const int64_t want = ceil_div(elems * es, 128 * kQThreads);           // four pieces of 32 bytes a thread
        amax_grid = (uint32_t)(want < 1 ? 1 : want > 148 * 4 ? 148 * 4 : want);
        static_assert(148 * 4 <= kAmaxMaxBlocks, "parts fit the workspace");
        p.partial = static_cast<const float*>(workspace);
        p.n_partial = amax_grid;
    }
    const uint32_t grid = (uint32_t)(d.batch * p.row_tiles * p.col_tiles);
    const cudaError_t e = d.dtype == MOR_DTYPE_BF16 ? quant_mode<__nv_bfloat16>(p, d.format, amax_grid, grid, static_cast<float*>(workspace), st)
                                                    : quant_mode<float>(p, d.format, amax_grid, grid, static_cast<float*>(workspace), st);
    return e == cudaSuccess ? MOR_OK : MOR_ERR_CUDA;
}

mor_status_t mor_fp4_dequantize(const mor_fp4_matrix_t* host_in, void* out, int dtype, int64_t ld_out, void* cuda_stream)
{
    if (host_in == nullptr || !is_dtype(dtype)) return MOR_ERR_INVALID_ARG;
    const mor_fp4_matrix_t& m = *host_in;
    const mor_status_t s = check_matrix(m);
    if (s != MOR_OK) return s;
    if (ld_out < m.cols) return MOR_ERR_INVALID_ARG;
    const int es = (int)dtype_bytes(dtype);
    if (!is_aligned(out, es)) return MOR_ERR_ALIGNMENT;
    if (m.batch == 0 || m.rows == 0 || m.cols == 0) return MOR_OK;
    if (out == nullptr) return MOR_ERR_INVALID_ARG;
    DequantParams p = {};
    p.codes = m.codes;
    p.scales = m.scales;
    p.t = m.tensor_scale;
    p.rows = m.rows;
    p.cols = m.cols;
    p.ld = m.ld;
    p.ldo = ld_out;
    p.row_tiles = (uint32_t)ceil_div(m.rows, 128);
    p.col_tiles = (uint32_t)ceil_div(m.cols, 128);
    p.ktiles = (uint32_t)scale_ktiles(m.cols, m.format);
    p.access = access_bytes(out, ld_out * es, 0, es);
    p.out = out;
    const uint32_t grid = (uint32_t)(m.batch * p.row_tiles * p.col_tiles);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const bool nv = m.format == MOR_FP4_E4M3_16;
    auto run = [&](auto kernel, int element, std::atomic<uint64_t>& done) {
        const int smem = p.access < 16 ? 128 * (128 * element + 16) : 0;
        if (smem > 0 && !allow_smem(kernel, smem, done)) return cudaErrorInvalidValue;
        return launch(kernel, grid, kQThreads, smem, st, grid <= kEarlyGrid, p);
    };
    static std::atomic<uint64_t> done[4];
    cudaError_t e;
    if (dtype == MOR_DTYPE_BF16)
        e = nv ? run(fp4_dequant_kernel<__nv_bfloat16, MOR_FP4_E4M3_16>, 2, done[0]) : run(fp4_dequant_kernel<__nv_bfloat16, MOR_FP4_E8M0_32>, 2, done[1]);
    else
        e = nv ? run(fp4_dequant_kernel<float, MOR_FP4_E4M3_16>, 4, done[2]) : run(fp4_dequant_kernel<float, MOR_FP4_E8M0_32>, 4, done[3]);
    return e == cudaSuccess ? MOR_OK : MOR_ERR_CUDA;
}

}  // extern "C"
