// Tokens sorted by expert and back: a stable counting sort of the slots, the gather of token rows, the weighted sum that brings
// the experts' rows back, and the gradient of that sum.
//
// The sort moves a few bytes per slot and is bound by launches and dependent steps: one launch up to kOneBlockSlots slots, two
// above.  The row movers are bound by memory and all work in token order: a token's row is read once for all of its slots,
// and the rows on the sorted side are whole contiguous rows in any order, which costs nothing extra.
#include "mor_fp4.cuh"

namespace mor {
namespace {

// ------------------------------------------------------------------------------------------------ sort ----

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int64_t kOneBlockSlots = 1024;      // one CTA sorts these in one round of its threads (6.8 us with its launch); beyond, a launch
                                              // that counts first is cheaper: 2048 slots 9.0 us by one CTA and 7.8 us by two launches, 4096
                                              // slots 11.9 us and 7.8 us
constexpr int kMaxChunks = 148;

struct SortParams {
    const int32_t* ids;
    int64_t n, chunk;          // slots; slots per CTA (a multiple of 1024)
    int64_t capacity;
    int32_t experts, align;
    int32_t *starts, *row_of_slot, *slot_of_row;
    int32_t* hist;             // [chunks][experts], of the chunks' slots per expert
};

// The part of a chunk that a warp walks: whole groups of 32 slots.  Returns how many warps have a part.
__device__ __forceinline__ int warp_part(const SortParams& p, int64_t& first, int64_t& last)
{
    const int64_t begin = (int64_t)blockIdx.x * p.chunk, end = min(begin + p.chunk, p.n);
    const int per = (int)(end - begin + kSortThreads - 1) / kSortThreads * 32;
    first = min(begin + (threadIdx.x >> 5) * per, end);
    last = min(first + per, end);
    return per == 0 ? 0 : ((int)(end - begin) + per - 1) / per;
}

// Slots per (warp, expert) of this CTA's chunk.  Lanes with the same expert are found by a match; one of them adds.  Returns how many
// warps have counts.
__device__ int count_slots(const SortParams& p, int32_t* counts)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int64_t first, last;
    const int warps = warp_part(p, first, last);
    for (int i = threadIdx.x; i < warps * p.experts; i += kSortThreads) counts[i] = 0;
    __syncthreads();
    for (int64_t at = first; at < last; at += 32) {
        const int32_t id = at + lane < last ? p.ids[at + lane] : -1;
        const uint32_t same = __match_any_sync(0xFFFFFFFFu, id);
        if (id >= 0 && id < p.experts && lane == __ffs(same) - 1) counts[warp * p.experts + id] += __popc(same);
        __syncwarp();
    }
    __syncthreads();
    return warps;
}

__global__ void __launch_bounds__(kSortThreads) expert_count_kernel(const __grid_constant__ SortParams p)
{
    extern __shared__ int32_t counts[];
    wait_for_predecessor();
    const int warps = count_slots(p, counts);
    for (int e = threadIdx.x; e < p.experts; e += kSortThreads) {
        int32_t sum = 0;
        for (int w = 0; w < warps; ++w) sum += counts[w * p.experts + e];
        p.hist[(int64_t)blockIdx.x * p.experts + e] = sum;
    }
}

// Inclusive sum over the CTA's threads.
__device__ int32_t block_scan(int32_t v, int32_t* shared)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int32_t u = __shfl_up_sync(0xFFFFFFFFu, v, o);
        if (lane >= o) v += u;
    }
    if (lane == 31) shared[warp] = v;
    __syncthreads();
    if (warp == 0) {
        int32_t s = shared[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t u = __shfl_up_sync(0xFFFFFFFFu, s, o);
            if (lane >= o) s += u;
        }
        shared[lane] = s;
    }
    __syncthreads();
    return v + (warp > 0 ? shared[warp - 1] : 0);
}

// Each CTA finds where every expert starts (from all chunks' counts) and where its own warps' slots of that expert go, and walks its
// slots once more: a slot's row is its expert's next place for the warp plus its rank among the lanes with the same expert.  No atomics,
// so equal experts keep slot order.  32768 slots of 64 experts, both kernels: 9 us, all of it latency.
__global__ void __launch_bounds__(kSortThreads) expert_place_kernel(const __grid_constant__ SortParams p)
{
    extern __shared__ int32_t counts[];                 // [warps][experts], then the next row of each
    __shared__ int32_t scan[32];
    __shared__ int32_t used[MOR_MAX_GROUPS + 1];        // first empty row of each expert; [experts]: first row past the last expert
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (gridDim.x == 1) wait_for_predecessor();             // else the predecessor is the count, and the ids are older
    const int warps = count_slots(p, counts);
    int32_t own = 0, before = 0, total = 0;
    if (tid < p.experts)
        for (int w = 0; w < warps; ++w) own += counts[w * p.experts + tid];
    total = own;
    if (gridDim.x > 1) {
        wait_for_predecessor();
        total = 0;
        if (tid < p.experts) {
            constexpr uint32_t kAhead = 16;                 // counts in flight: one after the other, each would wait for L2
            for (uint32_t c0 = 0; c0 < gridDim.x; c0 += kAhead) {
                int32_t h[kAhead];
#pragma unroll
                for (uint32_t i = 0; i < kAhead; ++i) h[i] = c0 + i < gridDim.x ? __ldcg(p.hist + (int64_t)(c0 + i) * p.experts + tid) : 0;
#pragma unroll
                for (uint32_t i = 0; i < kAhead; ++i) {
                    if (c0 + i < blockIdx.x) before += h[i];
                    total += h[i];
                }
            }
        }
    }
    const int32_t padded = (total + p.align - 1) / p.align * p.align;
    const int32_t end = block_scan(tid < p.experts ? padded : 0, scan), start = end - padded;
    if (tid < p.experts) {
        if (blockIdx.x == 0) {
            p.starts[tid] = start;
            if (tid == p.experts - 1) p.starts[p.experts] = end;
        }
        used[tid] = start + total;
        if (tid == p.experts - 1) used[p.experts] = end;
        int32_t next = start + before;
        for (int w = 0; w < warps; ++w) {
            const int32_t c = counts[w * p.experts + tid];
            counts[w * p.experts + tid] = next;
            next += c;
        }
    }
    __syncthreads();
    int64_t first, last;
    warp_part(p, first, last);
    for (int64_t at = first; at < last; at += 32) {
        const int64_t slot = at + lane;
        const int32_t id = slot < last ? p.ids[slot] : -1;
        const uint32_t same = __match_any_sync(0xFFFFFFFFu, id);
        const bool has = id >= 0 && id < p.experts;
        const int32_t next = has ? counts[warp * p.experts + id] : 0;
        __syncwarp();
        if (has && lane == __ffs(same) - 1) counts[warp * p.experts + id] = next + __popc(same);
        __syncwarp();
        const int32_t row = has ? next + __popc(same & ((1u << lane) - 1u)) : -1;
        if (slot < last) p.row_of_slot[slot] = row;
        if (has) p.slot_of_row[row] = (int32_t)slot;
    }
    // rows without a slot: those that alignment leaves behind each expert, and those past the last one
    if (p.align > 1)
        for (int e = blockIdx.x * kSortWarps + warp; e < p.experts; e += gridDim.x * kSortWarps) {
            const int32_t stop = (used[e] + p.align - 1) / p.align * p.align;
            for (int32_t r = used[e] + lane; r < stop; r += 32) p.slot_of_row[r] = -1;
        }
    for (int64_t r = used[p.experts] + (int64_t)blockIdx.x * kSortThreads + tid; r < p.capacity; r += (int64_t)gridDim.x * kSortThreads)
        p.slot_of_row[r] = -1;
}

// ---------------------------------------------------------------------------------------- row movement ----

struct MoveParams {
    int64_t tokens, rows, hidden;
    int64_t ld_token, ld_row, ld_out;
    uint32_t top;
    int32_t weight_dtype;
    uint32_t clear_blocks;     // gather and gradient: the first CTAs clear the rows without a slot
    const int32_t *row_of_slot, *slot_of_row;
    const void* weight;
    const void *tokens_in, *rows_in;   // token side (x, dy), row side (ys)
    void* out;                         // gather: rows; combine: tokens; gradient: rows (dys, may be NULL)
    void* dweight;
};

// Rows that start anywhere or are no whole number of pieces (ANY): pieces are laid out from the aligned addresses of the row that is
// written, what is read is shifted into place, and some forty elements at the ends go one by one, a thread each.
template <typename T, typename R, int BYTES> struct Inner {
    // kPer: elements that a chunk of either type may reach past a piece's
    static constexpr int kElems = BYTES / (int)sizeof(T), kPer = 16 / (int)(sizeof(T) < sizeof(R) ? sizeof(T) : sizeof(R));
    int64_t first, end;          // where whole pieces begin and end, far enough inside for any source's chunks
    int edges;                   // elements outside
    __device__ __forceinline__ Inner(const T* to, int64_t n)
    {
        static_assert(kElems >= kPer, "a piece is a chunk at least");
        first = kElems + (kElems - phase_of(to)) % kElems;
        end = n - kPer >= first ? first + (n - kPer - first) / kElems * kElems : first;
        if (end == first) first = end = n;
        edges = (int)(n - (end - first));
    }
    __device__ __forceinline__ int64_t edge(int i) const { return i < first ? i : i + (end - first); }
};

// Zeroes the rows without a slot among this CTA's kClearRows.  Masked tokens leave all their empty rows at the end, so a CTA
// takes few of them (256 rows of 8 KiB by one CTA took longer than the rest of the gather), and these CTAs come first.
constexpr int kClearRows = 16;
template <typename T, int BYTES, bool ANY> __device__ void clear_rows(const MoveParams& p, T* out, uint32_t block)
{
    using P = Piece<T, BYTES>;
    const int64_t row = (int64_t)block * kClearRows + (threadIdx.x & 31);
    const bool none = (threadIdx.x & 31) < kClearRows && row < p.rows && p.slot_of_row[row] < 0;
    P zero;
    zero.clear();
    for (uint32_t m = __ballot_sync(0xFFFFFFFFu, none); m != 0; m &= m - 1) {
        T* to = out + ((int64_t)block * kClearRows + __ffs(m) - 1) * p.ld_out;
        if constexpr (ANY) {
            const Inner<T, T, BYTES> in(to, p.hidden);
            for (int64_t c = in.first + (int64_t)threadIdx.x * P::kElems; c < in.end; c += (int64_t)blockDim.x * P::kElems) zero.store(to + c);
            for (int i = threadIdx.x; i < in.edges; i += blockDim.x) Piece<T, (int)sizeof(T)>{}.store(to + in.edge(i));
        } else {
            for (int64_t c = (int64_t)threadIdx.x * P::kElems; c < p.hidden; c += (int64_t)blockDim.x * P::kElems) zero.store(to + c);
        }
    }
}

constexpr int kAtOnce = 4;      // slots whose rows are in flight together

// Rows (-1: none) and weights of kAtOnce slots of a token.
struct Slots {
    int32_t row[kAtOnce];
    float w[kAtOnce];
    __device__ __forceinline__ Slots(const MoveParams& p, int64_t token, uint32_t first)
    {
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) row[j] = first + j < p.top ? p.row_of_slot[token * p.top + first + j] : -1;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) w[j] = row[j] < 0 || p.weight == nullptr ? 1.f : weight_at(p.weight, p.weight_dtype, token * p.top + first + j);
    }
};

// A token's row to the rows of its slots, times their weights.
template <typename T, int BYTES> __device__ __forceinline__ void spread_any(const MoveParams& p, const Slots& s, const T* x, T* out)
{
    using P = Piece<T, BYTES>;
    using One = Piece<T, (int)sizeof(T)>;
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
        if (s.row[j] < 0) continue;
        T* to = out + (int64_t)s.row[j] * p.ld_out;
        const Inner<T, T, BYTES> in(to, p.hidden);
        for (int64_t c = in.first + (int64_t)threadIdx.x * P::kElems; c < in.end; c += (int64_t)blockDim.x * P::kElems) {
            P v;
            load_shifted<T, BYTES>(v.w, x + c);
            if (p.weight == nullptr) v.store(to + c);
            else v.scaled(s.w[j]).store(to + c);
        }
        for (int i = threadIdx.x; i < in.edges; i += blockDim.x) {
            One v;
            v.load(x + in.edge(i));
            if (p.weight == nullptr) v.store(to + in.edge(i));
            else v.scaled(s.w[j]).store(to + in.edge(i));
        }
    }
}

// A token is read once and written to each of its rows.  Bound by memory, mostly by what it writes: 8192 tokens of 4096 BF16, top 4 of 64,
// 54 us (336 MB, 6.2 TB/s); 4095 wide 61 us (one element at a time: 123 us).
template <typename T, int BYTES, bool ANY> __global__ void __launch_bounds__(256) expert_gather_kernel(const __grid_constant__ MoveParams p)
{
    using P = Piece<T, BYTES>;
    T* out = static_cast<T*>(p.out);
    wait_for_predecessor();
    if (blockIdx.x < p.clear_blocks) {
        clear_rows<T, BYTES, ANY>(p, out, blockIdx.x);
        return;
    }
    const int64_t token = blockIdx.x - p.clear_blocks;
    const T* x = static_cast<const T*>(p.tokens_in) + token * p.ld_token;
    for (uint32_t j0 = 0; j0 < p.top; j0 += kAtOnce) {
        const Slots s(p, token, j0);
        if constexpr (ANY) spread_any<T, BYTES>(p, s, x, out);
        for (int64_t c = (int64_t)threadIdx.x * P::kElems; !ANY && c < p.hidden; c += (int64_t)blockDim.x * P::kElems) {
            P v;
            v.load(x + c);
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                if (s.row[j] < 0) continue;
                T* to = out + (int64_t)s.row[j] * p.ld_out + c;
                if (p.weight == nullptr) v.store(to);
                else v.scaled(s.w[j]).store(to);
            }
        }
    }
}

// What is read of a row beside N elements of a token.  FP32 rows beside BF16 tokens come by 16 bytes, which is all that the tokens' access
// promises of their start (8192 tokens, top 4, 4096 wide: sum 93 us, 99 by 32 bytes where the rows start on those; gradient 132 both ways).
template <typename T, typename R, int N> using RowPiece = Piece<R, N * (int)sizeof(R), sizeof(T) == sizeof(R) ? N * (int)sizeof(R) : 16>;

// A token's rows are in flight together and summed in slot order in FP32.  Bound by memory: the same sizes 56 us (336 MB, 6.0 TB/s); 4095
// wide 82 us (one element at a time: 133 us).
template <typename T, typename R, int BYTES, bool ANY> __global__ void __launch_bounds__(256) expert_combine_kernel(const __grid_constant__ MoveParams p)
{
    using P = Piece<T, BYTES>;
    wait_for_predecessor();
    const int64_t token = blockIdx.x;
    const R* ys = static_cast<const R*>(p.rows_in);
    T* out = static_cast<T*>(p.out) + token * p.ld_out;
    auto piece = [&](auto like, int64_t c) {
        using P = decltype(like);
        using Q = RowPiece<T, R, P::kElems>;
        float sum[P::kElems];
#pragma unroll
        for (float& s : sum) s = 0.f;
        for (uint32_t j0 = 0; j0 < p.top; j0 += kAtOnce) {
            const Slots s(p, token, j0);
            Q v[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                v[j].clear();
                if (s.row[j] < 0) continue;
                const R* from = ys + (int64_t)s.row[j] * p.ld_row + c;
                if constexpr (ANY && P::kElems > 1) load_shifted<R, (int)sizeof(v[j].w)>(v[j].w, from);
                else v[j].load(from);
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
                for (int i = 0; i < P::kElems; ++i) sum[i] = fmaf(s.w[j], v[j].get(i), sum[i]);
        }
        P r;
        r.set_all(sum);
        r.store(out + c);
    };
    if constexpr (ANY) {
        const Inner<T, R, BYTES> in(out, p.hidden);
        for (int64_t c = in.first + (int64_t)threadIdx.x * P::kElems; c < in.end; c += (int64_t)blockDim.x * P::kElems) piece(P{}, c);
        for (int i = threadIdx.x; i < in.edges; i += blockDim.x) piece(Piece<T, (int)sizeof(T)>{}, in.edge(i));
    } else {
        for (int64_t c = (int64_t)threadIdx.x * P::kElems; c < p.hidden; c += (int64_t)blockDim.x * P::kElems) piece(P{}, c);
    }
}

// The sums over hidden of <dy, ys> are taken per thread in column order, then over the CTA in a fixed tree: the result
// does not change from run to run.  Bound by memory: the same sizes 93 us (604 MB, 6.5 TB/s); 4095 wide, where dy is read once for the
// sums and once for the rows, 170 us (one element at a time: 237 us).  Four CTAs an SM (64 registers): with the 118 that the compiler would take, two, and not enough
// rows are in flight.
template <typename T, typename R, int BYTES, bool ANY> __global__ void __launch_bounds__(256, 4) expert_grad_kernel(const __grid_constant__ MoveParams p)
{
    using P = Piece<T, BYTES>;
    using Q = RowPiece<T, R, P::kElems>;
    T* out = static_cast<T*>(p.out);
    wait_for_predecessor();
    if (blockIdx.x < p.clear_blocks) {
        clear_rows<T, BYTES, ANY>(p, out, blockIdx.x);
        return;
    }
    __shared__ float part[kAtOnce][8];
    const int64_t token = blockIdx.x - p.clear_blocks;
    const T* dy = static_cast<const T*>(p.tokens_in) + token * p.ld_token;
    const R* ys = static_cast<const R*>(p.rows_in);
    const int warps = blockDim.x >> 5;
    for (uint32_t j0 = 0; j0 < p.top; j0 += kAtOnce) {
        const Slots s(p, token, j0);
        float dot[kAtOnce];
#pragma unroll
        for (float& d : dot) d = 0.f;
        if constexpr (ANY) {
            if (out != nullptr) spread_any<T, BYTES>(p, s, dy, out);
            // a pass of its own, so that the sums' order does not depend on where the written rows start
            auto add = [&](auto like, int64_t c) {
                using P = decltype(like);
                using Q = Piece<R, P::kElems * (int)sizeof(R)>;
                P g;
                Q v[kAtOnce];
                if constexpr (P::kElems > 1) load_shifted<T, (int)sizeof(g.w)>(g.w, dy + c);
                else g.load(dy + c);
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    if (s.row[j] < 0) continue;
                    const R* from = ys + (int64_t)s.row[j] * p.ld_row + c;
                    if constexpr (P::kElems > 1) load_shifted<R, (int)sizeof(v[j].w)>(v[j].w, from);
                    else v[j].load(from);
                }
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
                    if (s.row[j] >= 0)
#pragma unroll
                        for (int i = 0; i < P::kElems; ++i) dot[j] = fmaf(g.get(i), v[j].get(i), dot[j]);
            };
            if (p.dweight != nullptr) {
                const Inner<T, R, BYTES> in(static_cast<const T*>(nullptr), p.hidden);
                for (int64_t c = in.first + (int64_t)threadIdx.x * P::kElems; c < in.end; c += (int64_t)blockDim.x * P::kElems) add(P{}, c);
                for (int i = threadIdx.x; i < in.edges; i += blockDim.x) add(Piece<T, (int)sizeof(T)>{}, in.edge(i));
            }
        }
        for (int64_t c = (int64_t)threadIdx.x * P::kElems; !ANY && c < p.hidden; c += (int64_t)blockDim.x * P::kElems) {
            P g;
            Q v[kAtOnce];
            g.load(dy + c);
            if (p.dweight != nullptr) {
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
                    if (s.row[j] >= 0) v[j].load(ys + (int64_t)s.row[j] * p.ld_row + c);
            }
            if (out != nullptr) {
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
                    if (s.row[j] >= 0) {
                        T* to = out + (int64_t)s.row[j] * p.ld_out + c;
                        if (p.weight == nullptr) g.store(to);
                        else g.scaled(s.w[j]).store(to);
                    }
            }
            if (p.dweight != nullptr) {
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
                    if (s.row[j] >= 0)
#pragma unroll
                        for (int i = 0; i < P::kElems; ++i) dot[j] = fmaf(g.get(i), v[j].get(i), dot[j]);
            }
        }
        if (p.dweight == nullptr) continue;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) dot[j] += __shfl_xor_sync(0xFFFFFFFFu, dot[j], o);
            if ((threadIdx.x & 31) == 0) part[j][threadIdx.x >> 5] = dot[j];
        }
        __syncthreads();
        if (threadIdx.x < kAtOnce && j0 + threadIdx.x < p.top) {
            float sum = part[threadIdx.x][0];
            for (int k = 1; k < warps; ++k) sum += part[threadIdx.x][k];
            const int64_t slot = token * p.top + j0 + threadIdx.x;
            if (p.weight_dtype == MOR_DTYPE_BF16) static_cast<__nv_bfloat16*>(p.dweight)[slot] = __float2bfloat16(sum);
            else static_cast<float*>(p.dweight)[slot] = sum;
        }
        if (j0 + kAtOnce < p.top) __syncthreads();
    }
}

enum Move : int { MOVE_GATHER, MOVE_COMBINE, MOVE_GRAD };

template <typename T, typename R, int BYTES, bool ANY> cudaError_t move_launch(const MoveParams& p, Move what, uint32_t grid, cudaStream_t st)
{
    const int64_t pieces = ceil_div(p.hidden, BYTES / (int64_t)sizeof(T));
    const uint32_t threads = pieces >= 256 ? 256u : (uint32_t)(ceil_div(pieces, 32) * 32);
    if constexpr (sizeof(T) == sizeof(R))
        if (what == MOVE_GATHER) return launch(expert_gather_kernel<T, BYTES, ANY>, grid, threads, 0, st, true, p);
    if (what == MOVE_COMBINE) return launch(expert_combine_kernel<T, R, BYTES, ANY>, grid, threads, 0, st, true, p);
    return launch(expert_grad_kernel<T, R, BYTES, ANY>, grid, threads, 0, st, true, p);
}
template <typename T, typename R> cudaError_t move_access(const MoveParams& p, Move what, uint32_t grid, int access, cudaStream_t st)
{
    // vector pieces must not run past a row: the width has to be a multiple too.  Beside rows of FP32 a token's piece is 16 bytes, so that
    // the registers of four rows' pieces stay the same.
    const int64_t width = p.hidden * (int64_t)sizeof(T);
    if constexpr (sizeof(T) == sizeof(R))
        if (access == 32 && width % 32 == 0) return move_launch<T, R, 32, false>(p, what, grid, st);
    if (access >= 16 && width % 16 == 0) return move_launch<T, R, 16, false>(p, what, grid, st);
    return move_launch<T, R, 16, true>(p, what, grid, st);
}

// Checks what all movers share and fills the parameters.
mor_status_t move_params(const mor_expert_desc_t* d, MoveParams& p)
{
    if (d == nullptr || !is_dtype(d->dtype) || !is_dtype(d->ys_dtype) || d->top < 1) return MOR_ERR_INVALID_ARG;
    if (d->dtype == MOR_DTYPE_F32 && d->ys_dtype != MOR_DTYPE_F32) return MOR_ERR_INVALID_ARG;
    if (d->tokens < 0 || d->rows < 0 || d->hidden < 0 || d->tokens >= (1ll << 30) || d->rows >= (1ll << 31) || d->hidden >= (1ll << 31)) return MOR_ERR_INVALID_ARG;
    if (d->tokens * d->top >= (1ll << 30)) return MOR_ERR_INVALID_ARG;
    if (d->weight != nullptr && !is_dtype(d->weight_dtype)) return MOR_ERR_INVALID_ARG;
    if (d->weight != nullptr && !is_aligned(d->weight, dtype_bytes(d->weight_dtype))) return MOR_ERR_ALIGNMENT;
    if (d->tokens > 0 && d->row_of_slot == nullptr) return MOR_ERR_INVALID_ARG;
    if (d->rows > 0 && d->slot_of_row == nullptr) return MOR_ERR_INVALID_ARG;
    p = MoveParams{};
    p.tokens = d->tokens;
    p.rows = d->rows;
    p.hidden = d->hidden;
    p.top = (uint32_t)d->top;
    p.weight = d->weight;
    p.weight_dtype = d->weight_dtype;
    p.row_of_slot = d->row_of_slot;
    p.slot_of_row = d->slot_of_row;
    return MOR_OK;
}

// A matrix argument: pointer, pitch, alignment; `access` is narrowed to what it allows.
mor_status_t check_rows(const void* m, int64_t rows, int64_t ld, const mor_expert_desc_t& d, int dtype, int& access)
{
    const int es = (int)dtype_bytes(dtype);
    if (ld < d.hidden || (rows > 0 && d.hidden > 0 && m == nullptr)) return MOR_ERR_INVALID_ARG;
    if (!is_aligned(m, es)) return MOR_ERR_ALIGNMENT;
    const int a = access_bytes(m, ld * es, 0, es);
    access = a < access ? a : access;
    return MOR_OK;
}

mor_status_t move_run(const mor_expert_desc_t& d, const MoveParams& p, Move what, uint32_t grid, int access, void* cuda_stream)
{
    if (grid == 0 || p.hidden == 0) return MOR_OK;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const bool mixed = what != MOVE_GATHER && d.dtype == MOR_DTYPE_BF16 && d.ys_dtype == MOR_DTYPE_F32;
    const cudaError_t e = mixed                       ? move_access<__nv_bfloat16, float>(p, what, grid, access, st)
                          : d.dtype == MOR_DTYPE_BF16 ? move_access<__nv_bfloat16, __nv_bfloat16>(p, what, grid, access, st)
                                                      : move_access<float, float>(p, what, grid, access, st);
    return e == cudaSuccess ? MOR_OK : MOR_ERR_CUDA;
}

bool sort_args_ok(int64_t n_slots, int experts, int align)
{
    return n_slots >= 0 && n_slots < (1ll << 30) && experts >= 1 && experts <= MOR_MAX_GROUPS && align >= 1 && align <= 4096 &&
           n_slots + (n_slots < experts ? n_slots : experts) * (int64_t)(align - 1) < (1ll << 31);
}

}  // namespace
}  // namespace mor

using namespace mor;

extern "C" {

int64_t mor_expert_rows(int64_t n_slots, int experts, int align)
{
    if (!sort_args_ok(n_slots, experts, align)) return -1;
    return (n_slots + (n_slots < experts ? n_slots : experts) * (int64_t)(align - 1)) / align * align;
}

size_t mor_expert_workspace_bytes(int64_t n_slots, int experts)
{
    if (!sort_args_ok(n_slots, experts, 1)) return 0;
    return n_slots <= kOneBlockSlots ? 256 : (size_t)kMaxChunks * experts * sizeof(int32_t);
}

mor_status_t mor_expert_sort(const int32_t* ids, int64_t n_slots, int experts, int align, int32_t* starts, int32_t* row_of_slot,
                             int32_t* slot_of_row, void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    if (!sort_args_ok(n_slots, experts, align) || starts == nullptr) return MOR_ERR_INVALID_ARG;
    if (n_slots > 0 && (ids == nullptr || row_of_slot == nullptr || slot_of_row == nullptr)) return MOR_ERR_INVALID_ARG;
    if (!is_aligned(ids, 4) || !is_aligned(starts, 4) || !is_aligned(row_of_slot, 4) || !is_aligned(slot_of_row, 4)) return MOR_ERR_ALIGNMENT;
    SortParams p = {};
    uint32_t chunks = 1;
    p.chunk = kOneBlockSlots;
    if (n_slots > kOneBlockSlots) {
        if (workspace == nullptr || workspace_bytes < mor_expert_workspace_bytes(n_slots, experts)) return MOR_ERR_WORKSPACE;
        if (!is_aligned(workspace, 16)) return MOR_ERR_ALIGNMENT;
        p.chunk = ceil_div(ceil_div(n_slots, kMaxChunks), kSortThreads) * kSortThreads;
        chunks = (uint32_t)ceil_div(n_slots, p.chunk);
    }
    p.ids = ids;
    p.n = n_slots;
    p.capacity = mor_expert_rows(n_slots, experts, align);
    p.experts = experts;
    p.align = align;
    p.starts = starts;
    p.row_of_slot = row_of_slot;
    p.slot_of_row = slot_of_row;
    p.hist = static_cast<int32_t*>(workspace);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const size_t smem = (size_t)kSortWarps * experts * sizeof(int32_t);
    static std::atomic<uint64_t> done_count{0}, done_place{0};
    const int most = kSortWarps * MOR_MAX_GROUPS * (int)sizeof(int32_t);
    if (!allow_smem(expert_place_kernel, most, done_place)) return MOR_ERR_CUDA;
    if (chunks > 1) {
        if (!allow_smem(expert_count_kernel, most, done_count)) return MOR_ERR_CUDA;
        if (launch(expert_count_kernel, chunks, kSortThreads, smem, st, true, p) != cudaSuccess) return MOR_ERR_CUDA;
    }
    return launch(expert_place_kernel, chunks, kSortThreads, smem, st, true, p) == cudaSuccess ? MOR_OK : MOR_ERR_CUDA;
}

mor_status_t mor_expert_gather(const mor_expert_desc_t* host_desc, const void* x, int64_t ldx, void* out, int64_t ldo, void* cuda_stream)
{
    MoveParams p;
    mor_status_t s = move_params(host_desc, p);
    if (s != MOR_OK) return s;
    int access = 32;
    if ((s = check_rows(x, p.tokens, ldx, *host_desc, host_desc->dtype, access)) != MOR_OK) return s;
    if ((s = check_rows(out, p.rows, ldo, *host_desc, host_desc->dtype, access)) != MOR_OK) return s;
    p.tokens_in = x;
    p.ld_token = ldx;
    p.out = out;
    p.ld_out = ldo;
    p.clear_blocks = (uint32_t)ceil_div(p.rows, kClearRows);
    return move_run(*host_desc, p, MOVE_GATHER, p.clear_blocks + (uint32_t)p.tokens, access, cuda_stream);
}

mor_status_t mor_expert_combine(const mor_expert_desc_t* host_desc, const void* ys, int64_t ldy, void* out, int64_t ldo, void* cuda_stream)
{
    MoveParams p;
    mor_status_t s = move_params(host_desc, p);
    if (s != MOR_OK) return s;
    int access = 32;
    if ((s = check_rows(ys, p.rows, ldy, *host_desc, host_desc->ys_dtype, access)) != MOR_OK) return s;
    if ((s = check_rows(out, p.tokens, ldo, *host_desc, host_desc->dtype, access)) != MOR_OK) return s;
    p.rows_in = ys;
    p.ld_row = ldy;
    p.out = out;
    p.ld_out = ldo;
    return move_run(*host_desc, p, MOVE_COMBINE, (uint32_t)p.tokens, access, cuda_stream);
}

mor_status_t mor_expert_combine_grad(const mor_expert_desc_t* host_desc, const void* dy, int64_t lddy, const void* ys, int64_t ldy,
                                     void* dys, int64_t lddys, void* dweight, void* cuda_stream)
{
    MoveParams p;
    mor_status_t s = move_params(host_desc, p);
    if (s != MOR_OK) return s;
    if (p.tokens > 0 && p.hidden > 0 && dys == nullptr && dweight == nullptr) return MOR_ERR_INVALID_ARG;     // empty tensors have no address
    if (dweight != nullptr && !is_dtype(host_desc->weight_dtype)) return MOR_ERR_INVALID_ARG;
    if (dweight != nullptr && !is_aligned(dweight, dtype_bytes(host_desc->weight_dtype))) return MOR_ERR_ALIGNMENT;
    int access = 32;
    if ((s = check_rows(dy, p.tokens, lddy, *host_desc, host_desc->dtype, access)) != MOR_OK) return s;
    if (dweight != nullptr && (s = check_rows(ys, p.rows, ldy, *host_desc, host_desc->ys_dtype, access)) != MOR_OK) return s;
    if (dys != nullptr && (s = check_rows(dys, p.rows, lddys, *host_desc, host_desc->dtype, access)) != MOR_OK) return s;
    p.tokens_in = dy;
    p.ld_token = lddy;
    p.rows_in = ys;
    p.ld_row = ldy;
    p.out = dys;
    p.ld_out = lddys;
    p.dweight = dweight;
    p.clear_blocks = dys != nullptr ? (uint32_t)ceil_div(p.rows, kClearRows) : 0;
    if (p.hidden == 0 && dweight != nullptr && p.tokens > 0) {     // sums over nothing
        const size_t n = (size_t)p.tokens * p.top * dtype_bytes(host_desc->weight_dtype);
        return cudaMemsetAsync(dweight, 0, n, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? MOR_OK : MOR_ERR_CUDA;
    }
    return move_run(*host_desc, p, MOVE_GRAD, p.clear_blocks + (uint32_t)p.tokens, access, cuda_stream);
}

}  // extern "C"
