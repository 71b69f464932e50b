/*
 * mor.h -- C boundary of the B200 (sm_100a) MoR analyse-and-quantise library.
 *
 * MoR (Mixture of Representations) partitions a BF16 tensor into blocks, walks an ordered
 * list of formats from most to least aggressive for every block and keeps the first one
 * whose acceptance metric holds (Section 3, Algorithm 2 of the paper).  Scales follow the
 * Group Amax Mantissa scheme: one 23-bit mantissa per tensor plus one 8-bit exponent per
 * block (Section 2, Algorithm 1).
 *
 * Conventions for every entry point
 *   - Pointers inside descriptors are DEVICE pointers.  The descriptors themselves, and
 *     every argument named host_*, live in HOST memory and are read before the call returns.
 *   - The caller owns all buffers and the stream.  The library allocates nothing, keeps no
 *     state between calls and never synchronises: work is enqueued on `cuda_stream`
 *     (a cudaStream_t passed as void*, NULL = the default stream) and the call returns.
 *   - Argument problems are reported synchronously and nothing is launched.  Conditions
 *     found on the device (non-finite inputs) are reported in mor_tensor_stats_t.
 *   - Inputs are row-major with the last dimension contiguous; BF16 where nothing else is said.
 */
#ifndef MOR_H_
#define MOR_H_

#include <stddef.h>
#include <stdint.h>

/* The library is built with hidden symbol visibility; only the entry points below are exported. */
#if defined(__GNUC__)
#define MOR_API __attribute__((visibility("default")))
#else
#define MOR_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    MOR_OK = 0,
    MOR_ERR_INVALID_ARG = 1,   /* NULL where a pointer is required, negative size, bad enum   */
    MOR_ERR_UNSUPPORTED = 2,   /* a recipe the paper defines no metric for, or a block shape
                                  this build has no kernel for                                */
    MOR_ERR_ALIGNMENT = 3,     /* base pointer or leading dimension not aligned as stated     */
    MOR_ERR_WORKSPACE = 4,     /* workspace NULL or smaller than mor_workspace_bytes()        */
    MOR_ERR_CUDA = 5,          /* a CUDA runtime call failed (launch, copy)                   */
    MOR_ERR_TIMEOUT = 6,       /* a bounded device-side wait expired (reported in
                                  mor_tensor_stats_t.status; the outputs are then incomplete)  */
    MOR_ERR_STATIC_SCRATCH = 7 /* mor_analyze_quantize_static: the tensor needs more scratch than
                                  the built-in array holds                                    */
} mor_status_t;

/* Representation types.  Section 3 orders the candidates by how much precision they give up,
 * E4M3 first and BF16 last.  E4M3: 4 exponent / 3 mantissa bits, finite range 2^-9..448.
 * E5M2: 5 / 2 bits, 2^-16..57344 (Sections 1-2).  Casts round to nearest even and
 * saturate to the largest finite value. */
typedef enum { MOR_FMT_E4M3 = 0, MOR_FMT_E5M2 = 1, MOR_FMT_BF16 = 2 } mor_format_t;

/* How a block's scale is formed.
 *   GAM        Algorithm 1: mantissa of 448/tensor_amax shared by all blocks, per-block
 *              exponent of 448/block_amax lowered by one when the shared mantissa is the
 *              larger, so that no block saturates.
 *   E8M0       power-of-two scale per block (the ablation of Section 4.1.2): Algorithm 1
 *              with a zero mantissa.
 *   FP32_AMAX  fl32(448/block_amax) per block (same ablation); the full scale is returned
 *              in mor_outputs_t.scale_f32. */
typedef enum { MOR_SCALE_GAM = 0, MOR_SCALE_E8M0 = 1, MOR_SCALE_FP32_AMAX = 2 } mor_scale_mode_t;

/* Acceptance metric for E4M3.
 *   TENSOR_MEAN_REL  Section 3.1, Eq. 1-2: one decision for the whole tensor; mean over its
 *                    non-zero elements of |x - Q(x)| / |x| must be < threshold.  The scales
 *                    may still be per block: the block sums are added up into the tensor's error.
 *   BLOCK_VS_E5M2    Section 3.2, Eq. 3: per block, E4M3 is kept when its summed relative
 *                    error does not exceed that of E5M2.  With three formats a rejected
 *                    block takes E5M2 when Eq. 4 holds (max|b|/min|b| < 57344/2^-14).
 *   BLOCK_MEAN_REL   Eq. 1-2 applied to each block alone (an instance of Algorithm 2 the
 *                    paper does not evaluate). */
typedef enum {
    MOR_CRIT_TENSOR_MEAN_REL = 0,
    MOR_CRIT_BLOCK_VS_E5M2 = 1,
    MOR_CRIT_BLOCK_MEAN_REL = 2
} mor_criterion_t;

enum {
    MOR_FLAG_STRICT_TIES = 1u,             /* Eq. 3 with its literal '<': a block that is
                                              equally good in both formats is rejected.
                                              Default: a tie keeps E4M3.                    */
    MOR_FLAG_RANGE_MIN_INCLUDES_ZERO = 2u  /* Eq. 4 with the literal min|b|: a block that
                                              holds a zero never takes E5M2.  Default: the
                                              minimum runs over non-zero elements.          */
};

/* One tensor and the recipe to analyse it with (inputs of Algorithm 2: tensor, partition,
 * ordered type list, metric; input of Algorithm 1: q_amax is 448, and 57344 for E5M2). */
typedef struct mor_tensor_desc {
    const void* x;          /* DEVICE.  BF16 [rows, ld], 16-byte aligned                     */
    int64_t rows, cols;     /* >= 0; an empty tensor is valid                                */
    int64_t ld;             /* elements between row starts; >= cols; multiple of 8           */
    int32_t block_rows;     /* partition: (0,0) whole tensor, (1,128) sub-channel rows,      */
    int32_t block_cols;     /*            (128,128) or (64,64) 2-D blocks (Section 4.1.2 runs
                                           the smaller size as an ablation); per channel (Section 3;
                                           the paper's most FP8-efficient partition): (1,0) one
                                           block per row, (0,1) one block per column, whichever is
                                           the operand's dot-product dimension, two formats only,
                                           decided for the tensor (Eq. 2) or per channel (Eq. 3, or
                                           Eq. 1-2 on the channel); (128,1) sub-column blocks.  The
                                           column partitions (128,1) and (0,1) serve the operand whose
                                           dot-product dimension runs down the rows: their codes come
                                           out transposed, see codes.  Edge blocks may overhang:
                                           missing elements take part in nothing                  */
    int32_t n_formats;      /* 2 or 3                                                        */
    int32_t formats[3];     /* {E4M3,BF16} or {E4M3,E5M2,BF16}, in this order                */
    int32_t criterion;      /* mor_criterion_t; three formats need BLOCK_VS_E5M2             */
    float   threshold;      /* th of Eq. 2 as a fraction (0.045 = the paper's 4.5 %)         */
    int32_t scale_mode;     /* mor_scale_mode_t                                              */
    uint32_t flags;         /* MOR_FLAG_*                                                    */
    const float* group_amax;/* DEVICE, optional.  g_amax of Algorithm 1 if the caller has it
                               already: it fixes the shared mantissa; block amaxes are still
                               taken from the data, so a stale value cannot cause saturation.
                               NULL = the library computes it with one extra read of the
                               tensor (always done for the (0,0) and (1,0) partitions, whose
                               block amax spans tiles; never needed for the E8M0 and FP32-amax
                               scale modes of the other partitions, which have no shared
                               mantissa: those read the tensor once)                         */
} mor_tensor_desc_t;

#define MOR_ERROR_BINS 12

/* Per-block quantities behind the decisions (Eq. 3 sums, Eq. 4 range). */
typedef struct mor_block_stats {
    float    amax;          /* max|x| over the block's finite elements                       */
    float    min_abs_nz;    /* min|x| over finite non-zero elements, +inf if none; filled
                               only for three-format recipes                                 */
    uint32_t nnz;           /* finite non-zero elements (n of Eq. 1 restricted to the block) */
    uint32_t n_nonfinite;   /* NaN or +-inf elements                                         */
    float    sum_rel_e4m3;  /* sum over non-zeros of |x - Q_E4M3(x)| / |x|                   */
    float    sum_rel_e5m2;  /* same for E5M2; filled when the criterion is BLOCK_VS_E5M2     */
} mor_block_stats_t;

/* Per-tensor summary; always written. */
typedef struct mor_tensor_stats {
    double   sum_rel_e4m3;  /* numerator of Eq. 2                                            */
    uint64_t nnz;           /* n of Eq. 1                                                    */
    double   mean_rel_e4m3; /* error of Eq. 2; 0 when n = 0                                  */
    float    group_amax;    /* g_amax of Algorithm 1 (finite elements only)                  */
    uint32_t group_mantissa;/* m_g of Algorithm 1: low 23 bits                               */
    uint32_t tensor_format; /* Eq. 2 decision with `threshold`: MOR_FMT_E4M3 or MOR_FMT_BF16;
                               filled whatever the criterion                                 */
    uint32_t status;        /* mor_status_t of device-side conditions, MOR_OK normally       */
    uint64_t n_blocks, n_e4m3, n_e5m2, n_bf16;   /* blocks by selected format                */
    uint64_t n_nonfinite;   /* NaN / inf elements: ignored by every amax, count and sum;
                               they force their block, and tensor_format, to BF16            */
} mor_tensor_stats_t;

/* Outputs of Algorithm 2 (X_Q and the block metadata D) and of Algorithm 1 (S; M is in
 * mor_tensor_stats_t.group_mantissa).  All DEVICE pointers.  Block arrays are row-major
 * over the block grid [ceil(rows/block_rows), ceil(cols/block_cols)]. */
typedef struct mor_outputs {
    uint8_t* codes;         /* [rows, codes_ld] FP8 codes, 16-byte aligned ((128,1) and (0,1) blocks:
                               transposed, [cols, codes_ld] with codes_ld >= roundup(rows,16),
                               so that every block is contiguous).  E4M3 codes
                               everywhere except in blocks that selected E5M2; blocks that
                               selected BF16 still hold their E4M3 codes.  The tile store works
                               on 16-byte pieces of a row: the bytes of a row from column cols
                               up to the next multiple of 16 are overwritten (with the code of
                               zero); bytes from there to codes_ld-1 are left untouched       */
    int64_t  codes_ld;      /* bytes between row starts; >= roundup(cols,16); multiple of 16 */
    uint8_t* scale_e8m0;    /* [n_blocks] biased binary32 exponent of the selected format's
                               scale.  The scale is bits((e << 23) | group_mantissa); the
                               consumer de-scales by dividing by it                          */
    uint8_t* sel;           /* [n_blocks] mor_format_t chosen for the block                  */
    float*   scale_f32;     /* [n_blocks] optional (required for MOR_SCALE_FP32_AMAX): the
                               selected format's scale as a binary32                         */
    void*    bf16_fallback; /* optional, BF16 [rows, ld] like x: receives a copy of every
                               block that selected BF16 (other blocks are left untouched).
                               NULL = the fallback is the input itself.  Per-block criteria
                               only                                                          */
    mor_block_stats_t*  block_stats;  /* [n_blocks] optional                                 */
    mor_tensor_stats_t* tensor_stats; /* required                                            */
    void*    fake_quant;    /* optional, BF16 [rows, ld] like x: the tensor after "quantise,
                               dequantise, de-scale" (Section 4, the form the paper trains with).
                               Per element: the FP8 value of the block's selected format divided
                               by the block's scale (one binary32 division), rounded to BF16;
                               blocks that stay in BF16 and NaN/inf elements are copied.  Where the
                               decision is taken for the whole tensor (tensor-level criterion,
                               (0,0) partition) the E4M3 values are written: keep the input
                               instead when tensor_format says BF16.  Per-channel partitions take
                               this output and bf16_fallback with the tensor-level criterion only
                               (a per-channel decision is known after the codes are written)      */
    uint32_t* error_histogram; /* optional, DEVICE, [MOR_ERROR_BINS] counters of the relative-error
                               histogram of Section 4.1.3: the call adds one to the bin that holds the
                               tensor's error of Eq. 1 (tensor_stats.mean_rel_e4m3).  Bin k covers
                               [0.5 k %, 0.5 (k+1) %), the last bin everything from 5.5 % up.  The
                               caller zeroes the counters when a period starts and may hand the same
                               array to many calls (one row of the paper's heat map per tensor)      */
} mor_outputs_t;

/* Bytes of DEVICE scratch the calls below need for these `n` descriptors (one partial result per
 * 128 x 128 tile, block keys handed from the amax pre-pass to the main kernel, one amax slot per
 * tensor, one status word).  Only shapes and block shapes are read.  Returns 0 on
 * a NULL or negative argument.  The scratch needs no initialisation and 256-byte alignment. */
MOR_API size_t mor_workspace_bytes(const mor_tensor_desc_t* host_descs, int n);

/* Section 3, Algorithm 2 on one tensor: block amax, GAM scale, cast to E4M3 (and E5M2),
 * relative-error sums, per-block or per-tensor decision; writes codes, scales, selection,
 * optional BF16 copies and statistics.  Launches: tensor amax (unless supplied), the fused
 * main kernel, a small finalise kernel. */
MOR_API mor_status_t mor_analyze_quantize(const mor_tensor_desc_t* host_desc, const mor_outputs_t* host_out,
                                  void* workspace, size_t workspace_bytes, void* cuda_stream);

/* The same analysis for `n` tensors with one set of launches per block shape.
 * Section 3 applies the method to a tensor and to its transpose (the operand layouts of the forward
 * and the backward GEMM).  Two neighbouring entries that name the same tensor (same x, shape, ld,
 * recipe, group_amax) with block shape (1,128) first and (128,1) second, codes wanted, no BF16 copy or
 * fake-quantised output on the first, are served by one main kernel that reads every tile of the tensor
 * once and converts it along the rows and along the columns; every output equals that of two separate
 * calls. */
MOR_API mor_status_t mor_analyze_quantize_batched(const mor_tensor_desc_t* host_descs, const mor_outputs_t* host_outs,
                                          int n, void* workspace, size_t workspace_bytes, void* cuda_stream);

/* Optional CUDA events (cudaEvent_t passed as void*, created and owned by the caller, NULL to
 * skip) recorded on `cuda_stream` around the three stages, so that a caller can time each
 * stage of a call separately.  Order on the stream: amax_begin, [tensor-amax kernels],
 * main_begin, [all main kernels], main_end, [all finalise kernels], finalise_end. */
typedef struct mor_stage_events {
    void* amax_begin;
    void* main_begin;
    void* main_end;
    void* finalise_end;
} mor_stage_events_t;

/* mor_analyze_quantize_batched plus stage events (host_events may be NULL). */
MOR_API mor_status_t mor_analyze_quantize_batched_ex(const mor_tensor_desc_t* host_descs, const mor_outputs_t* host_outs,
                                             int n, void* workspace, size_t workspace_bytes, void* cuda_stream,
                                             const mor_stage_events_t* host_events);

/* Decisions and statistics only (Eq. 1-4 evaluated, nothing quantised out): reads the
 * tensor, writes `tensor_stats` and, when non-NULL, `block_stats`, `sel`, `scale_e8m0`.
 * Serves threshold calibration and the per-tensor error statistics of Section 4.1.3. */
MOR_API mor_status_t mor_select_stats(const mor_tensor_desc_t* host_desc, mor_block_stats_t* block_stats,
                              mor_tensor_stats_t* tensor_stats, uint8_t* sel, uint8_t* scale_e8m0,
                              void* workspace, size_t workspace_bytes, void* cuda_stream);

/* mor_select_stats for `n` tensors in one call (tensors sharing a partition and recipe share kernel launches,
 * 16 per launch).  host_outs[i].codes, .codes_ld, .bf16_fallback and .fake_quant are ignored; tensor_stats is
 * required, block_stats / sel / scale_e8m0 / scale_f32 / error_histogram are optional as in mor_analyze_quantize.
 * Same workspace as mor_analyze_quantize_batched for the same descriptors. */
MOR_API mor_status_t mor_select_stats_batched(const mor_tensor_desc_t* host_descs, const mor_outputs_t* host_outs, int n,
                                              void* workspace, size_t workspace_bytes, void* cuda_stream);

/* The first step of Algorithm 1 alone (the group's largest magnitude), with the whole tensor as the group:
 * writes max|x| over finite elements of tensor i to amax_out[i] (DEVICE, n floats), so
 * that later calls can pass it as group_amax. */
MOR_API mor_status_t mor_group_amax(const mor_tensor_desc_t* host_descs, int n, float* amax_out,
                            void* workspace, size_t workspace_bytes, void* cuda_stream);

/* End-to-end variant for data that lives in HOST memory: copies the tensor to the device,
 * runs mor_analyze_quantize and copies codes, scales, selection and statistics back, all
 * on `cuda_stream`; returns after enqueueing (synchronise the stream before reading).
 * In `host_desc` and `host_out` every data pointer is a HOST pointer here (pinned memory
 * makes the copies asynchronous); host_desc->group_amax must be NULL.  `device_staging`
 * is DEVICE scratch of at least mor_host_staging_bytes() bytes. */
MOR_API size_t mor_host_staging_bytes(const mor_tensor_desc_t* host_desc);
MOR_API mor_status_t mor_analyze_quantize_host(const mor_tensor_desc_t* host_desc, const mor_outputs_t* host_out,
                                       void* device_staging, size_t staging_bytes, void* cuda_stream);

/* No counterpart in the paper: a packaging variant of mor_analyze_quantize for callers that cannot
 * allocate device memory where they run (a plug-in inside a runtime that owns all device memory, a
 * latency-critical loop that must avoid the synchronisation an allocation implies, a process with a
 * memory budget fixed at start-up).  Inputs and outputs are the caller's as before; the scratch
 * comes from an array of MOR_STATIC_SCRATCH_BYTES that is part of the library image, so every GPU
 * that loads the library holds that much memory until the process exits.  The call makes no
 * cudaMalloc / cudaFree and uses no allocating library routine.
 *   - Limit: mor_workspace_bytes(host_desc, 1) must not exceed MOR_STATIC_SCRATCH_BYTES (2 MiB).
 *     The scratch holds 56 bytes per 128 x 128 tile, and 552 with the (1,128) partition (one key
 *     per block), so the limit is roughly 600 M elements, or 62 M elements for (1,128); larger
 *     tensors are refused with MOR_ERR_STATIC_SCRATCH and nothing is launched.
 *   - The first call on each device looks up the array's device address (with that device
 *     current) and keeps it for the life of the process; make that first call outside any stream
 *     capture.  The address belongs to the device that is current at the call, which must be the
 *     device of `cuda_stream`.  After a cudaDeviceReset() the remembered address is stale: a process
 *     that resets a device must not use this entry point on it afterwards.
 *   - All calls share the one array, and it keeps what the previous call left in it; the call
 *     clears the part that has to start at zero.  Two calls whose kernels overlap on the GPU
 *     (different streams, no ordering between them) race on it: order them.  */
#define MOR_STATIC_SCRATCH_BYTES (2 * 1024 * 1024)
MOR_API mor_status_t mor_analyze_quantize_static(const mor_tensor_desc_t* host_desc, const mor_outputs_t* host_out,
                                         void* cuda_stream);

/* ------------------------------------------------------------------ 4-bit operands and their products ----
 * The next step down from the 8-bit codes above: microscaled 4-bit floating point (the block formats that the
 * introduction's prior recipes use), made along the reduction axis of the product an operand enters.
 * Codes are E2M1 (+-0, .5, 1, 1.5, 2, 3, 4, 6; round to nearest even, saturating), two to a byte with the even
 * element in the low half.
 *   E8M0_32  blocks of 32; a = max|x| of the block; e = floor(log2 a) - 2 held to -127..127; scale byte e + 127
 *            (0 for a block of zeros); code = E2M1(x * 2^-e).  tensor_scale is 1.
 *   E4M3_16  blocks of 16; A = max|x| of the tensor, at least 2^-88; t = fl32(A * fl32(1 / 2688)) is the tensor scale;
 *            s = E4M3(fl32(448 a / A)), saturating, is the block scale; code = E2M1(fl32(x * fl32(1 / fl32(s t)))), zero
 *            where s is zero.  A value is fl32(fl32(code * s) * t).
 * NaN and infinities take part in no maximum; the scale byte of their block is NaN (0xFF, 0x7F) and its codes are
 * zero, so that everything the block enters is NaN. */
typedef enum { MOR_FP4_E4M3_16 = 0, MOR_FP4_E8M0_32 = 1 } mor_fp4_format_t;
typedef enum { MOR_DTYPE_BF16 = 0, MOR_DTYPE_F32 = 1 } mor_dtype_t;

/* A stack of `batch` matrices [rows, cols] in 4 bits, blocks along cols (the reduction axis).  codes: row i of matrix b
 * starts at byte (b * rows + i) * ld.  scales: tiles of 128 rows x 4 blocks, 512 bytes each, ordered
 * [batch][ceil(rows / 128)][ceil(blocks / 4)] with blocks = ceil(cols / block length); inside a tile the byte of a row
 * and a block is at (row % 32) * 16 + (row / 32 % 4) * 4 + block % 4, the order in which the tensor cores take
 * them.  Codes past cols up to the next multiple of 32 and every byte of the tiles are written (zeros where there is no
 * element). */
typedef struct mor_fp4_matrix {
    uint8_t* codes;         /* DEVICE, 16-byte aligned                                        */
    uint8_t* scales;        /* DEVICE, 16-byte aligned                                        */
    float*   tensor_scale;  /* DEVICE, one float for the whole stack                          */
    int64_t  batch, rows, cols;
    int64_t  ld;            /* bytes between rows; >= ceil(cols / 32) * 16; multiple of 16    */
    int32_t  format;        /* mor_fp4_format_t                                               */
} mor_fp4_matrix_t;

/* Bytes of the two arrays of such a stack (ld the smallest allowed); 0 on a bad argument. */
MOR_API size_t mor_fp4_scale_bytes(int64_t batch, int64_t rows, int64_t cols, int format);

/* What is quantised: a stack of matrices [batch][rows, cols], or rows of one matrix gathered on the way. */
typedef struct mor_fp4_quantize_desc {
    const void* x;          /* DEVICE, row-major, aligned to its element; full speed where x, ld and batch_stride
                               are multiples of 32 bytes                                      */
    int32_t dtype;          /* mor_dtype_t                                                    */
    int32_t format;         /* mor_fp4_format_t                                               */
    int64_t batch, rows, cols, ld, batch_stride;   /* in elements; ld >= cols                 */
    const float* amax;      /* DEVICE, optional (E4M3_16): A if the caller has it (larger values saturate).  NULL = the
                               library takes it from the data with one extra read             */
    const int32_t* slot_of_row;  /* DEVICE, optional: out row i is weight[slot] * x[slot / top], slot = slot_of_row[i],
                               zero where the slot is negative (batch must be 1)              */
    const int32_t* row_of_slot;  /* DEVICE [rows * top], with slot_of_row: negative = the slot has no row           */
    int64_t out_rows;       /* with slot_of_row: its length                                   */
    int32_t top;            /* with slot_of_row: slots per row of x                           */
    int32_t weight_dtype;   /* mor_dtype_t of weight                                          */
    const void* weight;     /* DEVICE [rows * top], optional                                  */
} mor_fp4_quantize_desc_t;

/* Quantises along cols (host_rows: [batch][out rows, cols]), along rows (host_cols: the transposes [batch][cols, out rows],
 * blocks along the rows of x), or both from one read; either may be NULL.  The caller fills every field of the
 * outputs; format and shape must match.  Both get the same tensor scale.
 * `workspace`: at least MOR_FP4_WORKSPACE_BYTES of DEVICE scratch, 16-byte aligned, no initialisation needed; may be NULL
 * where amax is given or the format is E8M0_32. */
#define MOR_FP4_WORKSPACE_BYTES 4096
MOR_API mor_status_t mor_fp4_quantize(const mor_fp4_quantize_desc_t* host_desc, const mor_fp4_matrix_t* host_rows,
                                      const mor_fp4_matrix_t* host_cols, void* workspace, size_t workspace_bytes, void* cuda_stream);

/* The values of a stack, [batch][rows, ld_out] in `dtype` (mor_dtype_t), rounded once. */
MOR_API mor_status_t mor_fp4_dequantize(const mor_fp4_matrix_t* host_in, void* out, int dtype, int64_t ld_out, void* cuda_stream);

/* How a product is cut into groups (experts).
 *   NONE    out[m, n] = sum_k a[m, k] b[n, k]
 *   ROWS    rows starts[g] .. starts[g+1] of a meet matrix g of b; rows of out past starts[groups] are left untouched
 *   REDUCE  group g sums over k in starts[g] .. starts[g+1]: out[g, m, n]; an empty group is zero            */
typedef enum { MOR_GROUP_NONE = 0, MOR_GROUP_ROWS = 1, MOR_GROUP_REDUCE = 2 } mor_grouping_t;
#define MOR_MAX_GROUPS 1024

/* Product of 4-bit operands of one format on the tensor cores, accumulated in binary32, times both tensor scales. */
typedef struct mor_fp4_matmul_desc {
    mor_fp4_matrix_t a;     /* [1][M, K]                                                      */
    mor_fp4_matrix_t b;     /* [1][N, K]; ROWS: [groups][N, K]                                */
    void*   out;            /* DEVICE [M, ldo]; REDUCE: [groups][M, ldo]; 16-byte aligned     */
    int32_t out_dtype;      /* mor_dtype_t                                                    */
    int32_t grouping;       /* mor_grouping_t                                                 */
    int64_t ldo;            /* elements between rows of out; >= N; a multiple of 16 bytes     */
    const int32_t* starts;  /* DEVICE [groups + 1], multiples of 128 from 0 up, at most M (ROWS) or K (REDUCE)   */
    int32_t groups;
    const int32_t* slot_of_row;  /* DEVICE, optional (ROWS), [M]: rows with a negative slot (which follow the others in their
                               group) are neither needed of a nor written                     */
    uint32_t* status;       /* DEVICE, optional: set to MOR_ERR_TIMEOUT when a bounded wait ran out (never cleared)   */
} mor_fp4_matmul_desc_t;
MOR_API mor_status_t mor_fp4_matmul(const mor_fp4_matmul_desc_t* host_desc, void* cuda_stream);

/* ------------------------------------------------------------------------- tokens sorted by expert ----
 * A token has `top` slots, slot = token * top + j, each with an expert id and a weight.  Sorting gives every slot with an
 * id of 0 .. experts-1 a row: an expert's rows are consecutive, in slot order, and start at a multiple of `align`.  Slots
 * with any other id (masked tokens, dropped slots) have no row. */

/* Rows that n_slots slots can take at most: each of up to min(n_slots, experts) experts may leave align-1 rows empty. */
MOR_API int64_t mor_expert_rows(int64_t n_slots, int experts, int align);
MOR_API size_t mor_expert_workspace_bytes(int64_t n_slots, int experts);

/* ids [n_slots] -> starts [experts + 1], row_of_slot [n_slots] (-1: none), slot_of_row [mor_expert_rows()] (-1: empty).
 * All DEVICE int32.  experts <= MOR_MAX_GROUPS, n_slots < 2^30. */
MOR_API mor_status_t mor_expert_sort(const int32_t* ids, int64_t n_slots, int experts, int align, int32_t* starts,
                                     int32_t* row_of_slot, int32_t* slot_of_row, void* workspace, size_t workspace_bytes,
                                     void* cuda_stream);

/* Rows of a token matrix and of the matrix sorted by expert, and what connects them. */
typedef struct mor_expert_desc {
    int64_t tokens, rows, hidden;  /* rows = mor_expert_rows()                                */
    int32_t top;
    int32_t dtype;                 /* mor_dtype_t of every matrix but ys                      */
    const int32_t* row_of_slot;    /* DEVICE [tokens * top]                                   */
    const int32_t* slot_of_row;    /* DEVICE [rows]                                           */
    const void* weight;            /* DEVICE [tokens * top], optional (NULL = 1)              */
    int32_t weight_dtype;          /* mor_dtype_t                                             */
    int32_t ys_dtype;              /* mor_dtype_t of ys: dtype, or FP32 beside BF16           */
} mor_expert_desc_t;

/* out[row] = weight[slot] * x[token] for every row with a slot, zero for the others (products in binary32, one rounding). */
MOR_API mor_status_t mor_expert_gather(const mor_expert_desc_t* host_desc, const void* x, int64_t ldx, void* out, int64_t ldo,
                                       void* cuda_stream);
/* out[token] = sum over its slots, in order, of weight[slot] * ys[row] (binary32 sums, one rounding); the gradient of a gather
 * without weights. */
MOR_API mor_status_t mor_expert_combine(const mor_expert_desc_t* host_desc, const void* ys, int64_t ldy, void* out, int64_t ldo,
                                        void* cuda_stream);
/* The gradient of combine: dys[row] = weight[slot] * dy[token] (zero for rows without a slot; dys may be NULL) and
 * dweight[slot] = <dy[token], ys[row]> in weight_dtype (0 for slots without a row; may be NULL, ys is then not read). */
MOR_API mor_status_t mor_expert_combine_grad(const mor_expert_desc_t* host_desc, const void* dy, int64_t lddy, const void* ys,
                                             int64_t ldy, void* dys, int64_t lddys, void* dweight, void* cuda_stream);

/* --------------------------------------------------------------------- norm before a projection ----
 * Root-mean-square norm of the rows of a matrix, with the residual's addition before it:
 *   h = x + residual, rounded once to the residual's type (h = x where there is none)
 *   y = (h * rs) * weight with rs = 1 / sqrt(mean(h^2) + eps) in binary32, rounded once to x's type or to 8 bits.
 * 8 bits: E4M3 codes of y * s and a scale s for every 128 columns of a row, or for a row: fl32(448 / a) with a the largest finite |y|
 * (at most the largest binary32; 1 where a is 0), or that cut to a power of two and kept as its biased exponent.  These are the codes and
 * scales of mor_analyze_quantize with the (1,128) and (1,0) partitions and the FP32-amax and E8M0 scale modes, made from y in binary32.
 * A NaN's code is 0x7F, an infinity's the largest finite value's. */
typedef struct mor_norm_desc {
    int64_t rows, cols;      /* cols < 2^31 - 16384                                            */
    const void* x;           /* DEVICE [rows, ldx], aligned to its element; full speed where rows start on 16 bytes      */
    const void* residual;    /* DEVICE [rows, ldr], optional                                   */
    const void* weight;      /* DEVICE [cols]                                                  */
    int64_t ldx, ldr;        /* in elements; >= cols                                           */
    float   eps;
    int32_t dtype;           /* mor_dtype_t of x and y                                         */
    int32_t residual_dtype;  /* of residual and h; without a residual ignored                  */
    int32_t weight_dtype;
} mor_norm_desc_t;
typedef struct mor_norm_outputs {
    void*    h;              /* [rows, ldh] optional, only with a residual; may be the residual itself                   */
    void*    y;              /* [rows, ldy] optional                                           */
    uint8_t* codes;          /* [rows, ldc] optional                                           */
    uint8_t* scale_e8m0;     /* [rows, blocks] with codes: this one or                         */
    float*   scale_f32;      /* this one                                                       */
    int64_t  ldh, ldy, ldc;
    int32_t  block;          /* columns of a scale: 128, or 0 for a whole row (1 where it has no columns)  */
} mor_norm_outputs_t;
MOR_API mor_status_t mor_rms_norm(const mor_norm_desc_t* host_desc, const mor_norm_outputs_t* host_out, void* cuda_stream);

/* The gradient.  host_desc->x is h (the sum as it was stored, in `residual_dtype` if `has_residual`, else x in `dtype`), ->residual the
 * gradient of h from elsewhere (optional, [rows, ldr], h's type).  dy [rows, lddy] in `dtype`.
 *   dh = rs (g - h rs mean(g h rs)) + residual with g = dy * weight
 * dx [rows, lddx] in `dtype` and dr [rows, lddr] in residual_dtype get dh (each optional, each rounded once); dweight [cols], optional, in
 * weight_dtype gets the sum over the rows of dy h rs, taken in binary32 in an order that depends on the shape alone.
 * `workspace`: mor_rms_norm_grad_workspace_bytes() of DEVICE scratch, 16-byte aligned, no initialisation needed; only for dweight. */
MOR_API size_t mor_rms_norm_grad_workspace_bytes(int64_t rows, int64_t cols);
MOR_API mor_status_t mor_rms_norm_grad(const mor_norm_desc_t* host_desc, int has_residual, const void* dy, int64_t lddy, void* dx, int64_t lddx,
                                       void* dr, int64_t lddr, void* dweight, void* workspace, size_t workspace_bytes, void* cuda_stream);

/* Values of E4M3 codes [rows, ldc] with one scale per `block` columns (0: per row), E8M0 or FP32 (one of the two): code / scale rounded once
 * to `dtype`, [rows, ldo].  cols <= 2^28. */
MOR_API mor_status_t mor_codes_dequantize(const uint8_t* codes, int64_t rows, int64_t cols, int64_t ldc, int block, const uint8_t* scale_e8m0,
                                          const float* scale_f32, void* out, int dtype, int64_t ldo, void* cuda_stream);

/* ----------------------------------------------- low-rank adapters beside a shared projection ----
 * out[t] = base[t] + f scale[g] (x[t] a[g]^T) b[g]^T with g = ids[t], the adapter of token t; a token whose id is no adapter's keeps base[t].  Inner
 * products of `rank` terms are kept in binary32 and enter the second product as two BF16 that add up to 16 bits and more; out is rounded once.  Where what they
 * are multiplied with is infinite (b here, in the gradients a in dx, dy in db and x in da) the result is not finite, but NaN where the second of the two is zero
 * or of the other sign, also where the formula has an infinity; no other result is touched. */
typedef struct mor_adapter_desc {
    int64_t tokens, n_in, n_out; /* widths 1 .. 2^21                                             */
    int32_t adapters, rank;      /* adapters <= MOR_MAX_GROUPS - 1; rank 1 .. MOR_MAX_RANK       */
    const void* a;               /* DEVICE BF16 [adapters][rank][n_in]                           */
    const void* b;               /* DEVICE BF16 [adapters][n_out][rank]                          */
    const int32_t* ids;          /* DEVICE [tokens]; NULL = every token has adapter 0            */
    const float* scale;          /* DEVICE [adapters], optional (1)                              */
    float factor;                /* f                                                            */
    uint32_t* status;            /* DEVICE, optional: set to MOR_ERR_TIMEOUT when a bounded wait ran out (never cleared)   */
} mor_adapter_desc_t;
#define MOR_MAX_RANK 512

/* DEVICE scratch of a call, 256-byte aligned, no initialisation needed; may be 0.  train: the scratch is what mor_adapter_grad reads of the
 * forward call (tokens sorted by adapter, the inner products), to be kept until then. */
MOR_API size_t mor_adapter_workspace_bytes(const mor_adapter_desc_t* host_desc, int train);
/* x BF16 [tokens, ldx]; base and out [tokens, ldb], [tokens, ldo] of `dtype` (mor_dtype_t), out may be base. */
MOR_API mor_status_t mor_adapter_add(const mor_adapter_desc_t* host_desc, const void* x, int64_t ldx, const void* base, int64_t ldb, void* out,
                                     int64_t ldo, int dtype, int train, void* workspace, size_t workspace_bytes, void* cuda_stream);
/* Gradients for dy, BF16 [tokens, lddy], with u[t] = f scale[g] dy[t] b[g]: dx [tokens, lddx] BF16 = base[t] + u[t] a[g] (base optional: the
 * gradient from the shared projection, BF16 [tokens, ldb]), da = sum u[t]^T x[t], db = sum f scale[g] dy[t]^T (x[t] a[g]^T), BF16 in a's and b's shapes;
 * zero for an adapter without tokens.  dx, da, db are optional.  `saved`: the workspace of mor_adapter_add with train. */
MOR_API size_t mor_adapter_grad_workspace_bytes(const mor_adapter_desc_t* host_desc);
MOR_API mor_status_t mor_adapter_grad(const mor_adapter_desc_t* host_desc, const void* x, int64_t ldx, const void* dy, int64_t lddy, const void* base,
                                      int64_t ldb, void* dx, int64_t lddx, void* da, void* db, const void* saved, size_t saved_bytes, void* workspace,
                                      size_t workspace_bytes, void* cuda_stream);

/* ------------------------------------------------------------------------------- an optimizer's step ----
 * AdamW with the decay apart from the gradient, over many tensors with one launch for every 512; what is written shares memory with nothing else of the call.  With g the gradient times grad_scale:
 *   m = beta1 m + (1 - beta1) g       v = beta2 v + (1 - beta2) g^2
 *   p = p (1 - lr weight_decay) - lr / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps)
 * in binary32; a second moment below 2^-126 counts as zero, and eps is 2^-63 at least.  Parameters and gradients are BF16 or FP32.  The moments are FP32, or 8 bits: blocks of 128 consecutive elements share a
 * power of two s, the largest that keeps the block's largest finite magnitude times s within 448 (kept as a biased exponent, at most 253; 127
 * for a block of zeros); the first moment is an E4M3 code of m s, the second of w = sqrt(v) s, so that an element may be 2^17 below its
 * block's largest and still count.  Nearest rounding would stop a moment that moves by a thousandth a step, so codes are rounded up or down by a
 * random number u: with t the magnitude over the distance d of its two neighbours n d and (n + 1) d, m takes the upper where t + u >= n + 1
 * (its mean is kept), w where u (2 n + 1) < (t - n)(t + n) (the mean of its square is kept), and a w above zero is at least the smallest code, since
 * it is divided by.  What is not finite becomes NaN.  BF16 parameters are rounded by 16 random bits added below the kept ones.
 * Random numbers are hashes, in 32 bits (C. Wellons, "Prospecting for hash functions", 2018): mix(z): z ^= z >> 16; z *= 0x7FEB352D; z ^= z >> 15; z *= 0x846CA68B; z ^= z >> 16.  With key =
 * mix(mix(seed + 0x9E3779B9 * step) + tensor's number) and z = mix(mix(high half of the element's number ^ key) + low half), the low 16 bits
 * of z / 65536 are u of m, the high ones u of w, the low ones of mix(z ^ 0x9E3779B9) the parameter's. */
typedef struct mor_adamw_tensor {
    void*       param;       /* DEVICE, contiguous, aligned to its element; full speed on 32 bytes  */
    const void* grad;
    void*       exp_avg;     /* FP32 or codes                                                  */
    void*       exp_avg_sq;
    uint8_t*    scales;      /* codes only: [blocks][2] of exp_avg and exp_avg_sq, 2-byte aligned */
    int64_t     numel;
} mor_adamw_tensor_t;
typedef struct mor_adamw_desc {
    double  lr, beta1, beta2, eps, weight_decay;
    int64_t step;            /* number of this step, from 1                                    */
    const int32_t* device_step;   /* DEVICE, optional: the step's number instead, for a captured call that is replayed   */
    const float*   device_lr;     /* DEVICE, optional: the learning rate instead               */
    const float*   grad_scale;    /* DEVICE, optional: factor of every gradient (clipping, loss scale)                   */
    const float*   found_inf;     /* DEVICE, optional: not zero = the call changes nothing     */
    uint64_t seed;           /* its low 32 bits count                                          */
    int32_t param_dtype, grad_dtype;   /* mor_dtype_t                                          */
    int32_t eight_bits;      /* moments as codes                                               */
    const uint32_t* numbers; /* HOST [n], optional: the tensors' numbers, below 2^31, instead of their places 0 .. n - 1 in the call: tensors of several calls
                              * of a step are rounded by random numbers of their own if they have numbers of their own */
    int32_t device_step_each;     /* not zero: device_step is [n], a step's number for every tensor                     */
} mor_adamw_desc_t;
MOR_API mor_status_t mor_adamw(const mor_adamw_desc_t* host_desc, const mor_adamw_tensor_t* host_tensors, int n, void* cuda_stream);
/* Values of 8-bit moments: m = code / s into exp_avg_out, v = (code / s)^2 into exp_avg_sq_out ([numel] in `dtype`, each optional). */
MOR_API mor_status_t mor_adamw_moments(const uint8_t* exp_avg, const uint8_t* exp_avg_sq, const uint8_t* scales, int64_t numel, void* exp_avg_out,
                                       void* exp_avg_sq_out, int dtype, void* cuda_stream);

MOR_API const char* mor_status_string(mor_status_t status);
MOR_API int mor_version(void);

#ifdef __cplusplus
}
#endif
#endif /* MOR_H_ */
