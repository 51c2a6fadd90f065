/*
 * lorafusion.h - C ABI of the MI355X (gfx950) fused LoRA linear layer.
 *
 * The layer is the LoRA-adapted linear of the LoRAFusion paper, Section 2.1, Eq. 1
 * (notation of its Table 1):
 *
 *     Y = X W + alpha * (dropout(X) A) B,        W frozen,
 *
 * and its backward pass (dX, dA, dB), executed as the paper's five fused operations
 * (Section 5.1, "FusedLoRA Design"): (1) dropout + down-projection, (2) base GEMM + up-projection,
 * (3) dS together with dB, (4) dA, (5) dX = base gradient GEMM + masked LoRA gradient; and the
 * mixed-adapter form of the same operations (Section 5.1, FusedMultiLoRA), where
 * contiguous row segments of a packed token batch belong to different adapters.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - All tensor pointers are DEVICE pointers to row-major, contiguous arrays, 16-byte aligned.
 *   Arrays named "host" below are HOST pointers, read before the call returns.
 * - lora_bf16 is a raw bfloat16 bit pattern.  Products accumulate in fp32; bf16 outputs are
 *   rounded to nearest even.
 * - Storage layouts are the transposes of the paper's math shapes (its Figure 10 holds the
 *   weights transposed for the hardware layout):
 *       X [M,K]   W [N,K]   A [r,K]   B [N,r]   Y,dY [M,N]   dX [M,K]   S_saved [M,r]
 *       dA [r,K] fp32       dB [N,r] fp32       multi: A [G,r,K]  B [G,N,r]  dA [G,r,K]  dB [G,N,r]
 * - `s` is the paper's alpha (already divided by the rank if the caller follows that custom).
 * - Dropout is inverted dropout on the LoRA branch only.  keep(i,j) is a counter-based hash
 *   of (seed, row i local to the adapter's segment, column j); p is quantised to T/65536 with
 *   T = min(65535, floor(p*65536)) and survivors are scaled by q = 65536/(65536-T).  The mask is
 *   never stored: forward and backward regenerate it from (seed, p), so the caller must pass
 *   the same seed and p to both.
 * - S_saved (M*r bf16) receives s*q*(mask.X)A in forward and must be handed back to backward.
 * - Ownership: the caller owns every buffer.  No entry point allocates or frees device
 *   memory, synchronises the device, or touches a stream other than `stream`; work is only
 *   enqueued.  Inputs are never modified.
 * - Supported sizes: M >= 0, K and N positive multiples of 64 and at most 2^22, r in {16, 32, 64},
 *   1 <= G <= 64, M < 2^31.  With M == 0 a forward call enqueues nothing; a backward call still
 *   defines its outputs: dA and dB are zero-filled (left untouched if accumulate != 0).
 * - Errors: every call returns a lora_status and enqueues nothing unless it returns LORA_OK.
 *   With M == 0 the token-sized arrays (X, Y, S_saved, dY, dX) are empty and may be NULL.
 */
#ifndef LORAFUSION_H
#define LORAFUSION_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    LORA_OK = 0,
    LORA_ERR_NULL = 1,        /* a required pointer is NULL */
    LORA_ERR_SHAPE = 2,       /* negative size, or K/N == 0, or M >= 2^31; a stride that does not fit its heads */
    LORA_ERR_ALIGN = 3,       /* a device pointer is not 16-byte aligned */
    LORA_ERR_PARAM = 4,       /* p outside [0,1), or p/s not finite; eps or scale not positive and finite */
    LORA_ERR_SEGMENTS = 5,    /* offsets do not rise from 0 to M */
    LORA_ERR_WORKSPACE = 6,   /* workspace smaller than the call's ..._workspace_bytes(); lora_bwd_noalloc: beyond its scratch */
    LORA_ERR_UNSUPPORTED = 7, /* K or N not a multiple of 64 or above 2^22, r not in {16,32,64}, G > 64; heads and pages: see the call */
    LORA_ERR_HIP = 8          /* a kernel launch failed */
} lora_status;

typedef uint16_t lora_bf16;
typedef void* lora_stream; /* hipStream_t; NULL = the default stream */

/* Forward, one adapter: operations (1) and (2) of Section 5.1 on Eq. 1.
 * Writes Y [M,N] and S_saved [M,r]. */
lora_status lora_fwd(const lora_bf16* X, const lora_bf16* W, const lora_bf16* A, const lora_bf16* B,
                     int64_t M, int64_t K, int64_t N, int32_t r, float s, float p, uint64_t seed,
                     lora_bf16* Y, lora_bf16* S_saved, lora_stream stream);

/* Bytes of scratch the backward entry points need for these sizes (G = number of adapters).
 * Returns 0 for unsupported sizes. */
size_t lora_bwd_workspace_bytes(int64_t M, int64_t K, int64_t N, int32_t r, int32_t G);

/* Backward, one adapter: operations (3), (4), (5) of Section 5.1 (chain rule on Eq. 1):
 *   dS = s dY B^T, dB = s S^T dY, dA = Xhat^T dS, dX = dY W^T + mask*q*(dS A^T).
 * dX may be NULL (skip the input gradient).  accumulate == 0 overwrites dA and dB, != 0 adds to
 * them.  workspace is device scratch of at least lora_bwd_workspace_bytes() bytes, 256-byte
 * aligned; its contents are undefined afterwards. */
lora_status lora_bwd(const lora_bf16* X, const lora_bf16* W, const lora_bf16* A, const lora_bf16* B,
                     const lora_bf16* S_saved, const lora_bf16* dY,
                     int64_t M, int64_t K, int64_t N, int32_t r, float s, float p, uint64_t seed,
                     lora_bf16* dX, float* dA, float* dB, int accumulate,
                     void* workspace, size_t workspace_bytes, lora_stream stream);

/* The same backward for callers that cannot allocate or carry device scratch: code that runs under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  Instead of a workspace argument
 * the kernels use an array of LORA_NOALLOC_SCRATCH_BYTES that is part of the library's device image (each
 * GPU the library runs on holds one from the first call on it until the process ends); the call itself
 * allocates and frees nothing and enqueues no memset.  Arguments, results (bit for bit) and errors are
 * those of lora_bwd, except: a problem whose partial sums do not fit the array - dS (2 M r bytes), its
 * per-column-chunk partials (4 M r ceil(N/512)) and one fp32 plane of dB and of dA per row panel - returns
 * LORA_ERR_WORKSPACE and enqueues nothing (M = 8192, K = N = 4096, r = 16 needs 20.3 MiB).  All calls on
 * one GPU share that GPU's array: two calls that overlap in time on one GPU (different streams, or
 * replays of graphs that hold such a call) race; calls on one stream are ordered and safe. */
#define LORA_NOALLOC_SCRATCH_BYTES (32u << 20)
lora_status lora_bwd_noalloc(const lora_bf16* X, const lora_bf16* W, const lora_bf16* A, const lora_bf16* B,
                             const lora_bf16* S_saved, const lora_bf16* dY,
                             int64_t M, int64_t K, int64_t N, int32_t r, float s, float p, uint64_t seed,
                             lora_bf16* dX, float* dA, float* dB, int accumulate, lora_stream stream);

/* Forward on a packed mixed-adapter batch (Section 5.1, FusedMultiLoRA): rows
 * [seg_offsets[g], seg_offsets[g+1]) use adapter g = (A[g], B[g], s[g], p[g], seeds[g]); the base
 * product X W is shared.  seg_offsets (host, G+1 entries) must rise from 0 to M; empty
 * segments are allowed.  The mask row index restarts at 0 in every segment, so the result equals
 * per-segment lora_fwd calls. */
lora_status multi_lora_fwd(const lora_bf16* X, const lora_bf16* W, const lora_bf16* A, const lora_bf16* B,
                           int64_t M, int64_t K, int64_t N, int32_t r, int32_t G,
                           const int64_t* seg_offsets, const float* s, const float* p,
                           const uint64_t* seeds,
                           lora_bf16* Y, lora_bf16* S_saved, lora_stream stream);

/* Backward on a packed mixed-adapter batch: gradients are routed to the adapter that owns each
 * row segment.  An empty segment's dA[g], dB[g] are zero-filled (left untouched if accumulate). */
lora_status multi_lora_bwd(const lora_bf16* X, const lora_bf16* W, const lora_bf16* A, const lora_bf16* B,
                           const lora_bf16* S_saved, const lora_bf16* dY,
                           int64_t M, int64_t K, int64_t N, int32_t r, int32_t G,
                           const int64_t* seg_offsets, const float* s, const float* p,
                           const uint64_t* seeds,
                           lora_bf16* dX, float* dA, float* dB, int accumulate,
                           void* workspace, size_t workspace_bytes, lora_stream stream);

/* Adapters of different rank in one packed batch (Section 5.1, FusedMultiLoRA: the lookup table holds
 * each adapter's rank, scale and dropout).  ranks (host, G entries; NULL = every adapter has rank r)
 * gives adapter g's rank, 16, 32 or 64 and at most r.  The arrays keep the uniform layout of the
 * calls above with r as the allocated rank: A [G,r,K], B [G,N,r], S_saved [M,r], dA [G,r,K],
 * dB [G,N,r]; adapter g uses rows 0..ranks[g]-1 of A[g] and columns 0..ranks[g]-1 of B[g].  The
 * remaining rows / columns of A and B are ignored whatever they hold; the corresponding entries of
 * S_saved, dA and dB are written as zeros (dA, dB: left untouched under accumulate).  Everything else
 * as in multi_lora_fwd / multi_lora_bwd; the result for segment g equals a lora_fwd / lora_bwd call
 * with r = ranks[g] on the compact arrays.  A rank outside {16,32,64} or above r:
 * LORA_ERR_UNSUPPORTED. */
lora_status multi_lora_fwd_ranked(const lora_bf16* X, const lora_bf16* W, const lora_bf16* A, const lora_bf16* B,
                                  int64_t M, int64_t K, int64_t N, int32_t r, int32_t G,
                                  const int64_t* seg_offsets, const int32_t* ranks, const float* s,
                                  const float* p, const uint64_t* seeds,
                                  lora_bf16* Y, lora_bf16* S_saved, lora_stream stream);
lora_status multi_lora_bwd_ranked(const lora_bf16* X, const lora_bf16* W, const lora_bf16* A, const lora_bf16* B,
                                  const lora_bf16* S_saved, const lora_bf16* dY,
                                  int64_t M, int64_t K, int64_t N, int32_t r, int32_t G,
                                  const int64_t* seg_offsets, const int32_t* ranks, const float* s,
                                  const float* p, const uint64_t* seeds,
                                  lora_bf16* dX, float* dA, float* dB, int accumulate,
                                  void* workspace, size_t workspace_bytes, lora_stream stream);

/* Diagnostic: writes keep(i,j) (1 = kept, 0 = dropped) for rows 0..M-1 and columns 0..K-1 of one
 * adapter into keep [M,K] (device, bytes).  Any M, K >= 0. */
lora_status lora_debug_mask(int64_t M, int64_t K, float p, uint64_t seed, uint8_t* keep,
                            lora_stream stream);

/* Tuning knob and test hook (process-wide, not thread safe).  Several kernels exist in more than
 * one height: the GEMMs of operations (2) and (5) (Section 5.1) with 256 down to 32 token rows per output
 * tile, the down-projection of operation (1) with 32, 16 or 8 token rows per workgroup, operation (3) as one pass with row
 * panels of 1024 down to 64 rows or, in batches of up to 6144 rows, as dS by itself and dB beside (4), and operation
 * (4) with whole segments or row panels of 256 rows (beside dB 512) and more.
 * By default every launch picks the height that fills the chip better (the small ones for short batches and
 * narrow projections; a GEMM may take two launches of different heights).  rows = 256 fixes the large height
 * of the GEMMs and of (1), one pass in (3) and panels of at least 256 rows in (3) and (4) for all later calls, rows = 128
 * GEMM tiles of 128 rows x 256 columns and 16 rows in (1), rows = 0 restores the automatic choice;
 * any other value returns LORA_ERR_PARAM.  Y, S_saved and dX are bit-identical under all three settings; dA
 * and dB are fp32 sums over the row panels and agree up to the order of those sums. */
lora_status lora_set_row_tile(int32_t rows);

/* Tuning knob and test hook (process-wide, not thread safe).  The GEMM kernels of operations (2) and (5)
 * (Section 5.1) with 256-row tiles copy their operand slabs from global memory to LDS either one or two 64-deep slabs
 * ahead of the matrix work.  By default every launch chooses (two ahead when the frozen weight is too large to stay cached -
 * operation (5) - or the contraction is long enough - operation (2)).  slabs = 1 or 2 fixes the distance for all
 * later launches, slabs = 0 restores the automatic choice; any other value returns LORA_ERR_PARAM.  Every output
 * is bit-identical under all three settings. */
lora_status lora_set_slab_lookahead(int32_t slabs);

/* Diagnostic (host only, nothing is enqueued): the row-panel height that operation (3) (Section 5.1) would choose as one pass
 * over dY (the form of larger batches: lora_debug_bwd_plan) for an activation of C columns over these segments under the
 * current lora_set_row_tile setting, the number of panels that gives (each leaves one fp32 plane of partial dB in the
 * workspace), and the number of planes lora_bwd_workspace_bytes provides for.  seg_offsets: host, G+1 entries rising from 0 to M. */
lora_status lora_debug_stream_panels(int64_t M, int64_t C, int32_t G, const int64_t* seg_offsets,
                                     int32_t* panel_rows, int64_t* panels, int64_t* panels_bound);

/* Diagnostic (host only): how operation (4) would cut its rows in a launch of its own, after (3) as one pass over dY, for an
 * input of K columns over these segments.  *panel_rows = 0: one panel per segment, no partial sums; otherwise panels of that
 * height, *panels fp32 partial sums in the workspace.  panels_bound as in lora_debug_stream_panels. */
lora_status lora_debug_da_panels(int64_t M, int64_t K, int32_t G, const int64_t* seg_offsets,
                                 int32_t* panel_rows, int64_t* panels, int64_t* panels_bound);

/* Diagnostic (host only): what a backward call of these sizes would launch under the current lora_set_row_tile setting.
 * scratch: bytes it may lay its partial sums out in, 0 for those of lora_bwd_workspace_bytes (lora_bwd_noalloc has
 * LORA_NOALLOC_SCRATCH_BYTES).  need_dx = 0: no operation (5). */
typedef struct {
    int32_t ds_alone;         /* 1: operation (3) forms dS by itself and dB goes beside (4); 0: one pass over dY */
    int32_t panel_rows_db;    /* row panels of dB and dA; 0: whole segments, no partial sums */
    int32_t panel_rows_da;
    int32_t added_in_strips;  /* 1: the last workgroup of a strip adds its partial sums; 0: a finalize launch does (if there are any) */
    int32_t with_dx;          /* 1: (4), and dB beside it, run in the launch of (5) */
    int64_t bytes;            /* of the scratch that the call writes */
} lora_bwd_plan;
lora_status lora_debug_bwd_plan(int64_t M, int64_t K, int64_t N, int32_t r, int32_t G, const int64_t* seg_offsets,
                                int32_t need_dx, size_t scratch, lora_bwd_plan* plan);

/* Diagnostic (host only): the output tiles that a GEMM over `contraction` elements to `columns` columns (operation (2):
 * K, N; operation (5): N, K) would run with under the current lora_set_row_tile setting; r = 0: no LoRA term.  *parts launches
 * (0 for M = 0, at most 2), launch i with tiles of tile_rows[i] x tile_columns[i] from row first_row[i] on; each array has
 * two entries.  256 and 192 x 256 are the large tiles, everything else the small ones. */
lora_status lora_debug_gemm_tiles(int64_t M, int64_t contraction, int64_t columns, int32_t r, int32_t G,
                                  const int64_t* seg_offsets, int32_t* parts, int32_t* tile_rows, int32_t* tile_columns,
                                  int64_t* first_row);

/* Diagnostic (host only): the kernels that operations (1), (2) and (5) of a forward and a backward call of these sizes would launch
 * under the current settings of the two knobs; the backward with dX and the workspace of lora_bwd_workspace_bytes.
 * fwd, dx: one or two launches each (M = 0: none); what is not launched is all zero. */
typedef struct {
    int32_t rows, columns;    /* output tile of a workgroup; 32 x 32 is half of a 32 x 64 tile of lora_debug_gemm_tiles */
    int32_t depth, stages;    /* contraction elements to a stage in LDS, and the number of stages */
    int32_t waves;            /* of a workgroup's tile, those that only copy among them */
    int32_t asks_ahead;       /* 1: lines are asked for a slab ahead of their copies */
    int64_t workgroups;       /* the strips of (4) and dB among them, where they run in the launch of (5) */
} lora_gemm_launch;
typedef struct {
    int32_t down_rows;        /* operation (1): token rows of a workgroup */
    int32_t down_parts;       /* ... and how many workgroups share the rank's columns */
    int32_t down_ring;        /* ... 1: through a ring of stages in LDS; 0: straight into registers */
    int64_t down_workgroups;
    lora_gemm_launch fwd[2], dx[2];
} lora_launches;
lora_status lora_debug_launches(int64_t M, int64_t K, int64_t N, int32_t r, int32_t G, const int64_t* seg_offsets,
                                lora_launches* out);

/* Diagnostic per-kernel timing for benchmarks.  Between lora_profile_begin() and
 * lora_profile_end() every kernel the entry points above enqueue is bracketed by a pair of HIP
 * events on the caller's stream (the events are created by the library: do not use inside graph
 * capture).  lora_profile_end() waits for the recorded events, adds the elapsed milliseconds and
 * the launch count of each kernel into ms_total / launches (host arrays of LORA_PROF_KERNELS
 * entries, indexed by lora_prof_kernel) and switches timing off.  A GEMM that takes two launches counts as
 * one, from the start of the first to the end of the second.  Not thread safe. */
typedef enum {
    LORA_PROF_DOWN = 0,       /* operation (1): dropout + down-projection            */
    LORA_PROF_FWD_GEMM = 1,   /* operation (2): Y = X W + S' B                        */
    LORA_PROF_DS_DB = 2,      /* operation (3): dS and dB partials, or dS by itself   */
    LORA_PROF_FIN_DS_DB = 3,  /* fixed-order reduction of the dS / dB partials        */
    LORA_PROF_DA = 4,         /* operation (4), unless in the launch of (5); dB too where (3) formed dS by itself */
    LORA_PROF_FIN_DA = 5,     /* fixed-order reduction of the dA partials, if any     */
    LORA_PROF_DX_GEMM = 6,    /* operation (5): dX = dY W^T + mask*q*(dS A^T)         */
    LORA_PROF_KERNELS = 7
} lora_prof_kernel;
lora_status lora_profile_begin(void);
lora_status lora_profile_end(float* ms_total, int32_t* launches);

/* Unfused multi-kernel baseline (one adapter, M > 0): the operator-by-operator sequence of the
 * paper's Section 3.1 / Figure 4 - dropout, X^ A, S B, scaling, X W, add, and the mirrored backward -
 * with every intermediate materialised in `workspace` (device, 256-byte aligned, at least
 * lora_unfused_workspace_bytes()).  It exists so that the fused path's HBM traffic and time can be
 * measured against it.  lora_unfused_bwd consumes the dropped input and S that lora_unfused_fwd left
 * in the same workspace (pass the same s, p, seed); results equal the fused entry points' up to
 * rounding of the extra bf16 intermediates.  dA, dB are overwritten. */
size_t lora_unfused_workspace_bytes(int64_t M, int64_t K, int64_t N, int32_t r);
lora_status lora_unfused_fwd(const lora_bf16* X, const lora_bf16* W, const lora_bf16* A, const lora_bf16* B,
                             int64_t M, int64_t K, int64_t N, int32_t r, float s, float p, uint64_t seed,
                             lora_bf16* Y, void* workspace, size_t workspace_bytes, lora_stream stream);
lora_status lora_unfused_bwd(const lora_bf16* W, const lora_bf16* A, const lora_bf16* B, const lora_bf16* dY,
                             int64_t M, int64_t K, int64_t N, int32_t r, float s, float p, uint64_t seed,
                             lora_bf16* dX, float* dA, float* dB, void* workspace, size_t workspace_bytes,
                             lora_stream stream);

/* The frozen linear layer alone, with the same GEMM kernels (no adapter): Y = X W and dX = dY W^T.
 * The reference line of the paper's Figure 3 (LoRA linear vs frozen linear).  M > 0. */
lora_status lora_frozen_fwd(const lora_bf16* X, const lora_bf16* W, int64_t M, int64_t K, int64_t N, lora_bf16* Y,
                            lora_stream stream);
lora_status lora_frozen_bwd(const lora_bf16* dY, const lora_bf16* W, int64_t M, int64_t K, int64_t N, lora_bf16* dX,
                            lora_stream stream);

/* Measured ceilings (diagnostics for benchmarks): what the GPU sustains in the two regimes that bound the
 * fused operations of Section 5.1, to set beside its published peaks.
 * lora_ceiling_mfma: `workgroups` workgroups of four waves (one per SIMD) each run `iters` rounds of 2^20
 *   floating-point operations per wave: shape 16 = 64 v_mfma_f32_16x16x32_bf16 on 64 independent accumulator
 *   chains - the instruction and register blocking of operations (2) and (5) - shape 32 = 32
 *   v_mfma_f32_32x32x16_bf16 on 16 chains (the other bf16 MFMA shape, for comparison); operands are read once
 *   from `operands` (device, at least 64 KiB of bf16 values of the caller's choice: the sustained rate
 *   depends on the data) and there is no memory traffic in the loop.  sink: device, workgroups * 256 floats,
 *   overwritten.  *flops (host, may be NULL) receives the floating-point operations of the launch; the
 *   caller times it.  Any other shape: LORA_ERR_PARAM.
 * lora_ceiling_hbm_read: `workgroups` workgroups of 256 lanes read `bytes` bytes (a multiple of 16) from
 *   src once, 16 bytes per lane and load, and do nothing else.  sink: device, workgroups * 256 words.
 * Only enqueue on `stream`; allocate nothing.  Bad counts: LORA_ERR_PARAM. */
lora_status lora_ceiling_mfma(const lora_bf16* operands, float* sink, int32_t workgroups, int32_t iters,
                              int32_t shape, double* flops, lora_stream stream);
lora_status lora_ceiling_hbm_read(const void* src, size_t bytes, uint32_t* sink, int32_t workgroups,
                                  lora_stream stream);

/* ---- Serving adapters, and what stands behind the query and key projections ------------------------
 *
 * Once trained, adapters are served: a step holds the rows of many requests, each with its own adapter, then the attention of
 * their new tokens over a cache of keys and values.  The same conventions as above; "device arrays" are read by the kernels, so their
 * values are not checked on the host, and what is out of range in them is handled as each call says.  Strides (ld*) are the
 * distances of rows in elements, multiples of 8, the heads of a row lying side by side.  Sums, norms and the softmax are fp32 and outputs are
 * rounded once; what stands between two products is rounded to bf16 before the second: S of lora_requests_fwd (and _quantised_fwd) and the weights of
 * lora_paged_attn_fwd. */

/* Forward of a batch in which every row names its adapter:
 *   Y[i] = X[i] W^T + s[g] (X[i] A[g]^T) B[g]^T,   g = ids[i];  a row with ids[i] outside 0 .. P-1 has no adapter.
 * X [M,K]  W [N,K]  A [P,r,K]  B [P,N,r]  Y [M,N];  device arrays ids [M], s [P], ranks [P].  ranks (may be NULL: all r): adapter g
 * uses the first ranks[g] rows of A[g] and columns of B[g], any number of 0 .. r (values outside are cut to it); the others may
 * hold anything.  S [M,r]: scratch that receives s (X A^T) in bf16, as the second product takes it, zero past the rank.  No dropout: a
 * row's result is that of lora_fwd with p = 0 up to the order of the sums in S and Y.  M < 2^21, K, N, r as above; any P >= 1; adapters may come in any order and number. */
lora_status lora_requests_fwd(const lora_bf16* X, const lora_bf16* W, const lora_bf16* A, const lora_bf16* B, const int32_t* ids,
                              const int32_t* ranks, const float* s, int64_t M, int64_t K, int64_t N, int32_t r, int64_t P, lora_bf16* Y,
                              lora_bf16* S, lora_stream stream);

/* RMS norm of every query and key head and rotation by the row's position, one pass:
 *   n = x / sqrt(mean(x^2) + eps);  y = R(gamma n)
 * for the H query heads and G key heads (D entries each) of M rows; gamma_q, gamma_k [D].  R turns the pairs (i, i + rot/2), or with
 * interleaved != 0 (2i, 2i+1), of the first rot entries by the angle whose cosine and sine stand in row pos[row] of cos_table,
 * sin_table [positions, rot/2] (fp32); pos [M] is a device array.  A row whose position is outside the tables gets zeros.
 * D: multiples of 16 up to 256; rot: multiples of 16 up to D; H, G up to 1024; M < 2^26; eps > 0.  An output may be its input, with the input's stride. */
lora_status lora_qk_norm_rope_fwd(const lora_bf16* q, const lora_bf16* k, const lora_bf16* gamma_q, const lora_bf16* gamma_k,
                                  const float* cos_table, const float* sin_table, const int32_t* pos, int64_t M, int32_t H, int32_t G, int32_t D,
                                  int32_t rot, int64_t positions, int64_t ldq, int64_t ldk, int64_t ldqo, int64_t ldko, float eps,
                                  int interleaved, lora_bf16* q_out, lora_bf16* k_out, lora_stream stream);

/* Its backward: dq, dk from dq_out, dk_out and the forward's inputs; dgamma_q, dgamma_k [D] fp32, overwritten or, with accumulate != 0,
 * added to (rows whose position is outside the tables add nothing; M = 0 leaves them at zero).  workspace: device scratch of at least
 * lora_qk_norm_rope_workspace_bytes(), 256-byte aligned.  The same inputs give the same bits. */
size_t lora_qk_norm_rope_workspace_bytes(int64_t M, int32_t H, int32_t G, int32_t D);
lora_status lora_qk_norm_rope_bwd(const lora_bf16* q, const lora_bf16* k, const lora_bf16* gamma_q, const lora_bf16* gamma_k,
                                  const float* cos_table, const float* sin_table, const int32_t* pos, const lora_bf16* dq_out,
                                  const lora_bf16* dk_out, int64_t M, int32_t H, int32_t G, int32_t D, int32_t rot, int64_t positions, int64_t ldq,
                                  int64_t ldk, int64_t lddqo, int64_t lddko, int64_t lddq, int64_t lddk, float eps, int interleaved, lora_bf16* dq,
                                  lora_bf16* dk, float* dgamma_q, float* dgamma_k, int accumulate, void* workspace, size_t workspace_bytes,
                                  lora_stream stream);

/* 4 bits, of weights and of the cache: e2m1 codes (bit 3 the sign, the others 0, 0.5, 1, 1.5, 2, 3, 4, 6 in this order), two to a byte, the first in its low
 * half, and for 32 entries in a row the biased exponent of one power of two, a byte; the value is e2m1 * 2^(exp - 127), which bf16 holds exactly.
 * Written, the power of two is the smallest (2^-125 at least, 1 for 32 zeros; exp 2 .. 253) that keeps the largest magnitude within 6; values are rounded to
 * nearest even (from 3.5 * 2^126 on to 2^128, which reads as infinity).  32 entries with one that is not finite are held as NaN, all of them: exp 255.  Exponents below 2 are
 * read where their values are zeros (what is cleared to zeros reads as zeros).
 *
 * Weights W [N,K] into that form, codes [N, K/2] and exps [N, K/32] (device bytes, 16-byte aligned), and back, exactly: what the training entry points take of
 * frozen weights that are held in 4 bits.  K and N: positive multiples of 64 up to 2^22. */
lora_status lora_weights_write(const lora_bf16* W, int64_t N, int64_t K, uint8_t* codes, uint8_t* exps, lora_stream stream);
lora_status lora_weights_read(const uint8_t* codes, const uint8_t* exps, int64_t N, int64_t K, lora_bf16* W, lora_stream stream);

/* lora_requests_fwd over such weights, without a copy of them in bf16: the arguments are its own, with codes and exps for W.  P = 0: no adapters (A, B, ids, ranks, s, S
 * may be NULL, r anything; S is left as it is). */
lora_status lora_requests_quantised_fwd(const lora_bf16* X, const uint8_t* codes, const uint8_t* exps, const lora_bf16* A, const lora_bf16* B,
                                        const int32_t* ids, const int32_t* ranks, const float* s, int64_t M, int64_t K, int64_t N, int32_t r, int64_t P,
                                        lora_bf16* Y, lora_bf16* S, lora_stream stream);
/* Diagnostic (host only): what lora_requests_quantised_fwd runs with for these sizes.  The same call gives the same bits; the same row in another batch need not: the tile goes
 * by M, K and N, S by the other rows' adapters too, and each sums in an order of its own. */
typedef struct {
    int32_t rows, columns;    /* output tile of a workgroup */
    int32_t ring_blocks;      /* blocks of 128 of the contraction that its rings hold at once */
    int32_t own_term;         /* 1: S is formed in the same launch, by every workgroup; 0: in a launch of its own, or there are no adapters */
} lora_quantised_tiles;
lora_status lora_debug_quantised_tiles(int64_t M, int64_t K, int64_t N, int32_t r, int64_t P, lora_quantised_tiles* out);

/* A paged cache of keys and values (the caller's device memory): k, v [pages, heads, page, dim].  fp8 == 0: lora_bf16.  fp8 == LORA_KV_FP4: 4 bits, k, v
 * [pages, heads, page, dim/2] bytes, k_exp, v_exp [pages, heads, page, dim/32], dim a multiple of 32.  Any other fp8 (any other true value): e4m3
 * bytes, and k_exp, v_exp [pages, heads, page] with the biased exponent of one power of two for every token and head; the value is
 * e4m3 * 2^(exp - 127), exp 10 .. 247 (what a write gives), or less beside codes of zero (a cache cleared to zeros).  page: a power of
 * two, 16 .. 1024 tokens; dim: multiples of 16 up to 256; heads up to 1024.  Written and read: M * heads of 2^27 - 8 and fewer. */
#define LORA_KV_FP4 (-4)
typedef struct {
    void* k;
    void* v;
    uint8_t* k_exp;
    uint8_t* v_exp;
    int64_t pages;
    int32_t page, heads, dim, fp8;
} lora_kv_cache;

/* Writes row i of k and v [M, heads, dim] to slot slots[i] = page number * page + place in it (device array; a slot outside the cache
 * is left out).  Slots of one call must differ: what a slot holds after two rows is undefined (keys of one beside values of the other, or
 * its codes under the other's exponent); no other slot is affected.  fp8: the power of two is the smallest (2^-117 at least, 1 for a head
 * of zeros) that keeps the head's largest finite magnitude within 448; values are rounded to nearest even (from 1.9375 * 2^127 on to 2^128,
 * which reads as infinity), what is not finite becomes NaN. */
lora_status lora_kv_cache_write(const lora_kv_cache* cache, const lora_bf16* k, const lora_bf16* v, int64_t ldk, int64_t ldv, const int64_t* slots,
                                int64_t M, lora_stream stream);
/* (4 bits: above.)  ... and reads slots back, exactly; a slot outside the cache reads as zeros. */
lora_status lora_kv_cache_read(const lora_kv_cache* cache, const int64_t* slots, int64_t M, lora_bf16* k, lora_bf16* v, int64_t ldk, int64_t ldv,
                               lora_stream stream);

/* lora_qk_norm_rope_fwd and lora_kv_cache_write in one pass: the normalised and turned queries go to q_out [M,H,dim], the keys and v [M,heads,dim] to their slots.
 * gamma_q and gamma_k NULL (both): no norm, the rotation alone; eps is checked all the same.  Keys that the cache holds in fewer bits are formed in 64 bits and rounded
 * once, to its codes (what is past the range of fp32 counts as not finite); everything else is as in those two calls, a row outside the tables: zeros for query
 * and keys, a slot outside the cache: left out.  q_out may be q, with its stride.  dim, rot, H and M as in the first. */
lora_status lora_kv_cache_append(const lora_kv_cache* cache, const lora_bf16* q, const lora_bf16* k, const lora_bf16* v, const lora_bf16* gamma_q,
                                 const lora_bf16* gamma_k, const float* cos_table, const float* sin_table, const int32_t* pos, const int64_t* slots, int64_t M,
                                 int32_t H, int32_t rot, int64_t positions, int64_t ldq, int64_t ldk, int64_t ldv, int64_t ldqo, float eps, int interleaved,
                                 lora_bf16* q_out, lora_stream stream);

/* Attention of new tokens over a paged cache that holds them already.  q, out [T, H, dim]: the new tokens of B sequences end to end,
 * sequence b's being rows offsets[b] .. offsets[b+1]-1; with kv_lens[b] tokens in the cache, the last of them the new ones; its token j
 * is row j % page of page table[b * ldt + j / page].  The new token at position pos sees the keys j <= pos and, with window > 0, only
 * j > pos - window; query head h uses key/value head h / (H / heads).
 *   out = sum_j softmax_j(scale q k_j) v_j;   a row that sees no key (fewer keys than new tokens): zeros.
 * The weights are rounded to bf16 after their exponential and divided by the sum of the rounded ones, so that equal values come back as they are.
 * offsets [B+1], kv_lens [B] and table are device arrays; max_new and max_kv (host) are the largest number of new tokens and the largest
 * length: rows past max_new of a sequence are not computed, and a larger length than max_kv costs time only.  Lengths are cut to max_pages
 * pages and page numbers to the cache.  Cache entries past a sequence's length, and keys that a row does not see, may hold anything.
 * dim 64 or 128; T * H < 2^31; lengths below 2^30; q k_j and scale q k_j up to 2^126 in magnitude.  workspace: device scratch of at
 * least lora_paged_attn_workspace_bytes(), 256-byte aligned, which is enough for every call with this H, window and form of cache whose T,
 * B, max_new and max_kv are at most these (fewer rows are cut into more parts, so that a smaller step may use more of it; never more than
 * 2^18 rows of dim + 2 floats, where T is within B * max_new).  Chunks beside decoding sequences of long caches are faster as two calls: the
 * longest chunk decides how all sequences of a call are taken.  The same inputs and sizes give the same bits. */
size_t lora_paged_attn_workspace_bytes(const lora_kv_cache* cache, int64_t T, int32_t H, int64_t B, int64_t max_new, int64_t max_kv, int32_t window);
lora_status lora_paged_attn_fwd(const lora_bf16* q, const lora_kv_cache* cache, const int32_t* table, const int32_t* offsets, const int32_t* kv_lens,
                                int64_t T, int32_t H, int64_t B, int64_t max_pages, int64_t ldq, int64_t ldt, int64_t ldo, int64_t max_new,
                                int64_t max_kv, float scale, int32_t window, lora_bf16* out, void* workspace, size_t workspace_bytes,
                                lora_stream stream);

const char* lora_status_string(lora_status st);
int lora_version(void);

#ifdef __cplusplus
}
#endif
#endif /* LORAFUSION_H */
