/*
 * tp_linear.h -- C ABI of libtplinear: one rank's share of a tensor-parallel linear layer on one
 * MI355X (gfx950), forward and backward.
 *
 * What is computed (paper Section 2.2 "Model Parallelism", tensor-parallelism paragraphs; Section
 * 3.1 and Table 1 for the notation): a linear layer  Y = GeLU(X W + 1 b^T)  whose input, weight and
 * output are cut into chunks over a rank grid -- 1D (Megatron feed-forward: first weight cut by
 * columns, second by rows, every rank holding a partial output that an all-reduce would sum), 2D
 * (SUMMA on a q x q square, chunks [P/q, Q/q]), 2.5D (q x q x d cuboid, N = S^2 D) and 3D (p x p x p
 * cube, chunks [P/p^2, Q/p]).  One rank's work is an ordered loop of local block products
 *      C += A_k B_k,   k = 0 .. n_steps-1,
 * followed by bias add and erf-GeLU, and in backward  dX = sum_k dA_k W_k^T,  dW = sum_k X_k^T dA_k.
 * The blocks other ranks would broadcast or gather are already in this GPU's memory: the library
 * performs no communication.
 *
 * Conventions.  Tokens are rows.  All blocks are row-major with a leading dimension `ld` counted in
 * elements.  X:[M,H], W:[H,F] (in x out), b:[F].  bf16 inputs, fp32 accumulation, fp32 or bf16
 * outputs (bf16 by round-to-nearest-even).  Every pointer in this ABI is a DEVICE pointer unless it
 * is explicitly called a host array; host arrays are read during the call and may be freed after it.
 *
 * Ownership / errors.  The caller owns every buffer; the library never allocates, frees or
 * synchronises.  Work is enqueued on the HIP stream passed in (a hipStream_t cast to void*, NULL =
 * the default stream) and the call returns immediately.  Inputs are read-only and may alias each
 * other but not the output of a product that reads them.  A backward call finishes its outputs in the
 * order dA, db, dX, dW as far as that can be seen: dW may be written over what only dX reads, and dW
 * reads what dX left where dX is written over blocks of dW's.  Every failure is a return code found before anything is launched; nothing
 * is written on error.  Row counts may be any value >= 1 (ragged tails are masked); column extents
 * of every block and every `ld` must be multiples of 8 elements and every pointer, the workspace
 * included, 16-byte aligned (128-bit loads and stores), else TP_ERR_ALIGN (TP_ERR_WORKSPACE for the
 * workspace).  The library keeps no mutable state between calls apart from per-device caches of kernel
 * attributes, of the device's compute-unit count and of the address of its built-in scratch array;
 * every entry point may be called from several threads at once (tp_linear_fwd_static: see its own
 * note on calls that overlap on one GPU).
 */
#ifndef TP_LINEAR_H
#define TP_LINEAR_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define TP_MAX_STEPS 16

typedef enum {
    TP_OK = 0,
    TP_ERR_NULL = 1,       /* a required pointer is NULL */
    TP_ERR_MODE = 2,       /* unknown mode / pass / epilogue */
    TP_ERR_GRID = 3,       /* q, d or p < 1, or a rank coordinate outside the grid */
    TP_ERR_SHAPE = 4,      /* M, H, F not divisible as the mode requires; n_steps out of range */
    TP_ERR_ALIGN = 5,      /* pointer not 16-byte aligned, or ld / column extent not a multiple of 8 */
    TP_ERR_DTYPE = 6,      /* output dtype not supported for this output */
    TP_ERR_WORKSPACE = 7,  /* workspace NULL or smaller than tp_linear_workspace_size() says */
    TP_ERR_HIP = 8,        /* a HIP call (launch) reported an error */
    TP_ERR_SCRATCH = 9     /* tp_linear_fwd_static: the product needs more than the built-in scratch */
} tp_status_t;

/* Partition modes.  The 1D scheme is two modes because its two weights are cut differently. */
typedef enum {
    TP_MODE_1D_COL = 10,   /* W cut by columns: rank r owns W[:, r];  Y[:, r] = act(X W[:, r] + b[r])   */
    TP_MODE_1D_ROW = 11,   /* W cut by rows:    rank r owns W[r, :];  partial Y_r = X[:, r] W[r, :]      */
    TP_MODE_2D = 2,        /* q x q,      rank (ri, rj)                                                  */
    TP_MODE_2P5D = 25,     /* q x q x d,  rank (ri, rj, rk = depth layer)                                */
    TP_MODE_3D = 3,        /* p x p x p,  rank (ri, rj, rk)                                              */
    TP_MODE_3D_GATHERED = 33 /* p x p x p with the operands as they are after the all-gathers: one product
                              per pass on slabs [P/p, Q/p], every result a partial (see tp_block_map)   */
} tp_mode_t;

typedef enum { TP_BF16 = 0, TP_F32 = 1 } tp_dtype_t;
typedef enum { TP_EPI_NONE = 0, TP_EPI_BIAS = 1, TP_EPI_BIAS_GELU = 2 } tp_epilogue_t;
typedef enum {
    TP_PASS_FWD = 0, TP_PASS_DX = 1, TP_PASS_DW = 2,
    TP_PASS_DX_PARTIALS = 3, TP_PASS_DW_PARTIALS = 4     /* tp_partials_map / tp_linear_bwd_partials only */
} tp_pass_t;

/* 1D: p = size, ri = rank (q = d = 1).  2D: q, (ri, rj).  2.5D: q, d, (ri, rj, rk).  3D: p, (ri, rj, rk).
 * Unused sizes must be 1 and unused coordinates 0. */
typedef struct { int mode; int q, d, p; int ri, rj, rk; } tp_grid_t;
/* The FULL (unpartitioned) layer: M tokens, H input features, F output features. */
typedef struct { int64_t M, H, F; } tp_dims_t;
/* A read-only device block: bf16, row-major, ld in elements. */
typedef struct { const void* ptr; int64_t ld; } tp_cblk_t;
/* An output device block: row-major, ld in elements, dtype a tp_dtype_t.  ptr == NULL means "not wanted". */
typedef struct { void* ptr; int64_t ld; int dtype; } tp_oblk_t;
/* Launch-plan options of one call (tuning and tests; NULL = all automatic).  The same options must be
 * given to the workspace query and to the call it sizes.
 *   tile   : macro-tile of C.  0 automatic; 1 = 256x256 (four-wave stream kernel); 2 = 128x256,
 *            3 = 256x128, 4 = 128x128 (four-wave kernel with a ring of stages); 5 = 256x256 on the
 *            eight-wave kernel.
 *   split_k: workgroups sharing one C tile along K.  0 automatic, 1..8.
 *   group_m: height, in tile rows, of the groups of the tile order.  0 automatic, 1..64.
 *   rotate : rotate the K-tile order inside a step from C tile to C tile.  0 automatic (on for the
 *            eight-wave kernel, off for the others), 1 on, 2 off.
 *   trim   : when the tiles are a little more than a whole number of rounds of the persistent
 *            workgroups, run the last tile rows as a second, smaller launch.  0 automatic (on), 1 on, 2 off. */
typedef struct { int tile, split_k, group_m, rotate, trim; } tp_plan_opts_t;

/*
 * tp_block_map -- the partition map (host only, no GPU needed).  For rank `grid` of a layer `dims`
 * and a pass, reports how many steps the exact share has, the local product's extents and which
 * chunks take part, as (row chunk, col chunk) indices into the chunk grids below.
 *   chunk grids: X, dX: [rc x kc];  W, dW: [kc x cc];  Y, A, dA: [rc x cc];  b: [cc]
 *     1D_COL: rc=1, kc=1, cc=p      1D_ROW: rc=1, kc=p, cc=1      2D: rc=kc=cc=q
 *     2.5D: rc=q d, kc=cc=q (row chunk of rank (i,j,l) is l q + i; W and b repeat on every layer)
 *     3D:   rc=p^2, kc=cc=p (row chunk of rank (i,j,l) is i p + l)
 *   TP_PASS_FWD: C[m,n] = sum_k X[a_k] W[b_k];          out indexes Y (bias chunk = out_col)
 *   TP_PASS_DX : C[m,n] = sum_k dA[a_k] W[b_k]^T;       out indexes dX
 *   TP_PASS_DW : C[m,n] = sum_k X[a_k]^T dA[b_k];       out indexes dW
 *   3D_GATHERED (Section 2.2: the stored chunk is [P/p^2, Q/p]; gathered along one cube axis it is
 *     the slab [P/p, Q/p]): rc=kc=cc=p, one step per pass, every output a partial:
 *       FWD: X[i,l] W[l,j] -> partial of (X W)[i,j] over l      DX: dA[i,j] W[l,j]^T -> dX[i,l] over j
 *       DW : X[i,l]^T dA[i,j] -> dW[l,j] over i.   Bias and GeLU belong after the summation
 *     (tp_bias_act); row chunk l of the summed slab (i,j) is rank (i,j,l)'s block under TP_MODE_3D.
 * m, n = extents of the output block, k_per_step = contraction length of one step.
 * a_row..b_col are host arrays of TP_MAX_STEPS ints (may be NULL if not wanted); *is_partial = 1
 * when the block is an additive partial that a reduction over other ranks would complete
 * (1D partial sums; 2.5D dW over depth; 3D dW over the first cube axis).
 * Errors: TP_ERR_NULL, TP_ERR_MODE, TP_ERR_GRID, TP_ERR_SHAPE.
 */
int tp_block_map(const tp_grid_t* grid, const tp_dims_t* dims, int pass,
                 int* n_steps, int64_t* m, int64_t* n, int64_t* k_per_step,
                 int* a_row, int* a_col, int* b_row, int* b_col,
                 int* out_row, int* out_col, int* is_partial);

/* Bytes of device workspace tp_linear_fwd (pass TP_PASS_FWD), tp_linear_bwd (TP_PASS_DX and
 * TP_PASS_DW each; pass the larger, the two products run one after the other) or
 * tp_linear_bwd_partials (TP_PASS_DX_PARTIALS, TP_PASS_DW_PARTIALS) may need for this share:
 * cross-workgroup split-K partials in fp32 (never more than 8 x m x n x 4 bytes per product), and, for
 * the two backward passes, the row-slab sums of the bias gradient (at most 64 x n_fwd x 4 bytes; a
 * smaller workspace makes tp_linear_bwd fall back to the single-slab column sum).  0 on invalid
 * arguments. */
size_t tp_linear_workspace_size(const tp_grid_t* grid, const tp_dims_t* dims, int pass);
/* The same for calls made with plan options (NULL = tp_linear_workspace_size). */
size_t tp_linear_workspace_size_ex(const tp_grid_t* grid, const tp_dims_t* dims, int pass, const tp_plan_opts_t* opts);

/*
 * tp_linear_fwd -- forward share:  C = sum_{k<n_steps} X_k W_k  with the fp32 accumulator kept
 * on-chip across all steps;  A = C + b (epi >= TP_EPI_BIAS);  Y = GeLU(A) (TP_EPI_BIAS_GELU), else Y = A.
 *   x_blocks, w_blocks : host arrays [n_steps] of device blocks; X_k is [m, k], W_k is [k, n] with
 *                        m, n, k as tp_block_map reports for TP_PASS_FWD.
 *   n_steps            : 1 .. the map's step count (fewer steps = a prefix of the sum).
 *   bias               : bf16 [n] (this rank's chunk) or NULL when epi == TP_EPI_NONE.
 *   y                  : [m, n], fp32 or bf16.
 *   preact             : optional bf16 [m, n]: A rounded to bf16, saved for backward.
 *   workspace          : >= tp_linear_workspace_size(.., TP_PASS_FWD) bytes, 16-byte aligned (may be
 *                        NULL when that size is 0).
 * Defined by: Section 2.2, tensor-parallelism paragraphs (1D: first weight cut by columns, second by
 * rows, partial outputs; 2D / 2.5D / 3D: the chunk shapes) with the layer Y = W X of Section 3.1
 * written tokens-major and completed by bias and erf-GeLU.  When the map marks the output as an
 * additive partial (1D_ROW with p > 1, 3D_GATHERED) bias, GeLU and preact are refused (TP_ERR_MODE:
 * they belong after the summation, see tp_bias_act) and y must be fp32 (TP_ERR_DTYPE).
 * Errors: TP_ERR_NULL, TP_ERR_MODE, TP_ERR_GRID, TP_ERR_SHAPE, TP_ERR_ALIGN, TP_ERR_DTYPE,
 * TP_ERR_WORKSPACE, TP_ERR_HIP; nothing is launched unless every check has passed.
 */
int tp_linear_fwd(const tp_grid_t* grid, const tp_dims_t* dims, int n_steps,
                  const tp_cblk_t* x_blocks, const tp_cblk_t* w_blocks,
                  const void* bias, int epi, tp_oblk_t y, tp_oblk_t preact,
                  void* workspace, size_t workspace_bytes, void* hip_stream);
int tp_linear_fwd_ex(const tp_grid_t* grid, const tp_dims_t* dims, int n_steps,
                     const tp_cblk_t* x_blocks, const tp_cblk_t* w_blocks,
                     const void* bias, int epi, tp_oblk_t y, tp_oblk_t preact,
                     void* workspace, size_t workspace_bytes, void* hip_stream, const tp_plan_opts_t* opts);

/*
 * tp_linear_fwd_static -- tp_linear_fwd for callers that cannot allocate device memory and have no
 * workspace to hand over: code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc.  Same arguments, same checks and the same result as tp_linear_fwd with default plan
 * options, minus the workspace: the fp32 partial planes of a K-split product go to a fixed array of
 * tp_static_scratch_bytes() = 64 MiB that is part of the library's device image (each GPU the library
 * runs on holds its own copy until the process ends).  The call allocates and frees nothing; the
 * first call on a device looks the array's address up once (not capturable: make one call on the
 * device before capturing).  A product whose planes need more than the array is refused with
 * TP_ERR_SCRATCH and nothing is launched.  All calls on one GPU share the array: calls that may
 * overlap in time on one GPU (different streams, different threads) race on it and must be ordered
 * by the caller.  Nothing in the array has to start at zero: every partial the fix-up pass reads
 * was written by the product kernel of the same call.
 * Errors: those of tp_linear_fwd except TP_ERR_WORKSPACE, plus TP_ERR_SCRATCH.
 */
int tp_linear_fwd_static(const tp_grid_t* grid, const tp_dims_t* dims, int n_steps,
                         const tp_cblk_t* x_blocks, const tp_cblk_t* w_blocks,
                         const void* bias, int epi, tp_oblk_t y, tp_oblk_t preact, void* hip_stream);
/* Size in bytes of the built-in scratch array of tp_linear_fwd_static (host only, no GPU call). */
size_t tp_static_scratch_bytes(void);

/*
 * tp_linear_bwd -- backward share.  In order, each part only if its outputs are wanted:
 *   (1) own dA:  da_own_out = bf16(dy_own * GeLU'(preact_own))          [m_y, n_y] of the forward block;
 *                needs dy_own, preact_own, da_own_out.  When own_slot_dx >= 0 (own_slot_dw >= 0) the
 *                block just written is used as da_row_blocks[own_slot_dx] (da_col_blocks[own_slot_dw]),
 *                whatever those host entries hold.  db (fp32 [n_y], optional) receives its column sums.
 *   (2) dX = sum_{k<n_steps_dx} da_row_blocks[k] w_blocks_dx[k]^T        extents from TP_PASS_DX;
 *                if dgelu_preact is given (bf16, same shape as dX: the previous layer's saved
 *                pre-activation; the 1D chain) the result is multiplied by GeLU' of it in the epilogue.
 *   (3) dW = sum_{k<n_steps_dw} x_blocks_dw[k]^T da_col_blocks[k]        extents from TP_PASS_DW;
 *                fp32 output only (TP_ERR_DTYPE otherwise).
 *   For a layer without activation (1D_ROW) pass the upstream gradient blocks as the "da" blocks.
 *   workspace: >= max(tp_linear_workspace_size(DX), tp_linear_workspace_size(DW)).
 * Defined by: the gradients of the layer of tp_linear_fwd under the same partition (Section 2.2; the
 * three products of a layer, forward and two backward, are what the factor 3 of Table 1, Section 3.1,
 * counts for 2D and 2.5D), each rank accumulating its own block of dX and dW over the steps.  A dX
 * that the map marks as an additive partial (1D_COL with p > 1, 3D_GATHERED) must be fp32
 * (TP_ERR_DTYPE) and takes no dgelu_preact (TP_ERR_MODE).
 * Errors: as tp_linear_fwd.
 */
int tp_linear_bwd(const tp_grid_t* grid, const tp_dims_t* dims, int n_steps_dx, int n_steps_dw,
                  const tp_cblk_t* dy_own, const tp_cblk_t* preact_own,
                  const tp_cblk_t* da_row_blocks, const tp_cblk_t* w_blocks_dx,
                  const tp_cblk_t* x_blocks_dw, const tp_cblk_t* da_col_blocks,
                  int own_slot_dx, int own_slot_dw,
                  const tp_cblk_t* dgelu_preact,
                  tp_oblk_t dx, tp_oblk_t dw, tp_oblk_t da_own_out, void* db_f32,
                  void* workspace, size_t workspace_bytes, void* hip_stream);
int tp_linear_bwd_ex(const tp_grid_t* grid, const tp_dims_t* dims, int n_steps_dx, int n_steps_dw,
                     const tp_cblk_t* dy_own, const tp_cblk_t* preact_own,
                     const tp_cblk_t* da_row_blocks, const tp_cblk_t* w_blocks_dx,
                     const tp_cblk_t* x_blocks_dw, const tp_cblk_t* da_col_blocks,
                     int own_slot_dx, int own_slot_dw,
                     const tp_cblk_t* dgelu_preact,
                     tp_oblk_t dx, tp_oblk_t dw, tp_oblk_t da_own_out, void* db_f32,
                     void* workspace, size_t workspace_bytes, void* hip_stream, const tp_plan_opts_t* opts);

/*
 * tp_partials_map -- the partition map of the backward products in their other SUMMA form, for 2D
 * and 2.5D grids (host only).  The rank's own dA block (own_row, own_col) stays in place, one block
 * of the other operand takes part per step, and step k's product is an additive partial of the
 * block (out_row[k], out_col[k]) that another rank of the same row (dX) or column (dW) group owns.
 * This is the form whose traffic Table 1 (Section 3.1) counts for 2D and 2.5D: per product,
 * (side - 1) operand blocks in and (side - 1) partial blocks out.  Chunk grids as in tp_block_map.
 *   TP_PASS_DX_PARTIALS: P_k[m,n] = dA[own] W[other_k]^T      out indexes dX;   m, n, k = M_blk, H_blk, F_blk
 *   TP_PASS_DW_PARTIALS: P_k[m,n] = X[other_k]^T dA[own]      out indexes dW;   m, n, k = H_blk, F_blk, M_blk
 * other_row .. out_col are host arrays of TP_MAX_STEPS ints (may be NULL).
 * Errors: TP_ERR_NULL, TP_ERR_MODE (other modes or passes), TP_ERR_GRID, TP_ERR_SHAPE.
 */
int tp_partials_map(const tp_grid_t* grid, const tp_dims_t* dims, int pass,
                    int* n_steps, int64_t* m, int64_t* n, int64_t* k,
                    int* own_row, int* own_col, int* other_row, int* other_col,
                    int* out_row, int* out_col);

/*
 * tp_linear_bwd_partials -- backward share in the form tp_partials_map describes: all n_dx (n_dw)
 * products of a pass run in ONE launch whose tile grid covers every product, so a share whose
 * single product has too few tiles for the chip still fills it.
 *   da_own        : the rank's own dA block, bf16 [M_blk, F_blk].
 *   w_blocks_dx   : host array [n_dx] of W blocks [H_blk, F_blk];  dx_partials: host array [n_dx] of
 *                   fp32 outputs [M_blk, H_blk];  dx_partials[k] = da_own w_blocks_dx[k]^T.
 *   x_blocks_dw   : host array [n_dw] of X blocks [M_blk, H_blk];  dw_partials: host array [n_dw] of
 *                   fp32 outputs [H_blk, F_blk];  dw_partials[k] = x_blocks_dw[k]^T da_own.
 *   n_dx, n_dw    : 0 (skip that pass) .. the map's step count.
 *   workspace     : >= max over the passes used of tp_linear_workspace_size(.., TP_PASS_D?_PARTIALS).
 * Outputs are fp32 (they are summands of a reduction): TP_ERR_DTYPE otherwise.  The output blocks of
 * one call must not overlap each other (their byte ranges [ptr, ptr + ((rows - 1) ld + cols) 4) are
 * compared pairwise): TP_ERR_SHAPE otherwise.
 * Defined by: Section 3.1, Table 1 (2D, 2.5D rows) read with Section 2.2's chunk shapes.
 */
int tp_linear_bwd_partials(const tp_grid_t* grid, const tp_dims_t* dims, int n_dx, int n_dw,
                           const tp_cblk_t* da_own,
                           const tp_cblk_t* w_blocks_dx, const tp_oblk_t* dx_partials,
                           const tp_cblk_t* x_blocks_dw, const tp_oblk_t* dw_partials,
                           void* workspace, size_t workspace_bytes, void* hip_stream);
int tp_linear_bwd_partials_ex(const tp_grid_t* grid, const tp_dims_t* dims, int n_dx, int n_dw,
                              const tp_cblk_t* da_own,
                              const tp_cblk_t* w_blocks_dx, const tp_oblk_t* dx_partials,
                              const tp_cblk_t* x_blocks_dw, const tp_oblk_t* dw_partials,
                              void* workspace, size_t workspace_bytes, void* hip_stream, const tp_plan_opts_t* opts);

/*
 * tp_bias_act -- what follows the summation of forward partials (1D_ROW and 3D_GATHERED outputs
 * after their reduction):  A = c + bias,  y = GeLU(A) (epi TP_EPI_BIAS_GELU) or A (TP_EPI_BIAS) or c
 * (TP_EPI_NONE: a dtype conversion).  c: fp32 [rows, cols] with leading dimension ld_c; bias: bf16
 * [cols] or NULL with TP_EPI_NONE; y: fp32 or bf16; preact: optional bf16 copy of A.  cols and every
 * ld multiples of 8.  HBM-bound.
 * Defined by: Section 2.2, 1D paragraph (every device holds a partial output and an all-reduce
 * completes it) and the 3D chunk shape [P/p^2, Q/p]: what is applied to the rank's chunk once the sum
 * exists.  Errors: TP_ERR_NULL, TP_ERR_MODE, TP_ERR_SHAPE, TP_ERR_ALIGN, TP_ERR_DTYPE, TP_ERR_HIP.
 */
int tp_bias_act(const void* c, int64_t ld_c, const void* bias, int epi, tp_oblk_t y, tp_oblk_t preact,
                int64_t rows, int64_t cols, void* hip_stream);

/*
 * tp_dgelu -- the elementwise part of backward on its own:  da = bf16(dy * GeLU'(preact)),
 * all three bf16 [rows, cols] row-major with their own leading dimensions.  HBM-bound.
 * Defined by: the derivative of the erf-GeLU of tp_linear_fwd, GeLU'(a) = Phi(a) + a phi(a), applied to
 * a rank's own block of the output gradient (the chunk [P/q, Q/q], [P/(q d), Q/q] or [P/p^2, Q/p] of
 * Section 2.2).  Errors: TP_ERR_NULL, TP_ERR_SHAPE, TP_ERR_ALIGN, TP_ERR_HIP.
 */
int tp_dgelu(const void* dy, int64_t ld_dy, const void* preact, int64_t ld_pre,
             void* da, int64_t ld_da, int64_t rows, int64_t cols, void* hip_stream);

/*
 * tp_bias_grad -- db = 1^T dA: column sums of a bf16 block [rows, cols] (leading dimension ld) into
 * fp32 [cols], in a summation order fixed by (rows, cols) and whether there is a workspace (the same bits on every call).  This is
 * what tp_linear_bwd writes to db_f32 for the block it forms itself; here for a dA block that already
 * exists (the 1D chain, where dA is the epilogue of the second layer's dX).  HBM-bound.
 *   workspace : optional device scratch of >= tp_bias_grad_workspace_size(rows, cols) bytes, 16-byte
 *               aligned: more than 512 rows are then summed in slabs by many workgroups and the slab
 *               sums added in a fixed order (eight interleaved chains) by a second kernel.  NULL: each
 *               workgroup sums all rows of its strip of columns (slow when cols is small).  The two
 *               forms add in different orders and may differ in the last bits; each is reproducible.
 *               Too small or misaligned: TP_ERR_WORKSPACE.
 * Defined by: the bias gradient of the layer of tp_linear_fwd for one column chunk of the bias
 * (Section 2.2 chunking of the output columns).
 * Errors: TP_ERR_NULL, TP_ERR_SHAPE, TP_ERR_ALIGN, TP_ERR_WORKSPACE, TP_ERR_HIP.
 */
int tp_bias_grad(const void* da, int64_t ld_da, int64_t rows, int64_t cols, void* db_f32,
                 void* workspace, size_t workspace_bytes, void* hip_stream);
/* Bytes of workspace the slab form of tp_bias_grad wants (0: it would not split the rows).  Host only. */
size_t tp_bias_grad_workspace_size(int64_t rows, int64_t cols);

/*
 * Dropout beside the layer, with a mask that is never stored.  Element (R, C) of the FULL matrix (R, C: its row and column there) is kept
 * where its 16 random bits are at least T = p 65536 rounded to the nearest integer, and then multiplied by 65536 / (65536 - T); a dropped one is 0,
 * whatever it was, NaN included.  The bits are Philox4x32-10 of the counter {C / 8, R, offset low, offset high} under the key {seed low, seed
 * high} (Salmon, Moraes, Dror, Shaw 2011): columns 8 g .. 8 g + 7 share one draw of four words, column 8 g + 2 i its word i's low half,
 * column 8 g + 2 i + 1 the high half.  So every rank of every grid draws its own part of one and the same mask, and backward draws it again.
 *   seed, offset : which mask: a number of its own for every layer and step.
 *   offset_dev   : optional DEVICE uint64, 8-byte aligned: added to offset (mod 2^64) when the kernels run, so that replays of a captured graph
 *                  draw new masks.
 *   row0, col0   : where the block's first element lies in the full matrix; col0 a multiple of 8.
 *   p            : probability of dropping, 0 <= p <= 1 (p = 1 drops everything).
 * Refused: p outside [0, 1] or NaN (TP_ERR_MODE), col0 not a multiple of 8 or offset_dev misaligned (TP_ERR_ALIGN), negative positions, rows that
 * end beyond 2^32 or columns beyond 2^35, and blocks of 2^32 columns or more (TP_ERR_SHAPE).
 */
typedef struct { uint64_t seed, offset; const uint64_t* offset_dev; int64_t row0, col0; double p; } tp_dropout_t;

/*
 * tp_dropout_fwd -- what follows a product or the summation of its partials, with dropout:
 *     A = x + bias,   y = drop(GeLU(A)) + residual  (epi TP_EPI_BIAS_GELU; TP_EPI_BIAS: drop(A) + residual; TP_EPI_NONE: drop(x) + residual)
 *   x        : fp32 or bf16 (x_dtype) [rows, cols];  bias: bf16 [cols] or NULL with TP_EPI_NONE;
 *   residual : optional bf16 [rows, cols] (NULL ptr: none);  y: fp32 or bf16;  preact: optional bf16 copy of A.
 * y, or preact, may be x or residual itself (same address, type and leading dimension); apart from that neither may overlap these or the other
 * (TP_ERR_SHAPE; rows equally far apart may lie between each other's, for others the spans count).  cols and every ld multiples of 8.  HBM-bound.
 * Defined by: Section 2.2, 1D paragraph and the chunk shapes of 2D / 2.5D / 3D, as tp_bias_act: what is applied to a rank's chunk of the output
 * once it exists.  Nothing is done with rows = 0 or cols = 0 (blocks may be NULL then).
 * Errors: TP_ERR_NULL, TP_ERR_MODE, TP_ERR_SHAPE, TP_ERR_ALIGN, TP_ERR_DTYPE, TP_ERR_HIP.
 */
int tp_dropout_fwd(const tp_dropout_t* drop, const void* x, int64_t ld_x, int x_dtype, const void* bias, int epi, tp_cblk_t residual,
                   tp_oblk_t y, tp_oblk_t preact, int64_t rows, int64_t cols, void* hip_stream);

/*
 * tp_dropout_bwd -- its gradient:  dx = drop'(dy) GeLU'(preact)  (without preact: drop'(dy)), bf16, and optionally db (fp32 [cols]): the
 * column sums of dx before its rounding, in an order fixed by (rows, cols) and whether there is a workspace (up to 2^30 - 256 columns then, else
 * TP_ERR_SHAPE).  The residual's gradient is dy itself.
 *   drop      : as in forward.   dy, preact, dx: bf16 [rows, cols];  dx may be dy or preact itself (same leading dimension), else must not overlap
 *               it (TP_ERR_SHAPE).
 *   workspace : as in tp_bias_grad (tp_bias_grad_workspace_size(rows, cols) bytes, 16-byte aligned, or NULL); read only if db is wanted.
 * With rows = 0 db is all zeros (blocks may be NULL then).  Errors: as tp_dropout_fwd, and TP_ERR_WORKSPACE.
 */
int tp_dropout_bwd(const tp_dropout_t* drop, const void* dy, int64_t ld_dy, const void* preact, int64_t ld_pre, void* dx, int64_t ld_dx,
                   void* db_f32, int64_t rows, int64_t cols, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Low-rank adapters of many requests beside the shared projection of tp_linear_fwd.  A pool holds n_adapters adapters of one rank (a smaller one is
 * filled up with zero rows); adapter i has the factors A_i: [rank, H] and B_i: [rank, F], bf16, both as `rank` rows, and the scale s_i.  The rows of
 * a block come in segments, a request each: segment s is rows offsets[s] .. offsets[s + 1] - 1 and uses adapter ids[s], or none where ids[s] is not one
 * of 0 .. n_adapters - 1.  Rows in no segment (before offsets[0], behind the last one) are left as they were in every output.  All three arrays are read
 * by the kernels: lengths may differ from call to call, and from replay to replay of a captured graph.  offsets must ascend (empty
 * segments are fine); values outside 0 .. rows are taken as the nearest of these, and from any others come wrong rows, but no access outside the blocks.
 *   offsets : DEVICE int32 [n_segments + 1];   ids : DEVICE int32 [n_segments];   scale : DEVICE fp32 [n_adapters] or NULL (all 1);
 *   rank    : a multiple of 8 up to TP_ADAPTER_MAX_RANK.
 */
#define TP_ADAPTER_MAX_RANK 128
#define TP_ADAPTER_MAX_POOL 32767
typedef struct { const int32_t* offsets; const int32_t* ids; const float* scale; int32_t n_segments, n_adapters, rank; } tp_adapters_t;
/* A chunk of one factor of every adapter: bf16, adapter i's [rank, cols] chunk at ptr + i stride, its rows ld apart (both in elements). */
typedef struct { const void* ptr; int64_t ld, stride; } tp_factor_t;
/* The same as an output: fp32. */
typedef struct { void* ptr; int64_t ld, stride; } tp_factor_out_t;

/*
 * tp_adapter_fwd -- the adapters' part of a rank's forward share, and what follows it:
 *     V = sum_{k<n_steps} drop(X_k) A_k^T   (row by row, with the row's own adapter),   A = c + s V B + bias,   y = GeLU(A) (TP_EPI_BIAS_GELU) or A
 *   grid, dims, n_steps, x_blocks : as in tp_linear_fwd: X_k is [m, k].
 *   a_blocks : host array [n_steps]: A_k is the chunk [rank, k] of A's columns that belongs to X_k (chunk a_col[k] of tp_block_map).
 *   b        : the chunk [rank, n] of B's columns (chunk out_col).
 *   drop     : dropout on the adapters' input, or NULL.  Positions are those in the full X [M, H] (the library adds the blocks' own), behind
 *              row0, col0.
 *   c, y     : [m, n], fp32 or bf16 each: the shared product (tp_linear_fwd with TP_EPI_NONE) and the output.  y may be c itself (same address, type and
 *              leading dimension), else the two must not overlap (TP_ERR_SHAPE; rows equally far apart may lie between each other's, for others the
 *              spans count).   bias, epi, preact: as in tp_linear_fwd.
 *   v        : optional fp32 [m, rank], rows rank apart: V, saved for backward (rows without an adapter are not written).
 *   workspace: >= tp_adapter_workspace_size(.., TP_PASS_FWD, ..) bytes, 16-byte aligned; one call's at a time.
 * Apart from y over c no output may overlap an input or another output.
 * V is the rank's own sum.  Where the shared product is an additive partial (1D_ROW, 3D_GATHERED), so is this: every rank adds the part of its own
 * columns of A, the reduction that completes c completes it, and epi, preact and a bf16 y are refused as in tp_linear_fwd.
 * Defined by: the adapted layer X (W + s A^T B) under the partition of tp_linear_fwd (Section 2.2): A is cut like W's rows, B like W's columns.
 * V is fp32; in the second product it stands as a sum of bf16 terms that is off by 2^-17 (bf16 y) or 2^-25 (fp32 y) of it.  What an infinite element of B
 * reaches may therefore be NaN where the formula says infinity (in backward: what one of A, X or dY reaches in dX, dA or dB).
 * Errors: TP_ERR_NULL, TP_ERR_MODE, TP_ERR_GRID, TP_ERR_SHAPE (also: rank, pool or segment counts out of range, or more than 2^22 tiles of 16 rows of
 * short segments or 64 of long ones), TP_ERR_ALIGN, TP_ERR_DTYPE,
 * TP_ERR_WORKSPACE, TP_ERR_HIP; nothing is launched unless every check has passed.
 */
int tp_adapter_fwd(const tp_grid_t* grid, const tp_dims_t* dims, int n_steps, const tp_adapters_t* adapters, const tp_cblk_t* x_blocks,
                   const tp_factor_t* a_blocks, const tp_factor_t* b, const tp_dropout_t* drop, tp_oblk_t c, const void* bias, int epi, tp_oblk_t y,
                   tp_oblk_t preact, float* v, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * tp_adapter_bwd -- the gradients of the adapters' part, each only if wanted:
 *     U = sum_{k<n_steps} dY_k B_k^T,   dX = dx_base + drop'(s U A),   dA_i = s_i sum U^T drop(X),   dB_i = s_i sum V^T dY   (sums over the rows of adapter i)
 *   n_steps, dy_blocks, b_blocks : dY_k [m, F chunk] and the chunk [rank, F chunk] of B that belongs to it, in the order of TP_PASS_DX's a blocks
 *              (needed for dX and dA).   dY is the gradient of A = c + s V B + bias.
 *   a        : the chunk [rank, n_dx] of A's columns that TP_PASS_DX's output has (needed for dX).
 *   dx_base, dx : [m, n_dx], fp32 or bf16 each: the shared product's dX (tp_linear_bwd) and the output; dx may be dx_base itself, as y and c above.
 *   x_own    : the rank's own X block [m, n_dx] (needed for dA);   dy_own: its own dY block [m, n_fwd] and v: V of these rows (needed for dB).
 *   da, db   : fp32, [rank, n_dx] and [rank, n_fwd] per adapter.  Adapters without rows get zeros.  accumulate != 0: added to what is there.
 *   drop     : as in forward (NULL: none).   workspace: >= tp_adapter_workspace_size(.., TP_PASS_DX, ..) bytes.
 * dA and dB are the sums over this rank's own rows: additive partials over the row chunks, and, where U or V is one (1D_COL, 1D_ROW, 3D_GATHERED), over those
 * ranks as well.  A dX that the map marks as a partial must be fp32.  The order of every sum is fixed by the arguments.  Apart from dx over dx_base no
 * output may overlap an input or another output.
 * Defined by: the gradients of tp_adapter_fwd under the same partition.  Errors: as tp_adapter_fwd.
 */
int tp_adapter_bwd(const tp_grid_t* grid, const tp_dims_t* dims, int n_steps, const tp_adapters_t* adapters, const tp_cblk_t* dy_blocks,
                   const tp_factor_t* b_blocks, const tp_factor_t* a, const tp_dropout_t* drop, tp_oblk_t dx_base, tp_oblk_t dx, const tp_cblk_t* x_own,
                   tp_factor_out_t da, const tp_cblk_t* dy_own, const float* v, tp_factor_out_t db, int accumulate, void* workspace,
                   size_t workspace_bytes, void* hip_stream);

/* Bytes of device workspace tp_adapter_fwd (TP_PASS_FWD) or tp_adapter_bwd (TP_PASS_DX) may need with n_segments or any smaller number of them: planes of
 * V or U, and of dA and dB where their rows are shared out (up to 32 of each adapter in the pool).  Only n_segments, n_adapters and rank of `adapters`
 * are looked at.  0 on invalid arguments.  Host only. */
size_t tp_adapter_workspace_size(const tp_grid_t* grid, const tp_dims_t* dims, int pass, const tp_adapters_t* adapters);

/* Human-readable name of a status code (static storage). */
const char* tp_strerror(int status);

#ifdef __cplusplus
}
#endif
#endif /* TP_LINEAR_H */
