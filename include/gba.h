/*
 * gba.h -- fused fp16 GEMM + bias + activation for AMD MI355X (gfx950).
 *
 * C ABI of libgba.so.  Plain pointers and sizes only; C99 compatible.
 *
 * The headline operation is the matmul followed by the pointwise
 * ReLU-of-add statement of the paper's Problem Statement section (Listing 1
 * and its expression tree, whose root is ReLU over the add of the matmul
 * result and the bias), computed in ONE kernel so the matmul result never
 * goes to global memory (Kernel Fusion section, "Pointwise Operations in
 * Epilogue").  gba_fused_gemm adds the section's other idioms: a ReLU
 * prologue, a second matmul feeding the epilogue, a full or subtracted bias
 * and the Sigmoid and Tanh activations.
 * Operands may be row- or column-major, the four layout specialisations of
 * the Matmul Compute Decomposition section.
 *
 * Common conventions for every entry point below:
 *   - All array pointers are DEVICE pointers (memory the caller allocated on
 *     the GPU that is current for `stream`).  fp16 means IEEE binary16.
 *   - The caller owns every buffer.  The library never allocates, frees or
 *     synchronises; it keeps no mutable global state and is thread-safe.
 *     The one exception is gba_fused_gemm_noalloc, which uses a static
 *     device array of the library's own (see there).
 *   - Calls are asynchronous: work is enqueued on `stream` (NULL = the null
 *     stream) and the function returns once the kernel is launched.
 *   - Arguments are validated on the host before anything is enqueued.  On
 *     any error nothing is launched and the output is left untouched (one
 *     exception: when the runtime fails between the two launches of a split
 *     reduction, GBA_EHIP, the workspace holds partial sums and has to be
 *     zero-filled before it is used again).
 *   - Outputs must not alias inputs.
 *   - Inputs are expected to be finite.  The outputs for NaN or infinite
 *     inputs, and for results beyond the fp16 range, are not specified.
 */
#ifndef GBA_H
#define GBA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ABI-identical to hipStream_t. */
typedef struct ihipStream_t *gba_stream_t;

typedef enum { GBA_ROW_MAJOR = 0, GBA_COL_MAJOR = 1 } gba_layout;
/* Epilogue activation (the pointwise ops of the Introduction's scope):
 * identity, ReLU max(x, 0), Sigmoid 1 / (1 + exp(-x)), Tanh. */
typedef enum { GBA_ACT_NONE = 0, GBA_ACT_RELU = 1, GBA_ACT_SIGMOID = 2, GBA_ACT_TANH = 3 } gba_act;
typedef enum { GBA_ACC_F32 = 0, GBA_ACC_F16 = 1 } gba_acc;
typedef enum {
    GBA_OK = 0,
    GBA_EINVAL = 1,        /* malformed argument (negative size, ld too small, NULL, bad enum) */
    GBA_EUNSUPPORTED = 2,  /* well-formed but outside what the library implements */
    GBA_EHIP = 3,          /* the HIP runtime reported an error at launch */
    GBA_ESCRATCH = 4       /* gba_fused_gemm_noalloc: the request needs more scratch than
                              GBA_NOALLOC_SCRATCH_BYTES */
} gba_status;

/*
 * gemm_bias_act -- C = act(A*B + bias), fp16 in, fp16 out.
 *
 * Follows the Problem Statement section (Listing 1): for 0<=i<M, 0<=j<N
 *     pre(i,j) = sum_{k<K} A(i,k) * B(k,j) + (bias ? bias[j] : 0)
 *     C[i*ldc + j] = fp16( act == GBA_ACT_RELU ? max(pre, 0) : pre )
 * with products summed in fp32 (accum == GBA_ACC_F32; fp16 inputs and fp32
 * accumulation as in the Background section) or with the running sum rounded
 * to fp16 after every aligned group of 32 k values (accum == GBA_ACC_F16).
 * The bias add and activation are done in fp32 and rounded once to fp16
 * (RNE).  act may also be GBA_ACT_SIGMOID or GBA_ACT_TANH (see
 * gba_fused_gemm for their accuracy).
 *
 * Layout and leading dimensions (BLAS meaning):
 *     A(i,k) = layoutA == GBA_ROW_MAJOR ? A[i*lda + k] : A[k*lda + i]
 *              (lda >= K resp. lda >= M)
 *     B(k,j) = layoutB == GBA_ROW_MAJOR ? B[k*ldb + j] : B[j*ldb + k]
 *              (ldb >= N resp. ldb >= K)
 *     C is always row-major, ldc >= N.
 *     bias: fp16[N] broadcast over rows, or NULL for no bias.
 * Sizes that are not tile multiples are handled inside the kernel (masked
 * loads and stores); nothing outside the stated extents is read or written.
 * Pointers need only fp16 (2-byte) alignment; 16-byte aligned A, B, C, bias
 * with lda, ldb, ldc multiples of 8 take the vectorised fast path.
 *
 * Degenerate sizes: M == 0 or N == 0 -> GBA_OK, nothing launched.
 * K == 0 -> C = act(bias) (the empty sum is zero).
 * Errors: GBA_EINVAL for M, N or K < 0, a leading dimension below its
 * extent, a NULL A/B (when M,N,K > 0) or C (when M,N > 0), or a bad enum;
 * GBA_EUNSUPPORTED for M, N or K above 2^31-1 or pointers not 2-byte
 * aligned; GBA_EHIP if the launch fails.
 */
gba_status gemm_bias_act(gba_layout layoutA, gba_layout layoutB,
                         int64_t M, int64_t N, int64_t K,
                         const void *A, int64_t lda,
                         const void *B, int64_t ldb,
                         const void *bias, void *C, int64_t ldc,
                         gba_act act, gba_acc accum, gba_stream_t stream);

/*
 * gemm_bias_act_tile -- gemm_bias_act with the tile configuration forced.
 *
 * The paper generates kernels for several block/warp tile sizes and keeps
 * the fastest per problem size (Experimental Evaluation section); this entry
 * point exposes that choice for sweeps.  tile_id indexes the table reported
 * by gba_tile_info; tile_id < 0 means "let the library choose" (identical to
 * gemm_bias_act).  The id that gba_select_tile answers runs the kernel the
 * library would run on that tile (a variant of it with more LDS stages and
 * waves that only copy, where that is the choice).  A tile larger than the
 * problem (bm > M or bn > N) is replaced by the library's choice, and operands
 * that miss the fast path's alignment conditions use the kernels for those
 * whatever tile_id says.  Errors
 * as gemm_bias_act, plus GBA_EINVAL for a tile_id at or beyond
 * gba_num_tiles().
 */
gba_status gemm_bias_act_tile(gba_layout layoutA, gba_layout layoutB,
                              int64_t M, int64_t N, int64_t K,
                              const void *A, int64_t lda,
                              const void *B, int64_t ldb,
                              const void *bias, void *C, int64_t ldc,
                              gba_act act, gba_acc accum, int tile_id,
                              gba_stream_t stream);

/* Left-operand prologue (Listing 4, ReLU + Matmul). */
typedef enum { GBA_PRO_NONE = 0, GBA_PRO_RELU = 1 } gba_prologue;
/* Second product (Listing 5, Sum of Matmuls): none, A.B + P.Q, A.B - P.Q. */
typedef enum { GBA_SECOND_NONE = 0, GBA_SECOND_ADD = 1, GBA_SECOND_SUB = 2 } gba_second;
/* Bias shape: none, fp16[N] broadcast over rows, or a full M x N fp16 tile. */
typedef enum { GBA_BIAS_NONE = 0, GBA_BIAS_ROW = 1, GBA_BIAS_FULL = 2 } gba_bias_kind;
/* Add or subtract the bias. */
typedef enum { GBA_OP_ADD = 0, GBA_OP_SUB = 1 } gba_op;

/*
 * gba_fused_desc -- one request of gba_fused_gemm.  Fill it with
 * gba_fused_desc_init first (which selects: row-major A and B, no prologue,
 * no second product, no bias, no activation, fp32 accumulation, library tile
 * choice), then set what the request needs.  Every pointer is a DEVICE
 * pointer; a field that the request does not use is ignored.
 */
typedef struct gba_fused_desc {
    gba_layout layoutA, layoutB;  /* also the layouts of P and Q */
    int64_t M, N, K;
    const void *A;                /* A(i,k): ROW A[i*lda+k] (lda >= K), COL A[k*lda+i] (lda >= M) */
    int64_t lda;
    const void *B;                /* B(k,j): ROW B[k*ldb+j] (ldb >= N), COL B[j*ldb+k] (ldb >= K) */
    int64_t ldb;
    gba_prologue prologue;        /* applied to A and, with a second product, to P */
    gba_second second;
    int64_t K2;                   /* reduction length of P.Q */
    const void *P;                /* M x K2, stored like A with leading dimension ldp */
    int64_t ldp;
    const void *Q;                /* K2 x N, stored like B with leading dimension ldq */
    int64_t ldq;
    gba_bias_kind bias_kind;
    gba_op bias_op;
    const void *bias;             /* ROW: bias[j]; FULL: bias[i*ldbias + j], ldbias >= N */
    int64_t ldbias;
    gba_act act;
    gba_acc accum;
    void *C;                      /* output, row-major: C[i*ldc + j], ldc >= N */
    int64_t ldc;
    int tile_id;                  /* < 0: library's choice; else as gemm_bias_act_tile */
    int split_k;                  /* 0: library's choice, 1: never, s >= 2: s-way (see below) */
    void *workspace;              /* device memory for a split reduction, or NULL */
    size_t workspace_bytes;
} gba_fused_desc;

/* Set *desc to the defaults listed above (tile_id = -1, split_k = 0, no
 * workspace, everything else zero / NONE / ADD / F32).  NULL is ignored. */
void gba_fused_desc_init(gba_fused_desc *desc);

/*
 * gba_fused_workspace_size -- bytes of workspace the request would use to
 * split its reduction across workgroups (0: it would not split).
 *
 * Splitting is an implementation choice of the fast path for fp32
 * accumulation (the paper partitions the reduction only inside a thread
 * block; this is the same partition across blocks): when an output has too
 * few tiles to occupy the GPU, or a long reduction, each output tile's
 * reduction steps (A.B's, then P.Q's) are divided among up to split_k
 * workgroups.  Each writes its fp32 partial tile to the workspace; a second
 * kernel on the same stream adds the partials in split order and runs the
 * epilogue.  Only the summation order changes, not the tolerance;
 * GBA_ACC_F16 never splits.
 *
 * Workspace contract (gba_fused_gemm): at least this many bytes, 256-byte
 * aligned, on the device the call runs on, and all zero when the call is
 * enqueued.  A call that splits uses it for the fp32 partial tiles (after a
 * reserved 32-bit word per output tile), and leaves every byte it used at
 * zero again when it completes, so a workspace zero-filled once serves
 * any number of calls in stream order, whatever their shapes and tiles;
 * calls that may run at the same time need separate workspaces.  With a NULL
 * or smaller workspace, or when a launch of the split would have 2^32 threads
 * or more, the call runs unsplit.  split_k >= 2 asks for that many splits
 * (fewer when the reduction has fewer 64-deep steps); 0 lets the library
 * decide.
 *
 * Errors: as gba_fused_gemm's validation; GBA_EINVAL also for bytes ==
 * NULL or split_k < 0.
 */
gba_status gba_fused_workspace_size(const gba_fused_desc *desc, size_t *bytes);

/*
 * gba_fused_tile -- the tile configuration gba_fused_gemm would run the
 * request on, given the workspace the descriptor carries (host-only
 * computation, no GPU access): *tile is the tile id (see gba_tile_info), or
 * -1 for a request that runs on none (outside the fast path, smaller than
 * every tile, or an empty output).  The library's choice
 * depends on the shape, the layouts, the accumulation and the prologue (see
 * gba_select_tile); a requested tile_id that fits is kept.  When the library
 * chooses, a request of few rows or few outputs over a long reduction may run
 * on the few-row kernel instead, which has no tile id: the answer is then the
 * tile it replaces.
 *
 * Errors: as gba_fused_gemm's validation; GBA_EINVAL also for tile == NULL.
 */
gba_status gba_fused_tile(const gba_fused_desc *desc, int *tile);

/* Kernel that runs a request: none (empty output), a tile of the fast path,
 * a deep variant of one, the few-row kernel, the kernel for large requests
 * outside the fast path, the general kernel. */
typedef enum {
    GBA_PATH_EMPTY = 0,
    GBA_PATH_TILE = 1,
    GBA_PATH_DEEP = 2,
    GBA_PATH_FEW_ROWS = 3,
    GBA_PATH_UNALIGNED = 4,
    GBA_PATH_GENERAL = 5
} gba_path;

typedef struct gba_plan {
    gba_path path;
    int bm, bn;           /* outputs of a workgroup: bm rows x bn columns */
    int splits;           /* workgroups each output tile's reduction is split across (1: not split) */
    int threads;          /* of a workgroup */
    int64_t workgroups;   /* of the launch (of a split's first launch) */
} gba_plan;

/*
 * gba_fused_plan -- the kernel gba_fused_gemm would run the request on and
 * its launch, given the workspace the descriptor carries (host-only
 * computation, no GPU access).  For tests and measurements: which kernel
 * runs a request is no part of its contract.
 *
 * Errors: as gba_fused_gemm's validation; GBA_EINVAL also for plan == NULL.
 */
gba_status gba_fused_plan(const gba_fused_desc *desc, gba_plan *plan);

/*
 * gba_fused_gemm -- the four computation idioms of the paper's scope
 * (Introduction) in one kernel: a matmul with a pointwise prologue
 * (Pointwise Operations in Prologue, Listing 4), with a pointwise epilogue
 * (Pointwise Operations in Epilogue, Listing 1), and two matmuls of the same
 * output shape feeding a pointwise op (Matmuls with Pointwise Epilogue,
 * Listing 5).  For 0<=i<M, 0<=j<N:
 *
 *     pro(x)   = prologue == GBA_PRO_RELU ? max(x, 0) : x
 *     Cp(i,j)  = sum_{k<K}  pro(A(i,k)) * B(k,j)
 *     R(i,j)   = sum_{k<K2} pro(P(i,k)) * Q(k,j)                 (second != NONE)
 *     Z(i,j)   = Cp + R (SECOND_ADD), Cp - R (SECOND_SUB), Cp (SECOND_NONE)
 *     pre(i,j) = Z +/- bias(i,j)   (bias_op; no term for GBA_BIAS_NONE)
 *     C[i*ldc + j] = fp16(act(pre))
 *
 * Neither Cp nor R ever reaches global memory: both products are summed in
 * ONE fp32 running sum per output (A.B's terms, then P.Q's, negated for
 * SECOND_SUB), so the P.Q operands may have a different reduction length
 * K2 as long as the output shape matches.  GBA_ACC_F16 rounds that running
 * sum to fp16 after every aligned group of 32 k values of each product.
 * The bias term and activation are evaluated in fp32 and the result rounded
 * once to fp16 (RNE).  Sigmoid and Tanh use the hardware exp2 and
 * reciprocal approximations (Tanh from its Taylor series for |x| < 1/16):
 * within a few fp32 ulps of the result, far below the fp16 rounding.
 *
 * Fast path: 16-byte aligned A, B, C and (if used) P, Q, bias; lda, ldb,
 * ldc (and ldp, ldq, ldbias when used) multiples of 8 and below 2^21 for
 * the operands; N and the contiguous extents of all operands multiples of 8.
 * Anything else takes the kernels for such requests, which need
 * 2-byte alignment only.  Outputs must not alias inputs.
 *
 * Degenerate sizes: M == 0 or N == 0 -> GBA_OK, nothing launched; K == 0
 * or K2 == 0 make that product's empty sum zero.
 * Reduction split across workgroups: see gba_fused_workspace_size.
 *
 * Errors: GBA_EINVAL for desc == NULL, a bad enum, a tile_id at or beyond
 * gba_num_tiles(), negative sizes or leading dimensions, a leading
 * dimension below its extent, a NULL pointer that the request reads
 * (A/B when K > 0, P/Q when K2 > 0, bias when bias_kind != NONE, C),
 * split_k < 0, or a workspace not 256-byte aligned;
 * GBA_EUNSUPPORTED for M, N, K or K2 above 2^31-1 or pointers not 2-byte
 * aligned; GBA_EHIP if a launch fails.  Nothing is launched on error (but see
 * the conventions above for a split).
 */
gba_status gba_fused_gemm(const gba_fused_desc *desc, gba_stream_t stream);

/*
 * gba_fused_gemm_noalloc -- gba_fused_gemm for callers that cannot allocate
 * device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc).  Same request, same result bits as
 * gba_fused_gemm given a workspace of at least gba_fused_workspace_size
 * bytes; desc->workspace and desc->workspace_bytes are ignored.
 *
 * When the request splits its reduction across workgroups, the split's
 * workspace is the library's own static device array of
 * GBA_NOALLOC_SCRATCH_BYTES bytes (one per GPU, created with the library's
 * code object and held until the process ends).  Requests that do not
 * split use no scratch.  The call allocates nothing (no hipMalloc, no
 * allocating library routine); its first call on a device looks up that
 * device's scratch address once, with the device current.
 *
 * Every call on one GPU shares that GPU's scratch: calls that may overlap on
 * one GPU (different streams, different host threads without ordering) race
 * on it and give undefined results.  Calls in one stream's order are safe.
 *
 * Errors: as gba_fused_gemm; GBA_ESCRATCH (nothing launched) when the split
 * the request asks for (or the library chooses) needs more than
 * GBA_NOALLOC_SCRATCH_BYTES; GBA_EUNSUPPORTED for a device index >= 64.
 */
#define GBA_NOALLOC_SCRATCH_BYTES ((size_t)16 << 20)
gba_status gba_fused_gemm_noalloc(const gba_fused_desc *desc, gba_stream_t stream);

/* Number of tile configurations compiled into the library. */
int gba_num_tiles(void);

/*
 * gba_tile_info -- describe tile configuration tile_id (Tiling for Blocks
 * and Warps and Split-K subsections): block tile bm x bn x bk (output rows x
 * output columns x reduction depth per step), waves per workgroup and the
 * intra-workgroup split-K factor.  Any output pointer may be NULL.
 * Returns GBA_EINVAL for an unknown tile_id.
 */
gba_status gba_tile_info(int tile_id, int *bm, int *bn, int *bk, int *waves, int *split_k);

/*
 * gba_select_tile -- the tile configuration gemm_bias_act would use for this
 * problem on its aligned fast path (host-only computation, no GPU access).
 * gba_fused_gemm makes the same choice for requests without the prologue
 * (K being the total reduction length of both products); with the prologue
 * it may take another tile, and requests of few rows or few outputs over a
 * long reduction may run on the few-row kernel instead (see gba_fused_plan).
 * Returns the tile id, or -1 if the arguments
 * are invalid or the problem is smaller than every tile (M < 32 or N < 32:
 * general path).
 */
int gba_select_tile(gba_layout layoutA, gba_layout layoutB, int64_t M, int64_t N, int64_t K,
                    gba_acc accum);

/*
 * Unfused baseline pieces (the separate-kernel chain that the paper's
 * evaluation compares against: a GEMM, then a bias add, then an
 * activation).  Same conventions as above; C is row-major M x N with
 * leading dimension ldc >= N and is updated in place:
 *   gba_bias_add_f16: C[i*ldc+j] = fp16(C[i*ldc+j] + bias[j])  (fp32 add)
 *   gba_relu_f16:     C[i*ldc+j] = max(C[i*ldc+j], 0)
 *   gba_add_f16:      C[i*ldc+j] = fp16(C[i*ldc+j] + X[i*ldx+j])  (fp32 add;
 *                     the separate add of two matmul results, Listing 5)
 *   gba_bias_act_f16: C[i*ldc+j] = fp16(act(C[i*ldc+j] + bias[j]))  (fp32;
 *                     the bias add and activation in one pass: the second
 *                     kernel of a two-launch chain, GEMM then bias+act)
 * Errors: GBA_EINVAL for negative sizes, ldc < N (or ldx < N), NULL C, bias
 * or X when the work is non-empty, a bad act; GBA_EUNSUPPORTED for sizes above 2^31-1
 * or pointers not 2-byte aligned; GBA_EHIP if the launch fails.
 */
gba_status gba_bias_add_f16(int64_t M, int64_t N, void *C, int64_t ldc, const void *bias,
                            gba_stream_t stream);
gba_status gba_relu_f16(int64_t M, int64_t N, void *C, int64_t ldc, gba_stream_t stream);
gba_status gba_bias_act_f16(int64_t M, int64_t N, void *C, int64_t ldc, const void *bias,
                            gba_act act, gba_stream_t stream);
gba_status gba_add_f16(int64_t M, int64_t N, void *C, int64_t ldc, const void *X, int64_t ldx,
                       gba_stream_t stream);

/*
 * ---------------------------------------------------------------------------
 * A decoding step: weights in 4 bits, a paged key/value cache, and the
 * attention of the new tokens of each request over it.  The conventions at
 * the top of this file hold.  Elements are fp16 or bf16, one type a call;
 * sums and softmax statistics are held in fp32 and every result is rounded
 * once to its type.
 *
 * The cache keeps the keys and values of a request's tokens in blocks of
 * block_size tokens that may lie anywhere in it.  Row r of the block table
 * names the blocks of request r in the order of its tokens: position p of
 * the request is token p % block_size of block table[r * width + p / block_size].
 * A slot is block * block_size + token.
 */
typedef enum { GBA_F16 = 0, GBA_BF16 = 1 } gba_dtype;

/*
 * gba_q4_weight -- a K x N matrix in 4 bits with one scale, and if zeros is
 * not NULL one zero point, for every `group` consecutive k of a column:
 *
 *     W(k,j) = scale(k / group, j) * (code(k,j) - zero(k / group, j))
 *
 * with codes 0..15 and zero 8 where zeros is NULL.  Storage:
 *   codes   32-bit words [ceil(N/16)][ceil(K/128)][64][4]: word (nb, kb, l, i)
 *           holds column 16 nb + l % 16 and the eight k from
 *           128 kb + 32 i + 8 (l / 16) on, the e-th of them in the four bits
 *           from 4 (e / 2) + 16 (e % 2) on.  What stands beyond K or N is
 *           not used.
 *   scales, zeros   elements [ceil(N/16)][ceil(K/group)][16] of type dtype:
 *           (nb, g, c) belongs to column 16 nb + c.
 * 16-byte aligned codes; group 32, 64 or 128.
 */
typedef struct gba_q4_weight {
    gba_dtype dtype;
    int group;
    int64_t K, N;
    const void *codes;
    const void *scales;
    const void *zeros;
} gba_q4_weight;

/*
 * gba_q4_pack -- the stored form of the codes of a K x N matrix: reads one
 * code a byte (its low four bits), codes[k * ld + j], ld >= N, and writes the
 * ceil(N/16) * ceil(K/128) * 256 words that gba_q4_weight describes (zeros
 * beyond K and N).
 * Errors: GBA_EINVAL for negative sizes, ld < N, or a NULL pointer with a
 * non-empty matrix; GBA_EUNSUPPORTED for K or N above 2^31-1 or packed not
 * 16-byte aligned; GBA_EHIP if the launch fails.
 */
gba_status gba_q4_pack(int64_t K, int64_t N, const void *codes, int64_t ld, void *packed,
                       gba_stream_t stream);

/*
 * gba_q4_linear -- C = act(A*W + bias) over a few rows: for 0<=i<M, 0<=j<N
 *     C[i*ldc + j] = act( sum_k A[i*lda + k] * W(k,j) + (bias ? bias[j] : 0) )
 * A (row-major, lda >= K), bias (N, or NULL) and C (row-major, ldc >= N) are
 * of the weight's dtype.  Products are exact and summed in fp32; scales are
 * applied to each group's fp32 sum.  Meant for up to 64 rows, which share one
 * pass over the weights; more rows run as blocks of 64.  Where that sum is not
 * finite, as with infinities or NaN in A, C is what the formula gives in 64 bits;
 * an activation of NaN is NaN.
 * A and C need the alignment of an element only.
 * M == 0 or N == 0: nothing is launched.  K == 0: C = act(bias).
 * Errors: GBA_EINVAL for w == NULL, a bad enum or group, negative sizes, a
 * leading dimension below its extent, a NULL pointer that is read or written;
 * GBA_EUNSUPPORTED for sizes above 2^31-1, codes not 16-byte aligned or
 * another pointer not 2-byte aligned, or M above 64 * 65535; GBA_EHIP if the
 * launch fails.
 */
gba_status gba_q4_linear(const gba_q4_weight *w, int64_t M, const void *A, int64_t lda, const void *bias,
                         gba_act act, void *C, int64_t ldc, gba_stream_t stream);

/*
 * gba_block_tables -- the block tables of a batch and the stack of blocks
 * that no request holds.  All arrays are on the device and the caller's:
 * table[requests * width], held[requests] (blocks a request holds: the first
 * held[r] entries of its row), free_blocks[num_blocks], free_count[1] (the
 * stack is free_blocks[0 .. free_count), its top last).  Entries of a row past
 * held are -1.  scratch: GBA_TABLES_SCRATCH(requests) words, 16-byte aligned,
 * for a step's own use.
 */
#define GBA_TABLES_SCRATCH(requests) (4 * ((requests) + 1))
typedef struct gba_block_tables {
    int64_t requests, width, num_blocks;
    int64_t block_size;
    int32_t *table;
    int32_t *held;
    int32_t *free_blocks;
    int32_t *free_count;
    int32_t *scratch;
} gba_block_tables;

/*
 * gba_tables_step -- make room for the next tokens of every request, give
 * back what it no longer needs, and say where each new token goes.
 *
 * lens[r] tokens of request r stay in the cache and count[r] new ones come
 * after them (both 0 for a request that has ended; negative ones count as 0).
 * With need = ceil((lens + count) / block_size):
 *   1. A request that holds more than need gives its last blocks back: in
 *      request order, and within one in table order, they are pushed on the
 *      stack of free blocks and their entries become -1.
 *   2. Requests that need more take them from the top of the stack, in request
 *      order and in table order, as long as the whole rest of one still fits;
 *      the first one that does not fit and those after it that want any get
 *      none.
 * Outputs (slots and positions may be NULL):
 *   offsets[requests + 1]   where a request's new tokens begin: the running
 *                           sum of count, at most `tokens`
 *   slots[tokens]           slot of each new token (position lens + i of its
 *                           request for its i-th); -1 where status is not 0
 *   positions[tokens]       lens + i, or lens + the token's depth in its tree
 *   status[requests]        0; 1: not enough free blocks; 2: need > width;
 *                           3: more new tokens than fit `tokens`, or a tree of
 *                           more than 64 -- the last two take no blocks
 *   mask[tokens]            bit j: the token is the j-th new token of its
 *                           request or descends from it
 * Entries past the last request's tokens are -1, -1 and 0, and so are those of
 * a tree of more than 64.
 * parents (NULL: every token follows the one before it, and mask is not
 * written) gives each new token's parent as an index among the new tokens of
 * its request; a value below 0, or not below the token's own index, makes it a
 * root (depth 0).
 * Sums are of 64 bits; a step is the same whatever order its threads run in.
 *
 * Errors: GBA_EINVAL for tables == NULL, negative sizes, block_size < 1, a
 * NULL table, held, free_blocks, free_count, scratch, lens, count, offsets or
 * status with requests > 0, parents without mask; GBA_EUNSUPPORTED for more than
 * GBA_MAX_REQUESTS requests, num_blocks * block_size, tokens or requests *
 * width above 2^31-1 or a pointer not aligned to its elements;
 * GBA_EHIP if a launch fails.
 */
#define GBA_MAX_REQUESTS 4096
gba_status gba_tables_step(const gba_block_tables *tables, const int32_t *lens, const int32_t *count,
                           const int32_t *parents, int64_t tokens, int32_t *offsets, int32_t *slots,
                           int32_t *positions, int32_t *status, uint64_t *mask, gba_stream_t stream);

/*
 * gba_paged_cache -- keys and values of num_blocks * block_size tokens, heads
 * of dim elements each.  Strides are in elements; dim is contiguous.
 */
typedef struct gba_paged_cache {
    gba_dtype dtype;
    int64_t num_blocks, block_size, heads, dim;
    void *k, *v;
    int64_t k_block, k_token, k_head;
    int64_t v_block, v_token, v_head;
} gba_paged_cache;

/*
 * gba_cache_store -- write new keys and values into the cache: for each token
 * t with 0 <= slots[t] < num_blocks * block_size, head h and element d
 *     K(slots[t], h, d) = k[t*k_token + h*k_head + d], and V from v likewise.
 * Tokens with any other slot are left out.  The others' slots differ: where two
 * tokens have one, every element of its row is one or the other's, in K and in
 * V, but the row may be a mixture of both.  k and v are of the cache's dtype
 * (strides in elements).
 * Errors: GBA_EINVAL for cache == NULL, a bad enum, negative sizes, block_size
 * < 1, a NULL pointer that is read or written; GBA_EUNSUPPORTED for
 * num_blocks * block_size, tokens or heads * dim above 2^31-1, or an array of
 * elements not 2-byte aligned; GBA_EHIP if the launch fails.
 */
gba_status gba_cache_store(const gba_paged_cache *cache, int64_t tokens, const void *k, int64_t k_token,
                           int64_t k_head, const void *v, int64_t v_token, int64_t v_head,
                           const int32_t *slots, gba_stream_t stream);

/*
 * gba_attention -- one request of gba_tree_attention.  q and out: rows of
 * query heads, element d of head h of token t at t*q_token + h*q_head + d
 * (out likewise), of the cache's dtype.
 */
typedef struct gba_attention {
    gba_paged_cache cache;
    int64_t requests, width;      /* rows and row length of the block table */
    int64_t tokens;               /* rows of q, out and mask */
    int64_t max_new;              /* no request has more new tokens than this */
    int64_t q_heads;              /* a multiple of cache.heads */
    float scale;
    const void *q;
    int64_t q_token, q_head;
    void *out;
    int64_t out_token, out_head;
    const int32_t *table;         /* [requests][width] */
    const int32_t *lens;          /* [requests]: cached tokens before the new ones */
    const int32_t *offsets;       /* [requests + 1]: rows of q of each request */
    const uint64_t *mask;         /* [tokens], or NULL */
    void *workspace;
    size_t workspace_bytes;
} gba_attention;

/*
 * gba_tree_attention -- attention of each request's new tokens over the cache.
 *
 * Request r has T = offsets[r+1] - offsets[r] new tokens, rows offsets[r] ...
 * of q, whose keys and values are already in the cache at positions lens[r]
 * ... lens[r] + T - 1.  Its i-th new token sees every position below lens[r],
 * and position lens[r] + j for j < T if bit j of its mask is set (j < 64), or
 * with mask == NULL if j <= i (a chain; T == 1 is ordinary decoding).  With
 * query head h reading key head h / (q_heads / heads):
 *     s_p = scale * q . K_p            p over the positions that it sees
 *     out = sum_p exp(s_p - m) V_p / sum_p exp(s_p - m),   m = max_p s_p
 * and zeros where it sees none.  The weights exp(s_p - m) are rounded to the
 * cache's dtype for the second product, as its matrix instructions take them,
 * and their sum is that of the rounded ones.  Sums are of fp32, and in bf16 of
 * weights of up to 2^8: where a row sees P positions they have room for every V
 * below 2^119 / P, and larger ones may overflow.
 * What the cache holds at positions that a token does not see has no effect
 * on its rows, infinities and NaN included (a position whose block is outside
 * the cache counts as not seen, and so does one with a score of -infinity).  A
 * row with a NaN among the scores that it sees is NaN, however its request is
 * split.  Rows of out that belong to no request are not written; neither are those of a request
 * past max_new.  Where offsets fall, a request has no new tokens, and rows that
 * several requests claim may be left unwritten; whatever they are, nothing
 * outside the arrays is read or written.
 *
 * Workspace: with at least gba_tree_attention_workspace_size bytes, 256-byte
 * aligned, long requests are split across workgroups and their parts joined;
 * with less each request and head is one workgroup's work.  Its first 256 KB
 * hold counters: zero-filled before its first use, they are zeros again when a
 * call completes, whatever its sizes.  Calls that may overlap need separate
 * ones.
 *
 * dim a multiple of 8 up to 256; q, out, K and V 16-byte aligned with strides
 * that are multiples of 8 (out: 4), but in dimensions of one element.
 * Errors: GBA_EINVAL for desc == NULL, a bad enum, negative sizes, block_size
 * < 1, q_heads no multiple of heads, heads == 0 with tokens, a NULL pointer
 * that is read or written, a scale that is infinite or NaN (or above 2^127), a
 * workspace not 256-byte aligned; GBA_EUNSUPPORTED for other dims, alignments
 * or strides, num_blocks * block_size, requests * width, width * block_size or
 * tokens above 2^31-1, the smaller of max_new and tokens times q_heads / heads
 * above 2^31-256, more than GBA_MAX_REQUESTS requests, a launch of 2^32 threads
 * or more (with a workspace, of tokens from 2^23 on), or max_new > 64 with a
 * mask; GBA_EHIP if a launch fails.
 */
gba_status gba_tree_attention(const gba_attention *desc, gba_stream_t stream);
gba_status gba_tree_attention_workspace_size(const gba_attention *desc, size_t *bytes);

/*
 * gba_window_attention -- gba_tree_attention of a bounded part of the text.
 *
 * The text of a new token is the lens[r] cached positions of its request and
 * then the new tokens that it sees, in their order (with mask == NULL those up
 * to itself, with a mask those of its set bits below T).  Of this text it sees
 * the last `window` positions -- its own among them, if it sees itself -- and
 * the first `sinks`; everything else is as in gba_tree_attention.  Positions
 * count whether or not their block is in the cache.
 *
 * The workspace is that of gba_tree_attention, of the size that
 * gba_window_attention_workspace_size gives for the same window and sinks.
 * Errors: those of gba_tree_attention, and GBA_EINVAL for window < 1 or
 * sinks < 0.
 */
gba_status gba_window_attention(const gba_attention *desc, int64_t window, int64_t sinks, gba_stream_t stream);
gba_status gba_window_attention_workspace_size(const gba_attention *desc, int64_t window, int64_t sinks,
                                               size_t *bytes);

/*
 * gba_q4_cache -- keys and values of num_blocks * block_size tokens in 4 bits.
 * With width = 64, 128 or 256, the smallest that is not below dim, and groups =
 * max(1, width / group), element d of a key or value is
 *     scale (code - 8) + offset
 * of the scale and offset of group d / group of its row.  Storage, of K and V
 * each, contiguous:
 *   codes   32-bit words [num_blocks][heads][block_size][width / 8]: a word
 *           holds the codes of eight elements, the e-th in the four bits from
 *           4 e on.  V: word w of a row has elements 8 w ... 8 w + 7.  K: word
 *           (width / 32) g + s of a row has elements 8 (4 s + g) ... + 7, for
 *           g < 4.
 *   scales  pairs of elements [num_blocks][heads][block_size][groups][2] of type
 *           dtype: scale and offset.
 * What stands past dim is not used.  A scale or an offset that is not finite
 * makes the values of its group NaN.
 * group 32, 64 or 128; dim a multiple of 8 up to 256; block_size a multiple of
 * 16; arrays 16-byte aligned.
 */
typedef struct gba_q4_cache {
    gba_dtype dtype;
    int group;
    int64_t num_blocks, block_size, heads, dim;
    void *k_codes, *v_codes, *k_scales, *v_scales;
} gba_q4_cache;

/*
 * gba_q4_cache_store -- gba_cache_store into a gba_q4_cache: the rows k[t], v[t]
 * of every token t with a slot in the cache, rounded to 4 bits.  Of a group's
 * elements v with the ends low and high, in fp32 (fl) and the cache's type (r16),
 * to the nearest, ties to even:
 *     scale  = r16( fl( fl(high / 2 - low / 2) * fl(2 / 15) ) ), 0 if below 2^-100
 *     offset = r16( fl( low + 8 scale ) )
 *     code   = fl( fl(v - offset) * fl(1 / scale) ) to the nearest whole number,
 *              plus 8, at least 0 and at most 15; 8 if scale is 0
 * A group with an infinity or a NaN has scale 0 and offset NaN.  Slots as in
 * gba_cache_store: of two tokens with one slot, each word, and each pair of a
 * scale and an offset, is one or the other's.
 *
 * gba_q4_cache_load -- back: row t of k and v becomes scale (code - 8) + offset
 * of the elements at slots[t], rounded once, to no further than the type's
 * largest finite value, or zeros where the slot is not in the cache.
 *
 * Strides in elements; dim is contiguous in k and v.
 * Errors: GBA_EINVAL for cache == NULL, a bad enum or group, negative sizes,
 * block_size < 1, a NULL pointer that is read or written; GBA_EUNSUPPORTED for
 * other dims, block sizes or alignments, num_blocks * block_size or tokens above
 * 2^31-1, more than 65535 heads, or a launch of 2^32 threads or more (from 2^24
 * tokens on); GBA_EHIP if the launch fails.
 */
gba_status gba_q4_cache_store(const gba_q4_cache *cache, int64_t tokens, const void *k, int64_t k_token,
                              int64_t k_head, const void *v, int64_t v_token, int64_t v_head,
                              const int32_t *slots, gba_stream_t stream);
gba_status gba_q4_cache_load(const gba_q4_cache *cache, int64_t tokens, const int32_t *slots, void *k,
                             int64_t k_token, int64_t k_head, void *v, int64_t v_token, int64_t v_head,
                             gba_stream_t stream);

/*
 * gba_q4_attention -- one request of gba_q4_attend: that of gba_tree_attention
 * over a cache in 4 bits, with window 0, or of gba_window_attention.
 */
typedef struct gba_q4_attention {
    gba_q4_cache cache;
    int64_t requests, width;      /* rows and row length of the block table */
    int64_t tokens;               /* rows of q, out and mask */
    int64_t max_new;              /* no request has more new tokens than this */
    int64_t q_heads;              /* a multiple of cache.heads */
    int64_t window, sinks;        /* window 0: a token sees all of its text */
    float scale;
    const void *q;
    int64_t q_token, q_head;
    void *out;
    int64_t out_token, out_head;
    const int32_t *table;         /* [requests][width] */
    const int32_t *lens;          /* [requests]: cached tokens before the new ones */
    const int32_t *offsets;       /* [requests + 1]: rows of q of each request */
    const uint64_t *mask;         /* [tokens], or NULL */
    void *workspace;
    size_t workspace_bytes;
} gba_q4_attention;

/*
 * gba_q4_attend -- attention of each request's new tokens over a cache in 4
 * bits: the formula of gba_tree_attention, or with a window that of
 * gba_window_attention, for the values that the codes stand for.  Those are not
 * rounded.  The softmax weights, times the scales of V, are for the second
 * product: with fp16 as two bf16 numbers, 16 bits, and with bf16 as one, 8 bits.
 * Their own sum is of weights that are not rounded, in fp32.  What is said there
 * of positions that a token does not see, of missing blocks, rows of no request,
 * offsets and the workspace holds here too.  A row whose query is not finite is
 * NaN, and zeros if it sees no position.
 *
 * q and out 16-byte aligned with strides that are multiples of 8 (out: 4), but in
 * dimensions of one element.
 * Errors: those of gba_tree_attention and of gba_q4_cache_store, and GBA_EINVAL
 * for window < 0 or sinks < 0.
 */
gba_status gba_q4_attend(const gba_q4_attention *desc, gba_stream_t stream);
gba_status gba_q4_attend_workspace_size(const gba_q4_attention *desc, size_t *bytes);

/* Static, human-readable name of a status code. */
const char *gba_status_string(gba_status status);

/* Library version string, e.g. "gba 0.1.0 gfx950". */
const char *gba_version(void);

#ifdef __cplusplus
}
#endif

#endif /* GBA_H */
