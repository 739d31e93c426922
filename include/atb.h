/*
 * libatb -- BFP16 x BF16 GEMM with asymmetric tile buffering (ATB) for AMD
 * MI355X (gfx950), after "Can Asymmetric Tile Buffering Be Beneficial?"
 * (arXiv 2511.16041).
 *
 * C ABI.  Every pointer argument says whether it is HOST or DEVICE memory.
 * The caller owns every buffer; the library allocates host memory only (in
 * atb_gemm_create) and never device memory.  No function throws, aborts or
 * synchronises the device; every function that can fail returns an
 * atb_status.  Streams are hipStream_t values passed as void* (NULL = the
 * default stream).
 *
 * Operation (Sec. 1 and Sec. 3 of the paper):  C = A x B with A in R^{MxK},
 * B in R^{KxN}, C in R^{MxN}.  A is stored in BFP16 (Sec. 2.4: blocks of 8
 * values along K share one 8-bit exponent and keep an 8-bit mantissa each),
 * B and C are bf16, accumulation is fp32.  The kernel is output-stationary
 * (Sec. 3.1): each workgroup owns one T_MC x T_N tile of C for the whole
 * reduction; per K-step of T_K it keeps a T_K x T_N tile of B resident and
 * streams A through in sub-tiles of T_MA <= T_MC rows (rho = T_MC / T_MA
 * "kernel switches" per K-step, Sec. 5).  T_MA == T_MC is symmetric tiling.
 *
 * BFP16 values (the reading of Sec. 2.4 used throughout):
 *     a[i][k] = m[i][k] * 2^(E[i][k/8] - 133),  m int8 in [-127, 127],
 *     E uint8 = 127 + max over the block of floor(log2 |x|)  (0 for a zero block),
 *     m = clamp(round_to_nearest_even(x * 2^(133 - E)), -127, 127).
 *
 * Device layout of an A_bfp buffer for an M x K matrix (atb_bfp16_layout gives
 * the numbers): K is cut into panels of 64; inside a panel the rows follow
 * each other, so the part of a tile that one K-step needs is one contiguous
 * run of bytes (the GEMM fetches it with fully coalesced 16-byte requests).
 *     mantissa plane  int8  [panels][M][64]  at byte 0,
 *                     panels = ceil(K / 64); m[i][k] at (k/64) * M*64 + i*64 + k%64
 *     exponent plane  uint8 [panels][M][8]   at byte exp_off = round_up(panels * M * 64, 256);
 *                     E[i][k/8] at exp_off + (k/64) * M*8 + i*8 + (k%64)/8
 *     total bytes = round_up(exp_off + panels * M * 8, 256)
 *   Mantissa bytes with k >= K (the tail of the last panel) MUST be zero; the
 *   exponent bytes there are ignored.  9 bytes per 8 elements as in the
 *   paper's packed bfp16ebs8, but planar so that all loads are aligned.
 * B: bf16, row-major K x N, leading dimension N.  C: bf16, row-major M x N,
 * leading dimension N.  A_bfp, B and C must be 16-byte aligned.
 */
#ifndef ATB_H
#define ATB_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum atb_status {
    ATB_OK = 0,
    ATB_ERR_INVALID_ARG = 1, /* NULL pointer, non-positive size, K % 8 != 0, misaligned buffer */
    ATB_ERR_BAD_TILE = 2,    /* T_MC % T_MA != 0, or (T_MA,T_MC,T_K,T_N) is not a compiled instance */
    ATB_ERR_LDS_BUDGET = 3,  /* the tile's A and B buffers exceed the 160 KiB LDS of a CU */
    ATB_ERR_REG_BUDGET = 4,  /* the T_MC x T_N fp32 C tile exceeds the accumulator registers */
    ATB_ERR_HIP = 5,         /* a HIP call failed (no device, bad launch); see atb_last_hip_error */
    ATB_ERR_NOMEM = 6        /* host allocation failed */
} atb_status;

/* Static string for a status code. Never NULL. */
const char *atb_status_string(atb_status s);

/* hipError_t value of the most recent failing HIP call on this thread (0 if none). */
int atb_last_hip_error(void);

/* ------------------------------------------------------------------ GEMM */

typedef struct atb_gemm atb_gemm; /* opaque plan, HOST memory */

/* Plan C[M][N] = A_bfp[M][K] x B[K][N] with the tile factors of Sec. 3
 * (T_MA rows of A buffered per sub-tile, T_MC x T_N C tile, T_K reduction
 * step).  Touches no device.  Requirements: M, N, K >= 1, K % 8 == 0,
 * T_MC % T_MA == 0, and the factors must name a compiled instance (see
 * atb_instance_count / atb_instance_get).  M and N need not be multiples of
 * the tile (edge tiles are masked); K need not be a multiple of T_K.
 * Size limits (32-bit element offsets inside the kernel; ATB_ERR_INVALID_ARG
 * beyond them): M, N <= 2^23, K <= 2^24, every operand below 2^31 elements
 * (M * round_up(K, 64), K * N, M * N; also N * round_up(K, 64) and
 * M * round_up(N, 64) for the BFP16 forms of B and C), and
 * 2 * N * (T_K + 1) < 2^31.
 * Problems of few rows and a long reduction (K > 1024; M <= 64, or few enough rows and columns for one
 * small tile per CU; not all of them, atb_gemm_streams tells) on the instances (64, 64, 128, 128), (32, 64, 256, 64)
 * and (32, 32, 256, 64), and with b_format BF16_T on any, are run by a kernel of their own whose waves take turns along K
 * and share no tiles; the factors then only select it.
 * Two kinds of plan run on other factors than theirs, where those are faster (the same bits; atb_gemm_kernel tells which):
 * odd N on (64, 128, 64, 128) and (128, 128, 64, 128) with K >= 1024 and many tiles on (128, 128, 64, 256), and b_format BF16_T
 * with few tiles on (64, 64, 64, 64) or (64, 128, 64, 128).  To compare factors, compare plans of which that is not so.
 * Bits: a plan gives the same bits on every run.  Plans that do not stream -- all of them up to K = 1024 -- add the
 * products of an element of C in one fp32 chain, k ascending: the same operands give the same bits on every instance,
 * with B row-major or transposed, and a row of C does not depend on M.  Plans that stream add one chain per wave, in
 * wave order: they agree among each other where the kernel has as many threads (atb_gemm_launch_info), and differ
 * from the others in the last bits.
 * On success *out is a new plan, else *out = NULL.
 * Environment (read here, both optional): ATB_LOG=1 prints the plan to
 * stderr; ATB_GROUP_M=<tile rows, 1..65536> overrides the height of the
 * patch of C tiles that the workgroups resident on one XCD cover (the
 * order in which tiles are walked, a measurement aid: results are the same
 * for every value). */
atb_status atb_gemm_create(atb_gemm **out, int64_t M, int64_t N, int64_t K,
                           int T_MA, int T_MC, int T_K, int T_N);

/* Launch the planned GEMM on `hip_stream`; returns after the launch (async).
 * A_bfp: DEVICE, layout above, read-only.  B_bf16: DEVICE, K x N bf16,
 * read-only.  C_bf16: DEVICE, M x N bf16, fully overwritten.  Inputs must be
 * finite.  Reports launch-time errors only. */
atb_status atb_gemm_run(const atb_gemm *g, const void *A_bfp, const void *B_bf16,
                        void *C_bf16, void *hip_stream);

void atb_gemm_destroy(atb_gemm *g);

/* Storage formats of the B and C operands (Sec. 6.1 of the paper lists three
 * precision configurations; its Configs 2 and 3 store every operand as BFP16).
 * A is always BFP16; accumulation is always fp32 in the MFMA accumulators. */
typedef enum atb_format {
    ATB_FMT_BF16 = 0,
    ATB_FMT_BFP16 = 1,
    ATB_FMT_BF16_T = 2      /* B only: bf16, handed over transposed (see atb_gemm_create_fmt) */
} atb_format;

/* atb_gemm_create with a storage format per operand.  The plan is run with
 * atb_gemm_run, whose B and C pointers then mean:
 *   b_format BF16 : B, K x N bf16 row-major (as in atb_gemm_create).
 *   b_format BFP16: B^T, N x K, as a BFP16 buffer with the layout
 *                   atb_bfp16_layout(N, K), i.e. blocks of 8 along K (the
 *                   reduction dimension, as the format requires, Sec. 2.4)
 *                   with the K index contiguous; atb_bfp16_quantize of a
 *                   row-major N x K fp32 matrix produces it.
 *   b_format BF16_T: B^T, N x K bf16 row-major (leading dimension K, the K index
 *                   contiguous) -- the layout in which frameworks keep the weight of a
 *                   linear layer.  The kernel then reads its B fragments with plain
 *                   16-byte LDS reads instead of transposing ones (half the LDS read
 *                   instructions for B).  Same values, and (atb_gemm_create: bits) the
 *                   result bits of b_format BF16.  Needs c_format BF16, an instance
 *                   with T_K = 64 and a C tile of at least 128 x 256, and
 *                   2 * T_N * K < 2^31 (else ATB_ERR_BAD_TILE / ATB_ERR_INVALID_ARG).
 *   c_format BF16 : C, M x N bf16 row-major.
 *   c_format BFP16: C as a BFP16 buffer with the layout atb_bfp16_layout(M, N)
 *                   (blocks of 8 along N), quantised from the fp32
 *                   accumulators by the same rule as atb_bfp16_quantize;
 *                   the tail of the last panel (columns N .. 64 * panels - 1) is
 *                   written as zero, so the buffer is a valid operand as it is.
 * c_format BFP16 needs N % 8 == 0 (whole blocks; else ATB_ERR_INVALID_ARG);
 * formats other than (BF16, BF16) need an instance that carries the variants: all but (32, 256, 64, 256) and
 * (32, 256, 128, 256), whose four waves of 256 accumulator registers leave none for a second staging pipeline
 * (else ATB_ERR_BAD_TILE).  All else as atb_gemm_create. */
atb_status atb_gemm_create_fmt(atb_gemm **out, int64_t M, int64_t N, int64_t K,
                               int T_MA, int T_MC, int T_K, int T_N,
                               atb_format b_format, atb_format c_format);

/* Launch geometry of a plan, for benches and tests: number of C tiles the
 * launch walks, rounded up to a multiple of 8 (the grid of the large tiles is persistent: it has
 * min(that, workgroups resident on the chip) workgroups, each looping over its
 * tiles), threads per workgroup, static LDS bytes per workgroup (as with a bf16 B): of the kernel that atb_gemm_run
 * launches, which atb_gemm_kernel describes in full.  Any pointer may be NULL. */
atb_status atb_gemm_launch_info(const atb_gemm *g, int64_t *workgroups, int *threads, int *lds_bytes);

/* The kernel that atb_gemm_run launches for a plan, whose factors are not always the plan's (atb_gemm_create). */
typedef struct atb_kernel_info {
    int T_MA, T_MC, T_K, T_N; /* tile factors of the instance that runs; of a plan that streams T_MA = T_MC the rows and T_N
                                 the columns of a workgroup's tile of C, T_K the 64 of a panel */
    int streams;              /* as atb_gemm_streams */
    int threads;              /* per workgroup */
    int lds_bytes;            /* all the LDS that a workgroup occupies, static and dynamic */
    int64_t workgroups;       /* as atb_gemm_launch_info */
} atb_kernel_info;
atb_status atb_gemm_kernel(const atb_gemm *g, atb_kernel_info *out);

/* 1 if atb_gemm_run sends this plan to the kernel for few rows and a long reduction (see
 * atb_gemm_create), which has no tile buffers and no use for the plan's factors; else 0 (also g == NULL). */
int atb_gemm_streams(const atb_gemm *g);

/* The compiled (T_MA, T_MC, T_K, T_N) instances. */
int atb_instance_count(void);
atb_status atb_instance_get(int index, int *T_MA, int *T_MC, int *T_K, int *T_N);

/* ----------------------------------------------------------------- BFP16 */

typedef struct atb_bfp16_layout_t {
    int64_t panel_k;     /* K extent of a panel: 64 */
    int64_t panels;      /* ceil(K / 64) */
    int64_t man_stride;  /* bytes between panels of the mantissa plane: M * 64 */
    int64_t exp_stride;  /* bytes between panels of the exponent plane: M * 8 */
    int64_t exp_off;     /* byte offset of the exponent plane */
    int64_t bytes;       /* total size of the buffer */
} atb_bfp16_layout_t;

/* Layout of an A_bfp buffer for an M x K matrix (K % 8 == 0). */
atb_status atb_bfp16_layout(int64_t M, int64_t K, atb_bfp16_layout_t *out);

/* Total bytes of an A_bfp buffer; 0 on invalid arguments. */
size_t atb_bfp16_bytes(int64_t M, int64_t K);

/* Quantise A_f32_dev (DEVICE, fp32, M x K, row pitch lda elements, lda >= K,
 * 16-byte aligned rows: lda % 4 == 0) into A_bfp_dev (DEVICE, layout above,
 * atb_bfp16_bytes(M,K) bytes; padding is written as zero).  Async on
 * hip_stream.  Inputs must be finite.  Bit-exact against the definition
 * in the header comment (Sec. 2.4 reading). */
atb_status atb_bfp16_quantize(const float *A_f32_dev, int64_t lda, void *A_bfp_dev,
                              int64_t M, int64_t K, void *hip_stream);

/* Decode an A_bfp buffer to bf16 (DEVICE, M x K, leading dimension K); exact.
 * For inspection and tests; the GEMM decodes inside its own kernel. */
atb_status atb_bfp16_decode(const void *A_bfp_dev, void *A_bf16_dev, int64_t M, int64_t K,
                            void *hip_stream);

/* ------------------------------------- a feed-forward sublayer's operators
 *
 * What a transformer's feed-forward sublayer needs around its matrix products: layer norm, the gated block in bf16 with
 * its gradients, and the same block's products with 4-bit weights for few tokens.  All matrices are row-major, a row's
 * elements next to each other; ld* is the distance between rows in elements, at least a row's length.  Sums and
 * statistics are held in fp32, and a norm's are added in chains of at most 620, so that their error stays below 2^-14 of the sum
 * of the terms' sizes however many there are.  M == 0 (no tokens) is a valid call: gradients of parameters are then written as zero.
 * Non-finite inputs give what the formulas give (4-bit products: see atb_q4_matvec); they reach no row or column that does
 * not depend on them.  A call of more rows than a launch can take is several launches. */

typedef enum atb_type { ATB_TYPE_BF16 = 0, ATB_TYPE_F32 = 1 } atb_type;
typedef enum atb_activation {
    ATB_ACT_SILU = 0,      /* g / (1 + exp(-g)) */
    ATB_ACT_GELU = 1,      /* g (1 + erf(g / sqrt 2)) / 2, beside fp32's rounding to 2.2e-7; of its own size 1.6e-3 at g = -5, 1e-2 at -8 */
    ATB_ACT_GELU_TANH = 2, /* g (1 + tanh(sqrt(2 / pi) (g + 0.044715 g^3))) / 2 */
    ATB_ACT_NONE = 3       /* atb_linear only: g itself */
} atb_activation;

/* Layer norm of the M rows of x (D elements of `type`, DEVICE):
 *     mu = sum(x) / D,  r = 1 / sqrt(sum((x - mu)^2) / D + eps),  y = (x - mu) r weight + bias.
 * weight, bias: DEVICE, D elements of `param_type`, or NULL for 1 and 0.  y: DEVICE, type `type`; may be x itself.
 * mean, rstd: DEVICE, M floats each, or NULL: mu and r, which the backward pass takes.  1 <= D <= 2^24; every pointer
 * at least aligned to its elements.  Async on hip_stream. */
atb_status atb_layer_norm(const void *x, int64_t ldx, const void *weight, const void *bias, double eps, void *y, int64_t ldy,
                          float *mean, float *rstd, int64_t M, int64_t D, atb_type type, atb_type param_type, void *hip_stream);

/* Bytes of atb_layer_norm_backward's workspace (partial sums of the parameters' gradients); 0 on invalid arguments or M == 0. */
size_t atb_layer_norm_workspace(int64_t M, int64_t D);

/* Its backward pass: with xh = (x - mean) rstd and g = dy weight,
 *     dx = rstd (g - sum(g) / D - xh sum(g xh) / D),  dweight = sum over rows of dy xh,  dbias = sum over rows of dy.
 * dx: M rows of `type`; dweight, dbias: D elements of `param_type`, each may be NULL (not asked for; dx too).  workspace: DEVICE, 16-byte
 * aligned, needed where dweight or dbias is asked for.  The sums over rows are taken in an order that M and D alone
 * decide: the same inputs give the same bits. */
atb_status atb_layer_norm_backward(const void *dy, int64_t lddy, const void *x, int64_t ldx, const float *mean, const float *rstd,
                                   const void *weight, void *dx, int64_t lddx, void *dweight, void *dbias, void *workspace,
                                   int64_t M, int64_t D, atb_type type, atb_type param_type, void *hip_stream);

/* The gated block  y = (act(x Wg^T) o (x Wu^T)) Wd^T  of M tokens in bf16: x M x D, Wg and Wu F x D, Wd D x F (the
 * layout in which frameworks keep the weights of linear layers), y M x D.  Both first products, the activation and the
 * product are one kernel.  What is an operand of a further product is rounded to bf16, as the matrix instructions take it: h = act(x Wg^T) o (x Wu^T)
 * and, in the backward pass, dg and du.  With the result's own rounding y and the gradients are 2.4e-3 off in the 2-norm, where that
 * alone is 1.7e-3. */
typedef struct atb_ffn {
    const void *x, *w_gate, *w_up, *w_down;     /* DEVICE, bf16, 16-byte aligned */
    int64_t ldx, ld_gate, ld_up, ld_down;       /* multiples of 8, below 2^22 */
    int64_t M, D, F;                            /* 0 <= M <= 2^23; D, F multiples of 8, 8 .. 2^22 - 8 */
    atb_activation act;
    void *workspace;                            /* DEVICE, 16-byte aligned, of the bytes below for the call; NULL: long reductions of few tokens are not shared out */
} atb_ffn;

/* Bytes of the workspace of a forward pass (keeps != 0: one with `kept`) and of a backward pass, at most 64 MiB; 0: none is used, or invalid arguments. */
size_t atb_ffn_workspace(int64_t M, int64_t D, int64_t F, int keeps);
size_t atb_ffn_backward_workspace(int64_t M, int64_t D, int64_t F);

/* Bytes of the buffer that keeps x Wg^T and x Wu^T for the backward pass, 6 M F: three planes of M x F 16-bit words, the upper halves of
 * the two products in fp32 and the next byte of both (24 of their 32 bits: in bf16 they would double the variance of dx's error); 0 on
 * invalid arguments or M == 0. */
size_t atb_ffn_kept_bytes(int64_t M, int64_t F);

/* h: DEVICE, M x F bf16 (pitch F), the block's inner activations: workspace, and what the backward pass takes.  kept: DEVICE,
 * atb_ffn_kept_bytes(M, F) bytes, 16-byte aligned, or NULL: nothing is kept.  y: DEVICE, bf16, 16-byte aligned, pitch ldy (as ldx).
 * Async on hip_stream. */
atb_status atb_ffn_forward(const atb_ffn *f, void *h, void *kept, void *y, int64_t ldy, void *hip_stream);

/* Gradients of a loss with dy (M x D bf16, pitch lddy, as ldx): with g = x Wg^T, u = x Wu^T, dh = dy Wd,
 *     dg = dh o u o act'(g),  du = dh o act(g),
 *     dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x,  dWd = dy^T h.
 * h, kept: of the forward pass.  dgate, dup: DEVICE, M x F bf16 (pitch F), workspace: dg and du (rounded to bf16; dh is not).  dx: M x D,
 * pitch lddx (as ldx); dw_gate, dw_up: F x D, dw_down: D x F, contiguous, bf16; each of the four may be NULL: not asked for (dw_gate and
 * dw_up together).  All 16-byte aligned. */
atb_status atb_ffn_backward(const atb_ffn *f, const void *h, const void *kept, const void *dy, int64_t lddy, void *dgate, void *dup,
                            void *dx, int64_t lddx, void *dw_gate, void *dw_up, void *dw_down, void *hip_stream);

/* A weight of N outputs and K inputs in 4 bits: w[n][k] = s[n][k / group] (q[n][k] - z[n][k / group]), 0 <= q <= 15. */
typedef struct atb_q4 {
    const void *packed;    /* DEVICE, N x K/2 bytes: q[n][k] in the low half of byte k / 2 for even k, in the high half for odd k; 16-byte aligned */
    const void *scales;    /* DEVICE, N x K/group bf16 */
    const void *zeros;     /* DEVICE, N x K/group uint8 (0 .. 15), or NULL: 8 everywhere */
    int64_t N, K;          /* 1 <= N <= 2^24; K a multiple of group, at most 2^22 */
    int group;             /* 32, 64 or 128 */
} atb_q4;

/* Quantise W (DEVICE, N x K of `type`, pitch ldw) to 4 bits.  Without zero points (zeros == NULL) s = max|w| / 7 over the group, rounded to
 * bf16, and q = 8 + rint(w / s); with them s = (max(w, 0) - min(w, 0)) / 15 rounded, z = rint(-min(w, 0) / s) and q = z + rint(w / s); q and z are clamped to
 * 0 .. 15, and a group of zeros has s = 0 and q = z.  Inputs must be finite. */
atb_status atb_q4_quantize(const void *W, int64_t ldw, atb_type type, void *packed, void *scales, void *zeros,
                           int64_t N, int64_t K, int group, void *hip_stream);

/* The values that a 4-bit weight stands for: out, DEVICE, N x K of out_type (in fp32 exact, in bf16 rounded to nearest even). */
atb_status atb_q4_decode(const atb_q4 *w, void *out, atb_type out_type, void *hip_stream);

/* y = x W^T for few rows: x DEVICE, M x K bf16 (pitch ldx, a multiple of 8, at most 2^26; 16-byte aligned), y M x N of y_type (pitch ldy).  Any M up to 2^23
 * is right; weights are read once per 16 rows.  A row with an infinity in x, or whose sums pass fp32's range, is not finite, NaN also where the formula
 * has an infinity: (16 + q) x is summed and (16 + z) x taken off again.  Async on hip_stream. */
atb_status atb_q4_matvec(const atb_q4 *w, const void *x, int64_t ldx, void *y, int64_t ldy, atb_type y_type, int64_t M, void *hip_stream);

/* h = act(x Wg^T) o (x Wu^T) in one launch, h M x N bf16: Wg and Wu with the same N, K, group, both with or both without zero points. */
atb_status atb_q4_gated(const atb_q4 *w_gate, const atb_q4 *w_up, atb_activation act, const void *x, int64_t ldx, void *h, int64_t ldh,
                        int64_t M, void *hip_stream);

/* ------------------------- what a block has around its feed-forward sublayer
 *
 * A product with its epilogue and its gradients; norms on both sides of a residual sum, and theirs; a mixture of experts for few tokens.  As above: row-major matrices with pitches in elements, sums and statistics in fp32,
 * no atomics (the same inputs give the same bits), workspaces that the caller owns for the call, M == 0 a valid call, non-finite inputs as the formulas
 * give them and never outside the rows and columns that depend on them. */

/* y = act(x W^T + bias) + residual in bf16: x M x K, W N x K (the layout in which frameworks keep the weight of a linear layer). */
typedef struct atb_linear {
    const void *x, *w;                          /* DEVICE, bf16, 16-byte aligned */
    int64_t ldx, ldw;                           /* multiples of 8, below 2^22 */
    const void *bias;                           /* DEVICE, N elements of bias_type, or NULL */
    int64_t M, N, K;                            /* 0 <= M <= 2^23; N any, 1 .. 2^22 - 8; K a multiple of 8, 8 .. 2^22 - 8 */
    atb_activation act;                         /* ATB_ACT_NONE too */
    atb_type bias_type;
    void *workspace;                            /* DEVICE, 16-byte aligned, of the bytes below for the call; forward also NULL: long reductions of few rows are not shared out */
} atb_linear;

/* Bytes of the workspace of a forward pass and of a backward pass; 0: none is used, or invalid arguments.  Of a backward pass they
 * hold act'(z) o dy in bf16 (unless act is ATB_ACT_NONE and N a multiple of 8) and sums of it, or of products, in fp32. */
size_t atb_linear_workspace(int64_t M, int64_t N, int64_t K);
size_t atb_linear_backward_workspace(int64_t M, int64_t N, int64_t K, atb_activation act);

/* residual: DEVICE, M x N bf16 (pitch ldr), or NULL; may be y.  slope: DEVICE, M rows of round_up(N, 8) fp16, 16-byte aligned, of which N are written with act'(x W^T + bias)
 * for the backward pass, or NULL; with ATB_ACT_NONE there is none.  Beside fp32's errors it is off by 2^-11 of itself at most, or by 2^-25 where that is more: slopes below 2^-14 lose digits, and their part of the
 * gradients with them.  y: DEVICE, M x N bf16 (pitch ldy).  y and residual at any element.  Async on hip_stream. */
atb_status atb_linear_forward(const atb_linear *l, const void *residual, int64_t ldr, void *slope, void *y, int64_t ldy, void *hip_stream);

/* Gradients of a loss with dy (M x N bf16, pitch lddy): with dz = dy o act'(z), rounded to bf16 for the products,
 *     dx = dz W,  dW = dz^T x,  dbias = sum over rows of dz (not rounded);  the residual's gradient is dy itself.
 * slope: of the forward pass; NULL with ATB_ACT_NONE.  dy: at any element, but with ATB_ACT_NONE and N a multiple of 8 16-byte aligned with a pitch as ldx.  dx: M x K (pitch
 * lddx, as ldx), dw: N x K contiguous, both bf16 and 16-byte aligned; dbias: N elements of bias_type; each may be NULL: not asked for.  The values of l->bias are not read. */
atb_status atb_linear_backward(const atb_linear *l, const void *slope, const void *dy, int64_t lddy, void *dx, int64_t lddx, void *dw, void *dbias, void *hip_stream);

/* What lies between two blocks: the first one's result z is normed, gated and added to the residual stream x, and the sum is normed for the next one:
 *     r = scale x + gate o N1(z),  h = N2(r),
 * N a layer norm, (v - mu) / sqrt(sum((v - mu)^2) / D + eps) weight + bias, a root-mean-square norm, v / sqrt(sum(v^2) / D + eps) weight + bias, or nothing: N1(z) = z, no h. */
typedef enum atb_norm_kind { ATB_NORM_NONE = 0, ATB_NORM_RMS = 1, ATB_NORM_LAYER = 2 } atb_norm_kind;
typedef struct atb_norm {
    const void *weight, *bias;                  /* DEVICE, D elements of param_type, or NULL for 1 and 0 */
    double eps;                                 /* >= 0, finite in fp32 and 0 there only if it is 0 */
    atb_norm_kind kind;                         /* ATB_NORM_NONE: the rest is not looked at */
} atb_norm;
typedef struct atb_residual_norm {
    const void *x, *z;                          /* DEVICE, M x D of stream_type and of block_type, at any element */
    int64_t ldx, ldz;
    atb_norm post, pre;                         /* N1, N2 */
    const void *gate;                           /* DEVICE, groups x D of param_type, contiguous, or NULL for 1 */
    int64_t groups;                             /* 1 .. 65535, M a multiple: row i is gated by row i / (M / groups) of gate; 1 without a gate */
    double scale;                               /* finite in fp32 */
    int64_t M, D;                               /* 0 <= M <= 2^23, 1 <= D <= 2^24 */
    atb_type stream_type, block_type, param_type;       /* of x, r and their gradients; of z, h and theirs, not wider than the first; of gate, weights and biases */
} atb_residual_norm;

/* r: DEVICE, M x D of stream_type (pitch ldr); may be x.  h: M x D of block_type (pitch ldh), with a norm `pre`; may be z.  Both at any element.  h is the norm of the sum before it is
 * rounded to stream_type.  stats: DEVICE, 4 x M floats, what the backward pass takes of both norms, or NULL.  Async on hip_stream. */
atb_status atb_residual_norm_forward(const atb_residual_norm *p, void *r, int64_t ldr, void *h, int64_t ldh, float *stats, void *hip_stream);

/* Where the gradients go: dx M x D of stream_type, dz of block_type, the others as what they are gradients of; each may be NULL: not asked for. */
typedef struct atb_residual_norm_grads {
    void *dx, *dz;
    int64_t lddx, lddz;
    void *dgate, *dpost_weight, *dpost_bias, *dpre_weight, *dpre_bias;
} atb_residual_norm_grads;

/* Bytes of the workspace of a backward pass that one of the last five is asked of; 0 on invalid arguments. */
size_t atb_residual_norm_workspace(int64_t M, int64_t D, int64_t groups);

/* dr: DEVICE, M x D of stream_type (pitch lddr), the gradient of r by all that follows but h, or NULL for 0; dh: of block_type (pitch lddh), with a norm `pre`.  x and z as in the forward pass (r is
 * computed again: rounded to bf16 it would cost the gradients digits, and x is no longer to read).  stats: of the forward pass.  workspace: DEVICE, 16-byte aligned.  The sums over rows are taken in an order
 * that M, D and groups alone decide.  With t the whole gradient of r and v N1's normed row, dgate is summed as weight sum(t v) + bias sum(t), a term whose weight or bias is 0 left out: where t is infinite and both are not 0,
 * it may be NaN in place of an infinity. */
atb_status atb_residual_norm_backward(const atb_residual_norm *p, const float *stats, const void *dr, int64_t lddr, const void *dh, int64_t lddh,
                                      const atb_residual_norm_grads *grads, void *workspace, void *hip_stream);

/* A mixture of E experts, each a gated block, for few tokens: with l = x R^T, every token's k largest l (of equal ones the lowest expert), p = softmax(l) (renormalize != 0: of the chosen l alone),
 *     y = sum over the chosen experts e of p_e (act(x Wg_e^T) o (x Wu_e^T)) Wd_e^T,
 * weights in bf16 or all three in 4 bits.  l is summed in fp64, the products, p and the sum over the experts are fp32; the inner activations are rounded to bf16.  Only the chosen experts' weights are read, once for every 16 tokens
 * (32 where an expert has more than 12 on average; 4 bits: 16) that chose them.  A NaN among a token's l is behind all others, -infinity too, and its p as softmax gives it; 4-bit weights: see atb_q4_matvec. */
typedef struct atb_moe_weight {                 /* of all experts, one expert's rows after the other's, contiguous; DEVICE */
    const void *w;                              /* bf16, or codes as atb_q4's; 16-byte aligned */
    const void *scales, *zeros;                 /* 4 bits: as atb_q4's; all three weights with zero points or none */
} atb_moe_weight;
typedef struct atb_moe {
    const void *x, *router;                     /* DEVICE, bf16, 16-byte aligned: M x D, and E x D */
    int64_t ldx, ld_router;                     /* multiples of 8, below 2^22 */
    atb_moe_weight w_gate, w_up, w_down;        /* E x F x D, E x F x D, E x D x F */
    int64_t M, D, F;                            /* 0 <= M <= 64; D, F multiples of 8 (4 bits: of group), below 2^22 */
    int experts, top_k;                         /* 1 <= E <= 256, 1 <= k <= min(E, 16) */
    int group;                                  /* 0: bf16; 32, 64 or 128 */
    atb_activation act;
    int renormalize;
    void *workspace;                            /* DEVICE, 16-byte aligned, of the bytes below for the call */
} atb_moe;

/* Bytes of the workspace: the l, the plan of the call, the inner activations, partial sums; 0 on invalid arguments. */
size_t atb_moe_workspace(int64_t M, int64_t D, int64_t F, int experts, int top_k, int group);

/* y: DEVICE, M x D bf16 (pitch ldy), at any element.  chosen, p: DEVICE, M x k int32 and fp32, or NULL: the experts of every token from its largest l on, and their p.  Async on hip_stream. */
atb_status atb_moe_forward(const atb_moe *m, void *y, int64_t ldy, int32_t *chosen, float *p, void *hip_stream);

/* ------------------------------------------------- model and tile selector */

/* Machine constants of the paper's performance model (Secs. 3 and 5). */
typedef struct atb_hw_params {
    double peak_core_flops;   /* Perf_core^peak: one core (XDNA2) / one CU (MI355X), flop/s */
    int    n_core;            /* N_core */
    int    array_rows;        /* cores sharing a B tile: L2 tile is array_rows*T_MC x array_cols*T_N (Eq. 2) */
    int    array_cols;
    double bw_offchip;        /* BW_offchip, byte/s */
    double buffer_bytes;      /* S of Eq. (1): L1 (XDNA2) or LDS (MI355X) per core */
    double acc_bytes;         /* MI355X only: accumulator-register bytes per core; 0 = C lives in `buffer_bytes` */
    double clock_hz;
    double delta_cycles;      /* delta: cost of one microkernel switch (Sec. 5) */
    double fill_cycles;       /* MI355X extension, 0 on XDNA2: pipeline-fill cost per K-step that an A sub-tile of
                                 T_MC rows exposes; a sub-tile of T_MC/rho rows exposes fill_cycles/rho (see atb_model_eval) */
    double eta, eps, II;      /* Eff_micro(T_K) = eta T_K / (eps + eta II T_K), Eq. (12) */
    double a_bytes, b_bytes, c_bytes; /* bytes per element of A, B, C moved from off-chip */
    double a_buf_bytes, b_buf_bytes;  /* bytes per element of A, B as buffered (Eq. 1); 0 = same as above */
    int    n_b_buffers;       /* B buffers in Eq. (1): the paper uses 2 */
} atb_hw_params;

/* Fill *hw with the paper's XDNA2 constants (Secs. 2.4, 3.2, 5; precision
 * Config 1 byte costs) or with this library's MI355X constants. */
void atb_hw_params_xdna2(atb_hw_params *hw);
void atb_hw_params_mi355x(atb_hw_params *hw);

typedef struct atb_choice {
    int T_MA, T_MC, T_K, T_N;
    int rho;               /* T_MC / T_MA */
    int feasible;          /* buffer (and accumulator) constraints hold */
    double ai;             /* AI_array, Eq. (2)  [flop/byte] */
    double ai_core;        /* AI_rho, Sec. 3.1 */
    double buffer_bytes;   /* left side of Eq. (1) (C term dropped when acc_bytes > 0) */
    double acc_bytes;      /* 4 * T_MC * T_N when acc_bytes > 0 in hw, else 0 */
    double eff_micro;      /* Eq. (12) */
    double eff_core;       /* Eq. (15) */
    double mem_bound;      /* AI_array * BW_offchip, flop/s */
    double compute_bound;  /* Eff_core * Perf_core^peak * N_core, flop/s */
    double pred_flops;     /* Eq. (11): min of the two */
} atb_choice;

/* Evaluate the model (Eqs. 1, 2, 11, 12, 15) for one set of tile factors.
 * hw == NULL means MI355X.  Pure host arithmetic.  Per output tile and K-step
 * the time is  2 T_MC T_N T_K / (Peak_core Eff_micro) + delta rho + fill / rho  (Eq. 14 plus the
 * fill term; with fill_cycles = 0 this is the paper's Eq. 14 / Eq. 15 exactly). */
atb_status atb_model_eval(int64_t M, int64_t N, int64_t K, int T_MA, int T_MC, int T_K, int T_N,
                          const atb_hw_params *hw, atb_choice *out);

/* Rank the compiled instances for a problem by predicted throughput
 * (infeasible ones last): atb_model_eval's prediction, with the compute bound
 * scaled by the measured full-load factor an instance may carry, rounds of
 * tiles counted in workgroups resident per CU, partly filled rounds credited
 * with the clock the idle CUs leave, and a fixed launch cost.  Writes min(capacity, count) entries to `ranked`
 * (HOST) and the number of instances to *count.  ranked[0] is the pick. */
atb_status atb_select_tiles(int64_t M, int64_t N, int64_t K, const atb_hw_params *hw,
                            atb_choice *ranked, int capacity, int *count);

/* ------------------------------------------------- microkernel issue model */

/* Sec. 4 of the paper models its microkernel on a VLIW core: a prolog bounded
 * by load latency and load-unit throughput (Eq. 4), a steady state whose
 * initiation interval is the larger of the MAC pipeline constraint and the
 * load constraint (Eq. 5), an epilog (Eq. 8), and their sum per kernel call
 * (Eq. 9), overlapped when several accumulation clusters are in flight
 * (Eq. 10).  This is the same decomposition for one gfx950 CU, with unit costs
 * measured on MI355X (csrc/microbench/unit_costs.hip): per C tile and K-step,
 * in shader-clock cycles,
 *   mfma   = n_mfma * 32 / 4                    matrix pipes (32 cycles per unit of 32768 flop, 4 SIMDs)
 *   valu   = (n_mfma * 17 + n_decode * 6.5 + n_addr * 4) / 4
 *                                               VALU issue ports: an MFMA blocks its SIMD's port for
 *                                               17 of its 32 cycles; a decode instruction costs 6.5
 *   lds    = 4.7 n_b128_reads + 4.6 n_tr_reads + bytes_written / 76
 *   vmem   = bytes_requested / 64
 *   steady = max of the four / 0.85             (II; 0.85 = co-issue efficiency, one global constant)
 *   switch = (120 + 4.7 * first-band reads + 150) / waves per SIMD
 *                                               prolog (LDS latency, Eq. 4 form) + epilog (barrier)
 *   kstep  = steady + rho * switch              (Eq. 9; workgroups sharing a CU overlap, Eq. 10)
 * (n_mfma counts units of 32 x 32 x 16 = 32768 flop: one v_mfma_f32_32x32x16_bf16 or two
 * v_mfma_f32_16x16x32_bf16, which cost the same pipe and port cycles.)
 * mfma_util = mfma / kstep; the chip is power-limited under this kernel, the
 * measured clock follows c * mfma_util^-0.617 (capped at 2.4 GHz) with c = 1.339 GHz for
 * instances that multiply with the 32 x 32 x 16 form and 1.45 GHz for the 16 x 16 x 32
 * form, which draws less power per flop, and
 * pred_flops = flop per K-step * CUs / (kstep / clock).
 * Predicts the full-load throughput of the compiled instances within 15 %
 * from the tile factors and the wave grid alone (measured values: tests/measured/mi355x_instances.txt);
 * it does not see pipeline stalls of a particular schedule. */
typedef struct atb_micro_model {
    double n_mfma;         /* MFMA units (32768 flop) per C tile and K-step */
    double mfma_cycles, valu_cycles, lds_cycles, vmem_cycles;
    double steady_cycles;  /* II of one K-step */
    double switch_cycles;  /* prolog + epilog of one microkernel call */
    double kstep_cycles;
    double mfma_util;      /* predicted share of cycles the matrix pipes are busy */
    double clock_hz;       /* predicted shader clock under that load */
    double pred_flops;     /* whole chip, full load */
} atb_micro_model;

/* wave_m x wave_n: the wave grid of the workgroup (64-lane waves); wg_per_cu:
 * workgroups that share a CU; mfma_rows: 16 or 32, the form of the MFMA.
 * ATB_ERR_INVALID_ARG / ATB_ERR_BAD_TILE if the factors do not divide (32-row
 * bands per wave row, 32-column bands per wave column, T_K % 16). */
atb_status atb_model_microkernel(int T_MA, int T_MC, int T_K, int T_N, int wave_m, int wave_n,
                                 int wg_per_cu, int mfma_rows, atb_micro_model *out);

/* Wave grid, residency and MFMA form of compiled instance `index` (inputs of the call above;
 * any of the four pointers may be NULL). */
atb_status atb_instance_geometry(int index, int *wave_m, int *wave_n, int *wg_per_cu, int *mfma_rows);

/* ------------------------------------------------------- measurement aid */

/* An MFMA-only loop on register operands (no memory traffic, no LDS), for
 * benches that quote the GEMM against what the matrix pipes of this chip
 * sustain in practice as well as against the nominal peak (the nominal figure
 * assumes a clock the chip does not hold under full matrix load).  Not a step
 * of the GEMM.
 * Launches `workgroups` workgroups of 8 waves (two per SIMD, as the GEMM's
 * large tiles); each wave issues iters * 32 v_mfma_f32_32x32x16_bf16
 * (mfma_rows = 32) or iters * 64 v_mfma_f32_16x16x32_bf16 (mfma_rows = 16:
 * the same flop; the form the large GEMM tiles use, and the one that draws
 * less power) on
 * operands that rotate over four register sets; random_operands != 0 fills
 * them with pseudo-random bf16 (random sign and mantissa, exponents 2^-7 .. 2),
 * 0 with the constant 1.0 (which draws less power, hence a higher clock).
 * sink_dev: DEVICE, at least workgroups * 512 * 4 bytes, overwritten (keeps the
 * arithmetic alive).  clocks_dev: DEVICE or NULL; two uint64 written by the
 * first wave: the kernel's length in ticks of the shader-clock counter
 * (s_memtime; measured on MI355X: one tick per two shader cycles) and of the
 * constant-rate counter (s_memrealtime).
 * *flop (HOST, may be NULL) receives the floating-point operations of the
 * launch.  Async on hip_stream; workgroups in [1, 65536], iters in [1, 2^20],
 * mfma_rows 16 or 32 (anything else: ATB_ERR_INVALID_ARG). */
atb_status atb_mfma_probe(void *sink_dev, void *clocks_dev, int workgroups, int iters,
                          int random_operands, int mfma_rows, void *hip_stream, double *flop);

#ifdef __cplusplus
}
#endif
#endif /* ATB_H */
