/*
 * sp24 -- 2:4 fine-grained structured-sparse matrix multiply for NVIDIA B200 (sm_100a).
 *
 * C ABI of the library built from paper_2104_08378_b200/csrc.  The operations are the ones
 * "Accelerating Sparse Deep Neural Networks" (arXiv 2104.08378) defines:
 *
 *   - the 2:4 pattern: in every aligned group of four consecutive values along a row at
 *     least two are zero (Section 3, Section 3.1);
 *   - magnitude pruning: the two smallest-magnitude values of each group of four are removed
 *     (Section 4.1, step 2 of the workflow, Figure 5);
 *   - the compressed format: an R x C matrix is stored as R x C/2 kept values plus 2 bits of
 *     position metadata per kept value; a group with more than two zeros still stores two
 *     values (Section 3.1, Figure 1);
 *   - the sparse GEMM: sparse(M x K, stored M x K/2 + metadata) times dense(K x N) gives
 *     dense(M x N); B and C are dense (Section 3.2, Figure 2);
 *   - operand types FP16, BF16 (FP32 accumulate) and INT8 (INT32 accumulate) (Section 3.2,
 *     Table 1); dimensions are multiples of 16 for 16-bit and 32 for 8-bit types (Section 3.2).
 *
 * Conventions that hold for every entry point unless its comment says otherwise:
 *   - Every data pointer is a DEVICE pointer owned by the caller.  The library allocates no
 *     device memory and frees none.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the default stream).  Calls only
 *     enqueue work; they do not synchronise.
 *   - Argument errors are detected on the host, returned at once, and launch nothing.
 *   - Matrices are addressed as  element(i, j) = base[i * ld + j]  for ROW_MAJOR and
 *     base[j * ld + i] for COL_MAJOR; `ld` is in ELEMENTS.
 *   - A (the sparse operand) is always row-major with K contiguous, because the groups of
 *     four run along a row (Figure 1).
 *   - The device must be compute capability 10.0 (B200); anything else gives SP24_ERR_ARCH.
 *     There is no CPU fallback.
 */
#ifndef SP24_H_
#define SP24_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SP24_OK = 0,
  SP24_ERR_NULL = 1,        /* a required pointer is NULL                                  */
  SP24_ERR_DTYPE = 2,       /* dtype (or dtype combination) not supported by this call     */
  SP24_ERR_SHAPE = 3,       /* a dimension is negative or breaks the multiple-of rule      */
  SP24_ERR_STRIDE = 4,      /* a leading dimension is too small or not 16-byte granular    */
  SP24_ERR_ALIGN = 5,       /* a base pointer is not 16-byte aligned                       */
  SP24_ERR_UNSUPPORTED = 6, /* valid request outside what is built (e.g. int8 alpha != 1)  */
  SP24_ERR_WORKSPACE = 7,   /* workspace missing or smaller than sp24_gemm_workspace_bytes */
  SP24_ERR_CUDA = 8,        /* a CUDA runtime / driver call failed                         */
  SP24_ERR_TIMEOUT = 9,     /* a bounded device-side wait expired (see sp24_gemm_status)   */
  SP24_ERR_ARCH = 10        /* current device is not sm_100                                */
} sp24_status;

/* SP24_F32 as an OPERAND type selects the TF32 mode (Section 3.2, Table 1): FP32 storage, TF32
 * multiplication, FP32 accumulation, and the 1:2 pattern -- one kept value in every aligned
 * PAIR along K instead of two in every group of four.
 * SP24_E4M3 / SP24_E5M2 are the 8-bit floating-point encodings (1-4-3 without infinities, and
 * 1-5-2).  Table 1 of the paper has no 8-bit floating-point row (its hardware had none); they
 * use the 2:4 pattern and the format of the 8-bit integer row, with FP32 accumulation. */
typedef enum {
  SP24_F16 = 0, SP24_BF16 = 1, SP24_I8 = 2, SP24_F32 = 3, SP24_I32 = 4, SP24_E4M3 = 5, SP24_E5M2 = 6
} sp24_dtype;

/* Metadata layouts.
 * CANONICAL: row i occupies K/8 bytes starting at meta + i*K/8; group g of the row (columns
 *   4g..4g+3) owns bits 4g..4g+3 of that row's little-endian bit string; the nibble is
 *   p0 | (p1 << 2) with p0 < p1 the 0-based positions of the two kept values (Section 3.1:
 *   the example row with indices [[0,3],[1,2]] gives nibbles 0xC, 0x9, first byte 0x9C).
 * TCGEN05: the same nibbles permuted into the order the sm_100a sparse tensor-core
 *   instruction reads them from tensor memory, in 2048-byte blocks of 128 rows x 128 columns
 *   of A, rows padded to a multiple of 128 and K to a multiple of 256; padding nibbles are 0x4.
 *   This is the layout sp24_gemm consumes.
 * SP24_F32 (1:2 pattern): one nibble per PAIR, 0x4 if the first value of the pair is kept, 0xE if
 *   the second (the pair read as four 16-bit halves of which halves 0,1 or 2,3 survive).
 *   CANONICAL: K/4 bytes per row.  TCGEN05: the placement of the 16-bit types with a nibble
 *   standing for a pair: 2048-byte blocks of 128 rows x 64 columns, K padded to 128. */
typedef enum { SP24_META_CANONICAL = 0, SP24_META_TCGEN05 = 1 } sp24_meta_layout;

/* Which index of a matrix is contiguous in memory. */
typedef enum { SP24_ROW_MAJOR = 0, SP24_COL_MAJOR = 1 } sp24_order;

/* Human-readable name of a status code (static storage, never NULL). */
const char* sp24_status_string(sp24_status s);

/* Bytes of the kept-value array of an M x K matrix: M * (K/2) * sizeof(t)  (Figure 1:
 * R x C becomes R x C/2).  Returns 0 for an unsupported dtype or K % 4 != 0. */
size_t sp24_values_bytes(sp24_dtype t, int64_t M, int64_t K);

/* Bytes of the metadata of an M x K matrix.  CANONICAL: M*K/8 (2 bits per kept value,
 * Section 3.1, i.e. 12.5 % / 25 % of the kept values for 16-bit / 8-bit types).
 * TCGEN05: ceil(M/128) * ceil(K/256) * 4096.  Returns 0 for bad arguments. */
size_t sp24_meta_bytes(sp24_dtype t, int64_t M, int64_t K, sp24_meta_layout l);

/* Magnitude pruning to 2:4 (Section 4.1 step 2; pattern of Section 3).
 * For every row i < M and every aligned group of four columns 4g..4g+3 < K the two values of
 * largest magnitude are copied bit-for-bit to y, the other two positions receive +0.  Equal
 * magnitudes: the lower column index is kept.  Magnitude is |x| for I8 (so -128 ranks as
 * 128) and the bit pattern without its sign bit for F16/BF16/E4M3/E5M2 (denormals are not
 * flushed).
 *   t: SP24_F16, SP24_BF16, SP24_I8, SP24_E4M3 or SP24_E5M2.   M >= 0, K >= 0, K % 4 == 0.
 *      SP24_F32: the 1:2 pattern -- the larger magnitude of every aligned pair is kept, equal
 *      magnitudes keep the first (K % 8 == 0, 16-byte aligned pointers and rows required;
 *      the same holds for sp24_compress / sp24_decompress, whose vals are then M x K/2 FP32).
 *   x: device, M x K row-major, leading dimension ldx >= K (elements).
 *   y: device, same shape, leading dimension ldy >= K; may be the same buffer as x.
 * Fastest when x, y are 16-byte aligned and ldx*sizeof(t), ldy*sizeof(t), K*sizeof(t) are
 * multiples of 16; other cases take a scalar path with the same result. */
sp24_status sp24_prune(sp24_dtype t, int64_t M, int64_t K, const void* x, int64_t ldx,
                       void* y, int64_t ldy, void* stream);

/* Compression to kept values + metadata (Section 3.1, Figure 1).
 * Applies the selection rule of sp24_prune to x itself, so compress(x) == compress(prune(x))
 * and the call doubles as the fused prune+compress pass.  For group g of row i with kept
 * positions p0 < p1:  vals[i*ldv + 2g] = x[i, 4g+p0],  vals[i*ldv + 2g+1] = x[i, 4g+p1],
 * metadata nibble p0 | (p1<<2) stored as `l` says.  A group with fewer than two non-zeros is
 * completed with its lowest-index zeros (an all-zero group stores positions 0,1).
 *   vals: device, M x K/2 row-major, ldv >= K/2 (elements).
 *   meta: device, sp24_meta_bytes(t, M, K, l) bytes; for TCGEN05 the padding is written too.
 *   dropped_nonzeros: device counter or NULL.  If given, the number of non-kept positions
 *     holding a non-zero magnitude is ADDED to it (0 added iff x already was 2:4).
 * Requires K % 4 == 0 (K % 16 == 0 for the vectorised path). */
sp24_status sp24_compress(sp24_dtype t, int64_t M, int64_t K, const void* x, int64_t ldx,
                          void* vals, int64_t ldv, void* meta, sp24_meta_layout l,
                          unsigned long long* dropped_nonzeros, void* stream);

/* sp24_prune and sp24_compress in ONE pass over x (Section 4.1 step 2 followed by the storage
 * format of Section 3.1): y receives what sp24_prune(x) would write, vals / meta / dropped what
 * sp24_compress(x) would, bit for bit; x is read once instead of twice and the pruned matrix is
 * not re-read.  Arguments as for the two calls; y may be the same buffer as x.  Operands the
 * vectorised kernels cannot take (see sp24_prune) and the SP24_F32 1:2 pattern run as the two
 * separate passes. */
sp24_status sp24_prune_compress(sp24_dtype t, int64_t M, int64_t K, const void* x, int64_t ldx,
                                void* y, int64_t ldy, void* vals, int64_t ldv, void* meta,
                                sp24_meta_layout l, unsigned long long* dropped_nonzeros,
                                void* stream);

/* Inverse of sp24_compress (the metadata is what decodes the format, Section 3.1):
 * y is M x K row-major (ldy >= K) with y[i, 4g+p_t] = vals[i, 2g+t] and +0 elsewhere. */
sp24_status sp24_decompress(sp24_dtype t, int64_t M, int64_t K, const void* vals, int64_t ldv,
                            const void* meta, sp24_meta_layout l, void* y, int64_t ldy,
                            void* stream);

/* Problem description of D = alpha * op(A) * B + beta * C  (Section 3.2, Figure 2).
 *   ab_type: SP24_F16 or SP24_BF16 (FP32 accumulate), SP24_I8 (INT32 accumulate) or SP24_F32
 *            (TF32 mode, 1:2 pattern, FP32 accumulate; cd_type SP24_F32 only; inputs are used
 *            with their low 13 mantissa bits ignored) -- the operand/accumulator pairs of
 *            Table 1 (its FP16-accumulate row is sp24_gemm_f16acc).  SP24_E4M3 or SP24_E5M2
 *            (both operands the same type, FP32 accumulate) go beyond that table.
 *   cd_type: type of C and D.  F16/BF16 operands: SP24_F16, SP24_BF16 (ab_type's own) or
 *            SP24_F32.  I8 operands: SP24_I32.  E4M3/E5M2 operands: SP24_F16, SP24_BF16 or
 *            SP24_F32.
 *   M, N, K: K is the LOGICAL (uncompressed) reduction length.  M, N, K must be multiples of
 *            16 (16-bit types) or 32 (8-bit types) (Section 3.2); zero-sized problems return
 *            SP24_OK.
 *   lda:     leading dimension of the A-side value array: of vals (M x K/2) when
 *            a_is_dense == 0, of the dense M x K matrix when a_is_dense == 1.
 *   order_b: SP24_COL_MAJOR = K contiguous (B stored as N rows of K values: the
 *            [tokens, hidden] activation layout; ldb >= K), the faster order, or
 *            SP24_ROW_MAJOR = N contiguous (the K x N matrix stored row by row; ldb >= N).
 *   order_c / order_d: SP24_ROW_MAJOR (N contiguous; ldc, ldd >= N) or SP24_COL_MAJOR
 *            (M contiguous, the [tokens, out_features] layout; ldc, ldd >= M).  When C is
 *            used (beta != 0) it must have the same order as D.
 *   a_is_dense: 0 = 2:4 compressed A with TCGEN05 metadata (the sparse tensor-core path);
 *            1 = the dense variant on the same pipeline (`A` is M x K dense, `meta` unused).
 * All leading dimensions are in elements and, in bytes, multiples of 16. */
typedef struct {
  sp24_dtype ab_type, cd_type;
  int64_t M, N, K;
  int64_t lda, ldb, ldc, ldd;
  sp24_order order_b, order_c, order_d;
  int a_is_dense;
} sp24_gemm_desc;

/* Reports the tile shape sp24_gemm (and its variants) would use for this problem with beta = 0 on the
 * current device: CTAs per tile (1, or 2 = a pair working on one tile), columns per tile, 128-row
 * blocks per CTA.  The output tile is (128 * ctas * mblk) x block_n, or narrower where that spreads a
 * small problem over more SMs.  The choice may differ with C, and for sp24_conv3x3_nhwc, which has no
 * tiles of one CTA and two or three blocks.  Launches nothing. */
sp24_status sp24_gemm_plan(const sp24_gemm_desc* d, int* ctas, int* block_n, int* mblk);

/* Bytes of device workspace sp24_gemm needs for this problem (currently a fixed 256 bytes:
 * the device-side status record).  The workspace must be 16-byte aligned. */
size_t sp24_gemm_workspace_bytes(const sp24_gemm_desc* d);

/* The 2:4 sparse GEMM on the sparse tensor cores (Section 3.2, Figure 2):
 *   D[i,j] = alpha * sum_g sum_{t=0,1} vals[i,2g+t] * B[4g + p_t(i,g), j] + beta * C[i,j].
 *   alpha, beta: HOST pointers.  float for floating-point operands; int32_t for I8, where only
 *                alpha == 1 and beta in {0, 1} are built (else SP24_ERR_UNSUPPORTED).
 *   A:    device; vals (M x K/2) or dense A (M x K), row-major, 16-byte aligned.
 *   meta: device; TCGEN05-layout metadata of A (ignored when a_is_dense).
 *   B, C, D: device, 16-byte aligned.  C may be NULL iff beta == 0.  C may alias D.
 *   workspace: device, >= sp24_gemm_workspace_bytes(d), zero-filled before its first use.  The
 *              kernel records an expired wait there; see sp24_gemm_status.
 * Accumulation is FP32 (INT32) in hardware order; the result is rounded to cd_type once,
 * round-to-nearest-even.
 * The tile shape is chosen from the problem size (sp24_set_tile_override forces one).
 * The five tensor maps of a call are kept in a small per-thread host cache keyed by address,
 * shape and leading dimension, so repeated calls on the same buffers do not encode them again. */
sp24_status sp24_gemm(const sp24_gemm_desc* d, const void* alpha, const void* A,
                      const void* meta, const void* B, const void* beta, const void* C,
                      void* D, void* workspace, size_t workspace_bytes, void* stream);

/* The FP16-accumulation mode of Table 1 (FP16 operands, FP16 accumulator; Section 3.2): sp24_gemm
 * with the tensor cores adding the products into a binary16 accumulator instead of an FP32 one.
 *   d->ab_type must be SP24_F16; d->cd_type SP24_F16 or SP24_F32; everything else as for sp24_gemm
 *   (sparse or dense variant, both orders of B, C and D; alpha, beta and C are applied in FP32 to
 *   the widened accumulator).
 * Accuracy: the running sum is rounded to binary16 after every tensor-core instruction (32 values of
 * K for the sparse form, 16 for the dense one), so the error grows with K:
 * |err| <= (K/32 + 2) * 2^-10 * (|A|.|B|)_ij is the bound the tests use, against 2^-11 relative for
 * one final rounding with sp24_gemm.  On these tensor cores a binary16 accumulator occupies a full
 * 32-bit cell of tensor memory and the instruction rate is that of FP32 accumulation, so the mode
 * buys no speed here (measured; see the benchmark's other_configs): it exists for bit-compatibility
 * with deployments that used it. */
sp24_status sp24_gemm_f16acc(const sp24_gemm_desc* d, const void* alpha, const void* A,
                             const void* meta, const void* B, const void* beta, const void* C,
                             void* D, void* workspace, size_t workspace_bytes, void* stream);

/* INT8 sparse GEMM with a dequantising epilogue, for the deployment the paper describes in
 * Section 4.4 and Section 5.1: INT8 weights and activations, per-row scaling factors for the
 * weights of fully-connected layers and a per-tensor factor for the activations.
 *   D[i,j] = act( row_scale[i] * acc[i,j] + bias[i] ),   acc = INT32 result of the 2:4 product,
 * where row_scale[i] is the caller's product of the weight row's factor and the activation
 * tensor's factor, bias may be NULL (0) and act is the identity or max(., 0) (relu != 0).
 *   d->ab_type must be SP24_I8; d->cd_type: SP24_BF16, SP24_F16, SP24_F32, or SP24_I8.
 *   SP24_I8 output: q = round-to-nearest-even(D / out_scale) clamped to [-127, 127].
 *   row_scale, bias: device, M floats.  Everything is computed in FP32 in this order: acc to
 *   float, one fused multiply-add with scale and bias, the activation, one multiply by
 *   1/out_scale (rounded to float once on the host), the rounding.
 * Other arguments, layouts and the workspace are those of sp24_gemm (alpha, beta, C unused). */
sp24_status sp24_gemm_i8_dequant(const sp24_gemm_desc* d, const void* A, const void* meta,
                                 const void* B, const float* row_scale, const float* bias,
                                 int relu, float out_scale, void* D, void* workspace,
                                 size_t workspace_bytes, void* stream);

/* Activations of sp24_linear and the operators around it: the identity, max(z, 0) (NaN stays), z Phi(z) with the normal
 * distribution's Phi, z / (1 + exp(-z)), and the approximation of the second by tanh,
 * z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2.  Evaluated in FP32 with the special-function units' exponential and
 * reciprocal.  Of their value, where that is small too, the second loses at most 2^-19 + 1.25 z^2 2^-24 (z < 0), the others at most
 * 2^-20 + 2^-22 |v| with exp(v) the exponential in their 1 / (1 + exp(v)); beyond v = 87, and for the second below z = -13.2, they are 0. */
typedef enum {
  SP24_ACT_NONE = 0, SP24_ACT_RELU = 1, SP24_ACT_GELU = 2, SP24_ACT_SILU = 3, SP24_ACT_GELU_TANH = 4
} sp24_act;

/* (No counterpart in the paper.)  A linear layer in one call: the product with scales, bias, activation and residual in its
 * epilogue,
 *   z[i,j] = row_scale[i] * col_scale[j] * acc[i,j] + bias[i],   D[i,j] = act(z[i,j]) + residual[i,j],
 * acc = A * B as sp24_gemm accumulates it (FP32, INT32), everything after it in FP32 in the order written, D rounded once to
 * cd_type.
 *   row_scale, bias: device, M floats (a factor and an addend of each output feature), or NULL (1, 0).
 *   col_scale: device, N floats (a factor of each token, as sp24_rms_norm and sp24_gated_act give with their 8-bit results),
 *              or NULL (1); 8-bit operand types only.
 *   residual:  device, M x N of cd_type in D's order with leading dimension d->ldc, 16-byte aligned, or NULL.  May be D.
 *   pre:       device, receives z rounded to cd_type in D's order with leading dimension ld_pre (what the gradient of act
 *              needs, see sp24_act_backward), 16-byte aligned, or NULL.  Must not overlap D or the residual. */
typedef struct {
  const float* row_scale;
  const float* col_scale;
  const float* bias;
  sp24_act act;
  const void* residual;
  void* pre;
  int64_t ld_pre;
} sp24_linear_epilogue;

/*   d: as for sp24_gemm; cd_type: F16/BF16 operands: their own type or SP24_F32; I8, E4M3, E5M2 operands: SP24_F16, SP24_BF16
 *      or SP24_F32; F32 operands (TF32 mode): SP24_F32.  A, meta, B, D, workspace: as for sp24_gemm. */
sp24_status sp24_linear(const sp24_gemm_desc* d, const sp24_linear_epilogue* e, const void* A, const void* meta,
                        const void* B, void* D, void* workspace, size_t workspace_bytes, void* stream);

/* 3x3, stride-1, pad-1 convolution of an NHWC activation with 2:4-sparse weights as an implicit
 * GEMM (Section 4.2: a convolution's reduction dimension is C*R*S): the same kernel as sp24_gemm,
 * but the B operand is read straight from the activation by im2col-mode TMA loads instead of
 * from a materialised (Nb*H*W) x 9*Cin matrix.
 *   d:  as for sp24_gemm with N = Nb*H*W output pixels (pixel (n,h,w) is column (n*H+h)*W+w) and
 *       K = 9*Cin ordered (r, s, c), c fastest; d->M output channels; ldb ignored; order_b must
 *       be SP24_COL_MAJOR.  With order_d = SP24_COL_MAJOR the output is NHWC ([pixels, M]).
 *   x:  device, Nb x H x W x Cin, packed, 16-byte aligned, at least 128 KiB.
 *   Cin must be a multiple of 128 (16-bit types) or 256 (int8).
 *   A / meta / alpha / beta / C / D / workspace: as for sp24_gemm (a_is_dense selects the dense
 *   variant with A = Kout x 9*Cin). */
sp24_status sp24_conv3x3_nhwc(const sp24_gemm_desc* d, int64_t Nb, int64_t H, int64_t W, int64_t Cin,
                              const void* alpha, const void* A, const void* meta, const void* x,
                              const void* beta, const void* C, void* D, void* workspace,
                              size_t workspace_bytes, void* stream);

/* Reads the status record in `workspace` back to the host (synchronises `stream`) and returns
 * SP24_OK, or SP24_ERR_TIMEOUT if a bounded wait inside any GEMM kernel that used this workspace
 * since the last read expired (that kernel returned early and its D is incomplete).
 * The record is STICKY: `workspace` must be zero-filled once before its first use (e.g.
 * cudaMemsetAsync); the kernels never clear it, they only write the code of the first wait that
 * expired into word 0 and count expired waits in word 1.  One record therefore covers any number
 * of launches (a benchmark loop, the bands of sp24_pipeline_host): a timeout in any of them is
 * still there when this call reads it.  A reported timeout is cleared by this call (a memset on
 * `stream`), so that the next read concerns the launches that follow. */
sp24_status sp24_gemm_status(void* workspace, void* stream);

/* (No counterpart in the paper: a deployment variant of sp24_gemm.)
 * sp24_gemm for callers that cannot allocate device memory -- a process whose framework
 * allocator already owns all of the GPU's memory, so that cudaMalloc fails, or a serving loop
 * that cannot afford the device-wide synchronisation cudaMalloc implies.  The workspace
 * (status record) lives in a fixed 4096-byte device array inside the library, present on every
 * GPU that loads the library until the process exits; problems whose
 * sp24_gemm_workspace_bytes exceeds 4096 are refused with SP24_ERR_WORKSPACE.  Arguments and
 * results are those of sp24_gemm; inputs and outputs remain the caller's buffers.
 * The first call on each device looks up the array's device address (cudaGetSymbolAddress);
 * make that first call before any stream capture.  Nothing is allocated or freed.
 * All calls on a device share the array.  It starts zero-filled and nothing has to be cleared
 * between calls: the kernels only write into it when a bounded wait expires, and the record
 * then stays until sp24_gemm_static_ws_status reads it.  Two calls that overlap on the GPU
 * (different streams) share the one record, so a timeout cannot be attributed to one of them:
 * serialise such calls, or use sp24_gemm with a workspace per stream. */
sp24_status sp24_gemm_static_ws(const sp24_gemm_desc* d, const void* alpha, const void* A,
                                const void* meta, const void* B, const void* beta,
                                const void* C, void* D, void* stream);

/* (No counterpart in the paper.)  sp24_gemm_status for the array of sp24_gemm_static_ws on the
 * current device: synchronises `stream`, returns SP24_OK or SP24_ERR_TIMEOUT (and then clears
 * the record).  Allocates nothing. */
sp24_status sp24_gemm_static_ws_status(void* stream);

/* Benchmarking and test support (no counterpart in the paper): forces the tile shape of every
 * following sp24_gemm / sp24_gemm_i8_dequant / sp24_conv3x3_nhwc call in this process.
 *   ctas: 1 or 2 CTAs per tile; block_n: columns per tile; mblk: 128-row blocks per CTA (1 to 3);
 *   the shape must be one of the built ones, else those calls return SP24_ERR_UNSUPPORTED.
 *   (sp24_expert_linear and sp24_expert_linear_dx: ctas 1 and up to 128 columns, or 2 and up to 224, dense 256, whole 32; mblk 1.)
 *   ctas == 0 restores the automatic choice.  band: m-tiles per band of the tile sweep, 0 = default.
 * The environment variables SP24_TILE=<ctas>x<block_n>x<mblk>, SP24_BAND=<band> and SP24_LOG=1
 * (print the problem and the chosen tile shape of every call to stderr) give the initial values;
 * they are read ONCE, at the first GEMM call of the process. */
sp24_status sp24_set_tile_override(int ctas, int block_n, int mblk, int band);

/* Test support for the failure path, not for production use: shortens the limit of every
 * device-side wait to `wait_cycles` SM cycles (values below 1 000 000 restore the default of
 * about a second) and, with skip_stage != 0, makes the TMA producers leave out one k-block of
 * their first tile so that a wait expires; 2 + r: where several CTAs share the k-blocks of a tile,
 * only that of rank r does, whose own waits then have four times the limit: the others' waits for
 * its sums are the first to expire.  Nothing faults or hangs: the kernel returns early
 * and sp24_gemm_status reports SP24_ERR_TIMEOUT.  Never read from the environment. */
sp24_status sp24_test_set_fault_hooks(long long wait_cycles, int skip_stage);

/* Lowering of a 3x3, stride-1, pad-1 NHWC convolution input to the GEMM's B operand
 * (Section 4.2: a convolution's reduction dimension is C*R*S).  Output is K-contiguous:
 *   out[((n*H + h)*W + w) * ldo + (r*3 + s)*C + c] = in[n, h+r-1, w+s-1, c]  (0 outside).
 *   t: SP24_F16, SP24_BF16, SP24_I8, SP24_E4M3 or SP24_E5M2.  C*sizeof(t) must be a multiple
 *   of 16; ldo >= 9*C. */
sp24_status sp24_im2col_nhwc_3x3(sp24_dtype t, int64_t Nb, int64_t H, int64_t W, int64_t C,
                                 const void* in, void* out, int64_t ldo, void* stream);

/* Figure of merit of a channel permutation (Section 4.1: permuting the columns of the weight
 * matrix before pruning so that large values are spread over the groups keeps more total
 * magnitude).  Adds to *result (device double) the sum of |x[i, perm[k]]| over the positions
 * that 2:4 pruning of the column-permuted matrix x'[:, k] = x[:, perm[k]] keeps.
 *   perm: device, K int32 column indices (a permutation of 0..K-1), or NULL for the identity.
 *   t: SP24_F16, SP24_BF16, SP24_I8;  K % 4 == 0;  ldx >= K.  Summation is in double; the
 *   order of the partial sums is not fixed. */
sp24_status sp24_kept_magnitude(sp24_dtype t, int64_t M, int64_t K, const void* x, int64_t ldx,
                                const int32_t* perm, double* result, void* stream);

/* Re-imposes a fixed 2:4 pattern on updated weights, as sparse retraining does (Section 4.1,
 * step 3: the pattern found in step 2 is kept while the weights train on):
 * y[i, k] = w[i, k] where the metadata of sp24_compress names k as kept, +0 elsewhere.
 *   meta / l: metadata of an M x K matrix in either layout.  K % 8 == 0; y may alias w. */
sp24_status sp24_apply_mask(sp24_dtype t, int64_t M, int64_t K, const void* w, int64_t ldw,
                            const void* meta, sp24_meta_layout l, void* y, int64_t ldy,
                            void* stream);

/* 2:4 along rows AND columns (Section 6: the pattern must also hold for the transposed weights
 * if the backward pass is to be accelerated).  Every aligned 4 x 4 block keeps exactly two
 * values per row and per column; of the 90 such patterns the one keeping the largest total
 * magnitude is taken (exhaustive search).  Score of a pattern: ((s0 + s1) + s2) + s3 with
 * s_i = |x[i, c]| + |x[i, c']| for the row's kept columns c < c', in FP32; patterns are numbered
 * lexicographically by their rows' kept pairs in the order 01, 02, 03, 12, 13, 23, and the
 * lowest-numbered pattern with the largest score wins.  M % 4 == 0, K % 4 == 0; y may alias x. */
sp24_status sp24_prune_2d(sp24_dtype t, int64_t M, int64_t K, const void* x, int64_t ldx,
                          void* y, int64_t ldy, void* stream);

/* (No counterpart in the paper: the operators that stand before, between and behind the sparse products of a
 * feed-forward layer, and make their 8-bit operands.)
 *
 * Root-mean-square norm of rows, with the residual's addition before it:
 *   h = x + residual, rounded to t (h = x without residual);
 *   n = h / sqrt(mean(h^2) + eps) * weight, in FP32 from h as rounded;
 *   y = n rounded to t (out_type == t), or 8-bit codes with a scale for each row (SP24_I8, SP24_E4M3, SP24_E5M2):
 *   scale[i] = max |n[i, .]| / L with L = 127, 448, 57344, y = n / scale[i] rounded to the nearest code (ties to even).
 *   A row of zeros, or of |h weight| all below 2^-110, has scale 0 and codes 0.  A row with a NaN or an infinity in h has scale NaN and
 *   codes 0 (SP24_I8) or NaN.
 *   The codes are computed as h weight (L / max |h weight|): a value next to a tie may go the other way than n divided by the rounded scale.
 * The codes and scales are what the products with 8-bit operands take (the scales as sp24_linear's col_scale).  A row's results
 *   depend on its values and on where it and its result lie modulo 16 bytes (the order of its sum), not on the other rows or their number.
 *   t: SP24_F16, SP24_BF16 or SP24_F32.  rows >= 0, 1 <= K <= 2^30; any leading dimensions >= K, any alignment that the
 *   types have; fastest where rows start at 16-byte boundaries.
 *   residual: rows x K of type t, or NULL.  h: where x + residual goes, or NULL; without residual it has to be NULL.
 *   weight: K values of weight_type (t or SP24_F32), or NULL for ones.
 *   scale: rows floats for 8-bit results, else ignored.  rstd: rows floats that receive 1 / sqrt(mean(h^2) + eps), or NULL.
 *   h and y may each be the same buffer, with the same leading dimension, as x or residual (y: if out_type == t), but not
 *   each other.  Else outputs overlap neither inputs nor each other.
 *   mean(h^2) is held in FP32: rows with values above about 10^19 overflow it and give zeros (scale 0). */
sp24_status sp24_rms_norm(sp24_dtype t, int64_t rows, int64_t K, const void* x, int64_t ldx, const void* residual,
                          int64_t ldr, const void* weight, sp24_dtype weight_type, float eps, void* h, int64_t ldh,
                          sp24_dtype out_type, void* y, int64_t ldy, float* scale, float* rstd, void* stream);

/* Gradient of sp24_rms_norm (out_type == t) from dy, the h it normalised (x without residual) and its rstd:
 *   v = dy * weight;  dx = rstd v - rstd^3 h mean(v h) + dh;  dweight[k] = sum over rows of dy h rstd.
 * dh (or NULL): the gradient that arrives at h itself along the residual stream.  With a residual, dx is the gradient of
 * both x and the residual.  Everything in FP32, dx rounded once to t.  dweight: K floats, or NULL if it is not wanted.
 *   dx may be the same buffer as dy, h or dh (same leading dimension).
 *   workspace: sp24_rms_norm_backward_workspace_bytes(rows, K) bytes (0 for NULL dweight), 16-byte aligned, contents of no
 *   matter before or after (a row of K floats for each of the current device's SMs at most).  The rows' sums are added in an order that rows, K and the device fix: the same call gives the same bits. */
size_t sp24_rms_norm_backward_workspace_bytes(int64_t rows, int64_t K);
sp24_status sp24_rms_norm_backward(sp24_dtype t, int64_t rows, int64_t K, const void* dy, int64_t lddy, const void* h,
                                   int64_t ldh, const void* weight, sp24_dtype weight_type, const float* rstd,
                                   const void* dh, int64_t lddh, void* dx, int64_t lddx, float* dweight, void* workspace,
                                   size_t workspace_bytes, void* stream);

/* Gated activation y = act(g) * u of rows (u == NULL: act(g) alone; with SP24_ACT_NONE then the rows themselves, quantised),
 * in FP32, rounded once to t or to 8-bit codes with a scale for each row, as sp24_rms_norm has them (a NaN or an infinity in
 * act(g) * u gives scale NaN).  g and u may be the two halves of one product's result (leading dimensions >= F, any
 * alignment that the types have).  y may be the same buffer as g or u (out_type == t, same leading dimension). */
sp24_status sp24_gated_act(sp24_dtype t, sp24_act act, int64_t rows, int64_t F, const void* g, int64_t ldg, const void* u,
                           int64_t ldu, sp24_dtype out_type, void* y, int64_t ldy, float* scale, void* stream);

/* Its gradient (out_type == t):  dg = dy * u * act'(g),  du = dy * act(g), in FP32, rounded once to t.  u and du are both
 * given or both NULL.  dg may be the same buffer as g, u or dy, du too, each with its leading dimension, but not both the
 * same. */
sp24_status sp24_gated_act_backward(sp24_dtype t, sp24_act act, int64_t rows, int64_t F, const void* dy, int64_t lddy,
                                    const void* g, int64_t ldg, const void* u, int64_t ldu, void* dg, int64_t lddg,
                                    void* du, int64_t lddu, void* stream);

/* Gradient of the activation of sp24_linear: dz = dy * act'(z), a rows x cols matrix in the order of dy and z (row-major
 * here: rows are tokens if the product's D was column-major, features if it was row-major), in FP32 and rounded once to t.
 *   dz, or NULL; dzt: dz transposed (cols x rows, leading dimension lddzt >= rows), or NULL.  The gradients of a layer's
 *   input and of its weights contract dz over different axes, and each product wants its own contiguous.
 *   dbias: the sums of dz before its rounding over the rows (sum_over_rows != 0: cols floats) or the columns (rows floats),
 *   in an order that the sizes fix, or NULL.  z is not read for SP24_ACT_NONE and may be NULL then.
 *   dz may be the same buffer as dy or z (same leading dimension).
 *   workspace: sp24_act_backward_workspace_bytes(...) bytes for dbias, 16-byte aligned, contents of no matter. */
size_t sp24_act_backward_workspace_bytes(int64_t rows, int64_t cols, int sum_over_rows);
sp24_status sp24_act_backward(sp24_dtype t, sp24_act act, int64_t rows, int64_t cols, const void* dy, int64_t lddy,
                              const void* z, int64_t ldz, void* dz, int64_t lddz, void* dzt, int64_t lddzt, float* dbias,
                              int sum_over_rows, void* workspace, size_t workspace_bytes, void* stream);

/* ---- experts ------------------------------------------------------------------------------------------------------------
 * (No counterpart in the paper: a feed-forward layer of E experts with 2:4-sparse weights, of which each token uses k.)  The
 * calls in the order of a layer: sp24_route chooses the experts of each token, sp24_expert_order gives every chosen slot (token,
 * number) a row so that the rows of an expert lie together, sp24_expert_gather brings the tokens' rows there, sp24_expert_linear
 * multiplies each expert's rows with its own weights, and sp24_expert_combine adds a token's rows up.  How many rows an expert
 * has is known on the device only; nothing is read back.
 *
 * Routing.  l = logits[t, .] as FP32; scores s = softmax(l) or 1 / (1 + exp(-l)).
 *   Choice: experts by l (bias == NULL) or by s + bias, the largest first, the lower index first among equal ones.  With
 *   groups > 1 (a divisor of E; group g is experts g E / groups and on) only experts of the top_groups best groups: by the
 *   largest of those values (SP24_GROUP_MAX) or by the sum of the two largest s + bias (SP24_GROUP_TOP2).  The values are
 *   compared as real numbers: computed in FP32, and in FP64 where two are too close to tell.
 *   weights[t, i] = scale * s of the i-th chosen, with renorm != 0 divided by the sum of the chosen s (their sum is then scale).
 *   A logit of -infinity or NaN, and a bias of -infinity or NaN, is never chosen; where that leaves fewer than k, the rest has
 *   experts -1 and weights 0 (a token without any: a padded batch).  A NaN among the logits makes the weights of what the token
 *   chooses NaN; so does +infinity with softmax, where under a bias or SP24_GROUP_TOP2 nothing is chosen.
 *   t: SP24_F16, SP24_BF16 or SP24_F32.  T >= 0 tokens, 1 <= E <= 1024, ld >= E, any alignment that the types have.
 *   1 <= k <= min(32, top_groups * E / groups), groups <= 32.  bias: E floats.  weights: T x k floats, experts: T x k int32. */
typedef enum { SP24_SCORE_SOFTMAX = 0, SP24_SCORE_SIGMOID = 1 } sp24_score;
typedef enum { SP24_GROUP_MAX = 0, SP24_GROUP_TOP2 = 1 } sp24_group_score;
sp24_status sp24_route(sp24_dtype t, int64_t T, int64_t E, const void* logits, int64_t ld, sp24_score score, const float* bias, int groups,
                       int top_groups, sp24_group_score group_score, int k, int renorm, float scale, float* weights, int32_t* experts, void* stream);

/* Gradient of sp24_route's weights with respect to the logits, the choice being fixed: from dweights (T x k floats), the logits and
 * the experts chosen.  g = scale * dweights of the chosen, u = s / sum of the chosen s:
 *   renorm: dl = u (g - sum u g) of the chosen experts (sigmoid: times 1 - s), 0 of the others;
 *   else softmax: dl = s (g - sum of the chosen s g), g = 0 of the others; sigmoid: dl = g s (1 - s) of the chosen, 0 of the others.
 * In FP32, rounded once to t.  A slot whose expert is negative or not below E counts for nothing; an expert that stands in two slots of a token
 * gets both slots' gradients.  dlogits may be the logits themselves (same leading dimension), else may not overlap them (SP24_ERR_UNSUPPORTED). */
sp24_status sp24_route_backward(sp24_dtype t, int64_t T, int64_t E, const float* dweights, const void* logits, int64_t ld, const int32_t* experts,
                                int k, sp24_score score, int renorm, float scale, void* dlogits, int64_t ldd, void* stream);

/* Order of `slots` = T k slots by their experts, stable: the slots of expert e get the rows offsets[e] and on, in their own order.
 *   offsets: E + 1 int32; every one a multiple of `align`, the last where all rows end.
 *   position: slots int32, the row of each slot, -1 if its expert is negative or not below E.
 *   source: sp24_expert_rows(slots, E, align) int32, the slot of each row, -1 for rows that have none: between the experts where
 *           align > 1, and behind the last.
 *   1 <= E <= 1024, 1 <= align <= 256, 0 <= slots, sp24_expert_rows(...) < 2^31.  align = 1 is for inference; the gradient of the products'
 *   weights wants 16. */
int64_t sp24_expert_rows(int64_t slots, int64_t E, int64_t align);  /* slots + (align - 1) min(E, slots), up to a multiple of align */
size_t sp24_expert_order_workspace_bytes(int64_t slots, int64_t E);  /* 16-byte aligned, contents of no matter; 0 for few slots */
sp24_status sp24_expert_order(int64_t slots, int64_t E, int64_t align, const int32_t* experts, int32_t* offsets, int32_t* position,
                              int32_t* source, void* workspace, size_t workspace_bytes, void* stream);

/* Rows in the experts' order: out[position[t, i], .] = x[t, .] for i < k; rows whose source is negative become zeros.  With scale (T floats), also
 * out_scale[position[t, i]] = scale[t], 0 for those.  Any type of 1, 2 or 4 bytes; T x K of them, out rows x K.  Positions that are negative or not
 * below `rows` are left out.  Fastest where rows start at 16-byte boundaries.  out and x may not overlap (SP24_ERR_UNSUPPORTED). */
sp24_status sp24_expert_gather(sp24_dtype t, int64_t T, int64_t K, const void* x, int64_t ldx, const float* scale, int k, const int32_t* position,
                               int64_t rows, const int32_t* source, void* out, int64_t ldo, float* out_scale, void* stream);

/* The tokens' sums: out[t, .] = sum over i < k of weights[t, i] y[position[t, i], .] (weights == NULL: ones) + residual[t, .], in FP32 in this order,
 * rounded once to t (SP24_F16, SP24_BF16 or SP24_F32).  Slots without a row count for nothing, whatever their weight.  With NULL weights it is the gradient of
 * sp24_expert_gather.  out may be the residual (same leading dimension), else it may overlap neither that nor y (SP24_ERR_UNSUPPORTED). */
sp24_status sp24_expert_combine(sp24_dtype t, int64_t T, int64_t K, int64_t rows, const void* y, int64_t ldy, int k, const int32_t* position,
                                const float* weights, const void* residual, int64_t ldr, void* out, int64_t ldo, void* stream);

/* Its gradients: dy[position[t, i], .] = weights[t, i] dout[t, .], rounded once; dweights[t, i] = sum over . of dout[t, .] y[position[t, i], .] in FP32 (0 of
 * slots without a row); rows of dy whose source is negative become zeros.  dy may be y (same leading dimension), else it may overlap neither that nor dout
 * (SP24_ERR_UNSUPPORTED). */
sp24_status sp24_expert_combine_backward(sp24_dtype t, int64_t T, int64_t K, int64_t rows, const void* dout, int64_t lddo, const void* y, int64_t ldy, int k,
                                         const int32_t* position, const int32_t* source, const float* weights, void* dy, int64_t lddy, float* dweights,
                                         void* stream);

/* sp24_linear of every expert's rows with its own weights, in one launch.  For rows r from offsets[e] to offsets[e + 1]:
 *   z[r, i] = row_scale[e, i] * col_scale[r] * sum_k A_e[i, k] X[r, k] + bias[e, i],   D[r, i] = act(z[r, i]) + residual[r, i],
 * with the arithmetic of sp24_linear.  Rows before offsets[0] and from offsets[E] on are neither used nor written.
 *   A: the experts' values one after the other: E M rows of K / 2 (dense: K) values, leading dimension lda.
 *   meta: E times sp24_meta_bytes(ab_type, M, K, SP24_META_TCGEN05) bytes, each expert's as sp24_compress gives it (not for dense A).
 *   X: rows x K (leading dimension ldx), D, residual, pre: rows x M of cd_type (ldd, ld_residual, ld_pre), 16-byte aligned with leading
 *      dimensions of whole 16 bytes.  residual may be D (same leading dimension); else D and pre may overlap neither each other nor A, X or the
 *      residual (SP24_ERR_UNSUPPORTED).
 *   row_scale, bias: E x M floats; col_scale: rows floats; each may be NULL (col_scale: 8-bit operand types only).
 *   offsets: device, E + 1 int32, 0 <= offsets[0] <= ... <= offsets[E] <= rows (values outside count as the nearest that are not).
 *   ab_type: SP24_F16, SP24_BF16, SP24_I8, SP24_E4M3 or SP24_E5M2, cd_type as for sp24_linear.  M and K are multiples of 16, with 8-bit operands of
 *   32; rows is any number.  1 <= E <= 1024, E M < 2^31.
 *   workspace: as for sp24_gemm (sp24_gemm_status tells of an expired wait). */
typedef struct {
  sp24_dtype ab_type, cd_type;
  int64_t E, M, K, rows;
  int64_t lda, ldx, ldd, ld_residual, ld_pre;
  int a_is_dense;
} sp24_expert_desc;
typedef struct {
  const float* row_scale;
  const float* col_scale;
  const float* bias;
  sp24_act act;
  const void* residual;
  void* pre;
} sp24_expert_epilogue;
sp24_status sp24_expert_linear(const sp24_expert_desc* d, const sp24_expert_epilogue* e, const void* A, const void* meta, const void* X,
                               const int32_t* offsets, void* D, void* workspace, size_t workspace_bytes, void* stream);

/* The products of its gradient, for F16 or BF16 operands: dX[r, .] = sum_i dz[r, i] W_e[i, .] and dW_e[i, .] = sum over the expert's rows of dz[r, i] X[r, .], each
 * rounded once to ab_type, with dense W (E M rows of K values, leading dimension d->lda).
 *   dz: rows x M (leading dimension d->ldd), X, dX: rows x K (ldx; only rows of experts are written), dW: E M x K (lda; an expert without rows gets zeros).
 *   sp24_expert_linear_dw: every offset is a multiple of 16 (sp24_expert_order with align = 16): the weights' gradients of an expert that is not so placed are NaN.
 *      meta (or NULL): the weights' metadata, as for sp24_expert_linear; the entries of dW that it does not name as kept are zeros.
 *   d->cd_type is ab_type; d->ld_residual, d->ld_pre and d->a_is_dense are not used.  dX and dW may overlap no operand (SP24_ERR_UNSUPPORTED).  Sizes, alignment and
 *   workspace as above.
 * sp24_expert_act_backward: what they and the bias's gradient are made of, dz[r, i] = dy[r, i] act'(z[r, i]) rounded to t, for all rows (rows x M, or NULL), and dbias[e, i]
 *   (E x M floats or NULL) = the sum of the expert's dz before their rounding, in an order that the offsets fix.  z may be NULL for SP24_ACT_NONE.  t: SP24_F16, SP24_BF16 or
 *   SP24_F32; any leading dimensions and alignment; dz may overlap neither input (SP24_ERR_UNSUPPORTED: the sums read both again).  workspace (for dbias):
 *   sp24_expert_act_backward_workspace_bytes(...) bytes, 16-byte aligned, contents of no matter. */
size_t sp24_expert_act_backward_workspace_bytes(int64_t E, int64_t M, int64_t rows);
sp24_status sp24_expert_act_backward(sp24_dtype t, sp24_act act, int64_t E, int64_t M, int64_t rows, const void* dy, int64_t lddy, const void* z, int64_t ldz,
                                     const int32_t* offsets, void* dz, int64_t lddz, float* dbias, void* workspace, size_t workspace_bytes,
                                     void* stream);
sp24_status sp24_expert_linear_dx(const sp24_expert_desc* d, const void* dz, const void* W, const int32_t* offsets, void* dX, void* workspace,
                                  size_t workspace_bytes, void* stream);
sp24_status sp24_expert_linear_dw(const sp24_expert_desc* d, const void* dz, const void* X, const int32_t* offsets, const void* meta, void* dW,
                                  void* workspace, size_t workspace_bytes, void* stream);

/* End-to-end convenience for callers whose data lives in HOST memory (pinned for speed):
 * copies dense A (M x K, row-major, packed), B (N rows of K, packed) and, if beta != 0, C
 * (M x N packed) to the device buffers the caller provides, runs sp24_compress (TCGEN05
 * layout) and sp24_gemm, and copies D (M x N packed) back.  All h_* are host pointers, all
 * d_* device pointers sized for the packed matrices (d_vals, d_meta as the size helpers
 * say).  Work is enqueued on `stream`; the caller synchronises.  For M >= 16384 the work runs
 * in up to eight row bands: each band's D is copied out on a second, library-owned stream
 * (created once per device; `stream` is made to wait for it before the call returns) while
 * the next band's A and C are copied in, so both directions of the host link are busy.  The status
 * record in `workspace` is sticky (see sp24_gemm_status), so it covers every band.  The call may be
 * made from several host threads at once (events are created per call). */
sp24_status sp24_pipeline_host(const sp24_gemm_desc* d, const void* alpha, const void* h_A,
                               const void* h_B, const void* beta, const void* h_C, void* h_D,
                               void* d_A, void* d_vals, void* d_meta, void* d_B, void* d_C,
                               void* d_D, void* workspace, size_t workspace_bytes,
                               void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SP24_H_ */
