/*
 * mdbf.h -- C ABI of the MI355X (gfx950) forward product for Multi-Envelope
 * Double Binary Factorization (MDBF).
 *
 * The format (paper Sec. 4.2, Eq. "me-dbf-basis"): a weight matrix W (m x n) is
 * replaced by
 *        What = U V,   U = SA o (A Q^T)  (m x k),   V = SB o (G B^T)  (k x n)
 * with shared sign bases SA in {+-1}^{m x k}, SB in {+-1}^{k x n} (SB is the
 * paper's S_b transposed), rank-l real envelope factors A (m x l), Q (k x l),
 * G (k x l), B (n x l), and `o` the Hadamard product.  In the paper's symbols
 * m = N, n = M, k = R.
 *
 * The operation (paper Sec. 3.2 "Inference", generalised through the per-factor
 * expansion of Eq. "me-dbf-expand"): for every token b
 *        Y[b,:] = What X[b,:]
 * evaluated as two envelope-scaled binary products,
 *        z = sum_s g^(s) o ( SB (b^(s) o x) ),    y = sum_t a^(t) o ( SA (q^(t) o z) ).
 *
 * Conventions
 *  - Every pointer named *_dev is DEVICE memory owned by the caller; the library
 *    never allocates, frees or keeps device memory.  Everything else is host memory.
 *  - All launches are asynchronous on `stream` (a hipStream_t passed as void*;
 *    NULL is the default stream).  No call synchronises or reads device memory on
 *    the host, so the forward calls can be captured into a HIP graph.
 *  - Every function returns 0 (MDBF_OK) or a negative mdbf_status; arguments are
 *    validated before the first HIP call, so bad arguments are reported on hosts
 *    without a GPU as well.
 *  - Device pointers must be 16-byte aligned.
 */
#ifndef MDBF_H
#define MDBF_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define MDBF_VERSION 100
#define MDBF_MAX_L 16          /* envelope rank supported: 1..16 (the paper sweeps l in {1,2,3,8,16}) */

typedef enum {
  MDBF_OK = 0,
  MDBF_EINVAL = -1,        /* null pointer, non-positive shape, l out of range, T < 1, bad leading dimension */
  MDBF_EALIGN = -2,        /* a device pointer is not 16-byte aligned */
  MDBF_EDTYPE = -3,        /* unknown dtype code */
  MDBF_EWORKSPACE = -4,    /* workspace / output buffer too small */
  MDBF_EUNSUPPORTED = -5,  /* valid request this build cannot serve */
  MDBF_EHIP = -6           /* a HIP call failed; mdbf_last_hip_error() gives the text */
} mdbf_status;

typedef enum { MDBF_F16 = 0, MDBF_BF16 = 1, MDBF_F32 = 2 } mdbf_dtype;

/* flags of mdbf_desc_t */
#define MDBF_FLAG_PRECISE 1u   /* fp32 vector arithmetic throughout (no fp16 staging, no matrix cores); slow */
#define MDBF_FLAG_ACCUMULATE 4u /* Y += What x instead of Y = What x: the terms of a residual stack
                                   What = sum_p What^(p) with independent sign bases (paper Sec. 3.2,
                                   "Residual Compensation", Eq. "dbf-residual-comp") are applied by one call each
                                   on the same Y; the additions happen in the precision of Y.  Two terms of
                                   one Y must not sit in the same plan: a plan's layers run in no defined order */
#define MDBF_FLAG_BLOCK_SCALED 2u /* take the block-scaled matrix-core variant wherever it applies (l = 8 or 16, fp16
                                     envelopes, T <= 16), also for launches too small to fill the device with it;
                                     without the flag the library picks the variant by launch size.  (A single call
                                     with one token runs its own kernel with the flag too) */
#define MDBF_FLAG_FP16_STAGED 8u  /* never take the block-scaled variant: the scaled activations are staged in fp16
                                     (a plan takes the block-scaled variant only if none of its layers carries
                                     this flag); excludes MDBF_FLAG_BLOCK_SCALED (MDBF_EINVAL) */

typedef struct {
  int32_t m, n, k, l;      /* What is m x n, inner rank k, envelope rank l */
  int32_t x_dtype;         /* dtype of X            (mdbf_dtype) */
  int32_t env_dtype;       /* dtype of A, Q, G, B   (mdbf_dtype) */
  int32_t y_dtype;         /* dtype of Y            (mdbf_dtype) */
  uint32_t flags;
} mdbf_desc_t;

/* Envelope factors, row-major with the l modes of one row contiguous (the paper's
 * A = [a^(1) ... a^(l)] stored as m rows of l values). */
typedef struct {
  const void* A_dev;  /* m x l */
  const void* Q_dev;  /* k x l */
  const void* G_dev;  /* k x l */
  const void* B_dev;  /* n x l */
} mdbf_env_t;

/* ---- storage accounting (host only) ------------------------------------------------
 * Bits per weight: bit-packed signs plus the real envelope entries over the m*n entries
 * replaced (paper Sec. 3.2, last sentence of "Inference", applied to the factors listed
 * under Eq. "me-dbf-basis"):  [ (m+n)k + env_bits*l*(m+n+2k) ] / (mn).
 * merge_inner != 0 (only with l == 1) counts q o g as one vector, the plain DBF count.
 * Returns a negative value on invalid arguments. */
double mdbf_bpw(int m, int n, int k, int l, int env_bits, int merge_inner);

/* Inner rank for a bits-per-weight budget (paper Sec. 5.1, "largest inner rank that meets
 * the budget").  multiple <= 1: the largest k with mdbf_bpw <= bpw.  multiple > 1: the real
 * solution of mdbf_bpw(k) = bpw rounded to the nearest multiple (word-aligned ranks).
 * Returns k >= 0, or a negative mdbf_status. */
int mdbf_rank_for_budget(int m, int n, int l, double bpw, int env_bits, int multiple);

/* ---- sign bit-packing ("bit-packed sign matrices", paper Sec. 1 and Sec. 3.2) -------------
 * A sign matrix S (rows x cols) is contracted along `cols` in the forward product: for SA
 * rows = m, cols = k; for SB rows = k, cols = n.  One bit per entry, bit 1 <=> -1, in a
 * device tile layout private to this library (16-row tiles, 128-column blocks, padding bits 0).
 * mdbf_packed_bytes: size in bytes of the packed blob (host only). */
int mdbf_packed_bytes(int rows, int cols, size_t* bytes_out);

/* signs_dev: rows x cols int8, row-major with leading dimension ld >= cols; an entry < 0
 * packs as -1, an entry >= 0 as +1 (sign(0) = +1, paper Sec. 2).  packed_dev must hold
 * mdbf_packed_bytes(rows, cols) bytes (packed_bytes is checked) and is fully overwritten. */
int mdbf_pack(const int8_t* signs_dev, int rows, int cols, int64_t ld,
              void* packed_dev, size_t packed_bytes, void* stream);

/* Inverse of mdbf_pack: writes +1 / -1 into signs_dev (rows x cols int8, leading dim ld). */
int mdbf_unpack(const void* packed_dev, int rows, int cols,
                int8_t* signs_dev, int64_t ld, void* stream);

/* Envelope factor with zero modes appended (offline, like mdbf_pack): out_dev (rows x l_to, row-major)
 * receives env_dev (rows x l, row-major, elements of `dtype`) in its first l columns and zeros in the rest.
 * A layer whose four envelope factors are padded this way and whose descriptor says l_to denotes the same
 * What (paper Eq. "me-dbf-basis": the added modes are zero terms of the rank-l sums); ranks 8 and 16 with fp16
 * envelopes are the ones the decode kernels of plans serve, where other ranks run the slower generic kernel.  Single
 * calls of any rank and type run matrix-core kernels, those of ranks 8 and 16 in fp16 the ones with vector loads.
 * l_to >= l, l_to <= MDBF_MAX_L; both pointers 16-byte aligned; the buffers must not overlap. */
int mdbf_pad_envelope(const void* env_dev, int rows, int l, int dtype, void* out_dev, int l_to, void* stream);

/* ---- forward product ------------------------------------------------------------------
 * Workspace bytes needed by mdbf_forward for up to T tokens (room for the inner vector z in fp32, for the scaled
 * activations, for the partial sums of few-token calls and for the fp16 copies of long ones).  Host arithmetic only: the
 * same value on every machine, and never less for a larger T: a buffer of the longest call's size serves every
 * shorter call with the same kernels and the same bits as one of its own.  (mdbf_forward also takes less where it can do
 * without partial sums and copies: with one token if the rank is not 8 or 16 or the envelopes are not fp16, and
 * with more tokens always.  Such a call runs slower kernels; up to 64 tokens its results differ in the last bits.) */
int mdbf_workspace_bytes(const mdbf_desc_t* desc, int T, size_t* bytes_out);

/* Y[b,:] = What X[b,:] for b < T.
 *   SA_packed_dev  packed SA (m x k),  SB_packed_dev  packed SB (k x n)
 *   X_dev  T x n row-major, leading dimension ldx >= n (elements of x_dtype)
 *   Y_dev  T x m row-major, leading dimension ldy >= m (elements of y_dtype); overwritten.  It may overlap X in any way
 *          (a call in place: all of X is read before anything of Y is stored), and nothing else that the call reads
 *   workspace_dev / workspace_bytes  caller-owned scratch, >= mdbf_workspace_bytes()
 * Default arithmetic: fp32 accumulation on the matrix cores; z kept in fp32 with one token.  A single one-token call
 * rebuilds the factors S_A o (A Q^T), S_B o (G B^T) piece by piece in fp32 and applies them to the unrounded activations
 * in fp32, in two launches (one for small layers, three where the second factor has few rows and a long contraction): what remains is the
 * rounding of fp32 sums, added in a fixed order, so repeated calls return the same bits.  Plans with one to three tokens do the same if their layers are of other ranks than 16, of mixed ones or
 * not of fp16 envelopes, unless they are large and the block-scaled variant serves them.  The other plans quantise the
 * l-way scaled activations (b^(s) o x and q^(t) o z) once --
 * to three fp6 limbs under a shared power-of-two scale per 32 values (about 13 bits; the block-scaled variant, taken by
 * large plans of rank 8 or 16 with fp16 envelopes), or to fp16 (small plans of rank 16, MDBF_FLAG_FP16_STAGED) -- and
 * contract them with the sign words.  Two tokens or more: the factors
 * S_A o (A Q^T), S_B o (G B^T) are rebuilt piece by piece in fp16 and applied as dense products to the
 * fp16-rounded activations (x and z; z is stored in fp16 between the two products).  Magnitudes above
 * 65504 in those fp16 quantities overflow.  A token's result is the same bits in every single call of 2 to 16 tokens
 * with the same layer and types, in every one of 17 to 64 and in every one of 65 and more (of 17 and more with fp16
 * envelopes of rank 8 or 16, n and k multiples of eight and 16-byte aligned rows of X); between these ranges it
 * differs in the last bits.  Plans of four tokens and more may return a NaN where a value beyond fp16 makes a single
 * call return an infinity.  An infinity among the envelopes leaves no finite output it reaches; whether those are
 * infinities or NaNs is not specified (its products with entries of either sign are added, in parts).
 * Range: the block-scaled and fp16-staged variants carry their own power-of-two exponents (per 32 values, per 1024
 * columns of a scaled-activation vector) and keep z in fp32; single one-token calls, and the plans named with them above,
 * work in fp32 throughout: they hold their accuracy wherever the inputs and results are representable.  The general
 * kernel (plans that mix envelope types, or up to three tokens with more, of ranks and types that the variants above do
 * not serve; plans and single one-token calls of those with MDBF_FLAG_FP16_STAGED; single ones whose workspace has no
 * room for partial sums) stages
 * b^(s) o x and q^(t) o z in plain fp16, divided by up to 8: magnitudes below about 5e-4 lose accuracy.  The
 * many-token variant needs the entries of A Q^T and
 * G B^T, the activations and z inside fp16's normal range (6e-5 .. 65504); What is unchanged when A is divided
 * and B multiplied by the same positive constant (likewise Q, G), so a layer can be rebalanced offline.
 * With MDBF_FLAG_PRECISE everything is fp32 vector arithmetic. */
int mdbf_forward(const mdbf_desc_t* desc,
                 const void* SA_packed_dev, const void* SB_packed_dev,
                 const mdbf_env_t* env,
                 const void* X_dev, int64_t ldx,
                 void* Y_dev, int64_t ldy, int T,
                 void* workspace_dev, size_t workspace_bytes, void* stream);

/* mdbf_forward without a workspace argument, for callers that cannot allocate device memory at all (code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc) and therefore have no
 * workspace to pass.  Same arguments and arithmetic as mdbf_forward with a workspace of mdbf_workspace_bytes(),
 * and the same results bit for bit (a call of 65 or more tokens whose fp16 copies do not fit loads its operands one by
 * one instead: slower); the scratch memory
 * (the inner vector z and the scaled activations) lives in a static device array of
 * MDBF_STATIC_SCRATCH_BYTES inside the library, which every GPU the library runs on holds until the process
 * ends.  The call allocates and frees nothing.  A request for which the least workspace mdbf_forward takes exceeds
 * MDBF_STATIC_SCRATCH_BYTES returns MDBF_EWORKSPACE (checked on the host, before any HIP call): every layer
 * shape up to 11008 x 11008 with k <= 8192 fits with T <= 16; the 2048-token prefill does not.
 * All calls on one GPU share that GPU's array: calls that overlap in time on one GPU (different streams,
 * or a captured graph replayed while another call runs) race on it; calls on one stream are ordered and safe.
 * The array keeps the last call's contents; no kernel depends on them.  The first call on a device looks up
 * the array's address (hipGetSymbolAddress): make it outside stream capture. */
#define MDBF_STATIC_SCRATCH_BYTES (16u << 20)
int mdbf_forward_static(const mdbf_desc_t* desc,
                        const void* SA_packed_dev, const void* SB_packed_dev,
                        const mdbf_env_t* env,
                        const void* X_dev, int64_t ldx,
                        void* Y_dev, int64_t ldy, int T, void* stream);

/* ---- many independent layers in one pair of launches -----------------------------------
 * One entry per layer; the same meaning as the arguments of mdbf_forward.  Serves sibling
 * projections and whole stacks of independent products with two kernel launches in total. */
typedef struct {
  mdbf_desc_t desc;
  const void* SA_packed_dev;
  const void* SB_packed_dev;
  mdbf_env_t env;
  const void* X_dev;
  int64_t ldx;
  void* Y_dev;
  int64_t ldy;
  int32_t T;
} mdbf_layer_t;

/* Sizes of the plan (a table the kernels read) and of the device workspace for `count` layers. */
int mdbf_batch_plan_bytes(int count, const mdbf_layer_t* layers, size_t* plan_bytes_out,
                          size_t* workspace_bytes_out);

/* Fills plan_host (plan_bytes from mdbf_batch_plan_bytes; any alignment) for the given layers and workspace
 * address.  The caller copies the plan verbatim to device memory (plan_dev, 16-byte aligned) before calling
 * mdbf_forward_batch and keeps plan_host alive: the host reads launch sizes from it. */
int mdbf_batch_plan_build(int count, const mdbf_layer_t* layers, void* workspace_dev,
                          size_t workspace_bytes, void* plan_host, size_t plan_bytes);

/* Runs all layers of a plan.  Asynchronous on `stream`, no allocation, no host-device copy. */
int mdbf_forward_batch(const void* plan_host, const void* plan_dev, size_t plan_bytes, void* stream);

/* Name of the product kernel a built plan runs for `stage` (1 = first factor, 2 = second factor): one of
 * "stage_mx_kernel" (block-scaled), "stage_fast_kernel" (fp16-staged), "stage_gemm_kernel" (many tokens),
 * "stage_generic_kernel", "stage_precise_kernel"; "" for an invalid plan or stage.  Host only; the string is
 * static.  For reports that must name the kernel they timed. */
const char* mdbf_batch_plan_kernel(const void* plan_host, size_t plan_bytes, int stage);

/* Kernel launches one mdbf_forward_batch of the plan issues (host only): 4 for the block-scaled and fp16-staged
 * kernels with a scale-in launch per factor, 3 when both factors run the block-scaled kernel (the first factor's
 * launch writes the second factor's activation records itself), 2 for the others; a negative status for an
 * invalid plan. */
int mdbf_batch_plan_launches(const void* plan_host, size_t plan_bytes);

/* Runs a part of a plan, for measuring its kernels one by one: `stages` and `kernels` are bit masks.
 * stages: 1 = first factor (x -> z), 2 = second factor (z -> y).  kernels: 1 = the scale-in kernel of the
 * stage (plans that have none skip it: also the second factor of a three-launch plan, whose records the first
 * factor's product kernel writes), 2 = the product kernel.  mdbf_forward_batch is (3, 3).  Results are
 * only meaningful if the caller preserves the order scale-in -> product, stage 1 -> stage 2. */
int mdbf_forward_batch_part(const void* plan_host, const void* plan_dev, size_t plan_bytes, int stages,
                            int kernels, void* stream);

/* Measurement aid: reads `bytes` bytes at src_dev once with plain 16-byte loads and folds them with XOR;
 * wave w of the launch stores the fold of the 32-bit words it read in sink_dev[w].  The launch has
 * sink_words waves (sink_words / 4 workgroups of 256 lanes; element i of the buffer, in 16-byte units, is
 * read by lane i mod (64 * sink_words)), so the XOR of sink_dev[0 .. sink_words) is the XOR of all 32-bit
 * words of the buffer.  Timed over a buffer far larger than the caches it gives the read bandwidth a kernel
 * can reach on this device, the yardstick next to the nominal HBM peak for the decode kernels (whose
 * work is streaming the packed signs of paper Sec. 3.2 once).
 * bytes: positive multiple of 16; sink_words: multiple of 4 in [4, 1 << 20]; pointers 16-byte aligned. */
int mdbf_stream_read(const void* src_dev, size_t bytes, uint32_t* sink_dev, int sink_words, void* stream);

/* ---- quantizer projection (offline) ----------------------------------------------------------
 * MSVID_l of a real matrix Z (paper Sec. 4.2, Eq. "msvid-def"): the sign mask S = sign(Z) (sign(0) = +1) and the
 * best rank-l approximation of |Z| in Frobenius norm, A Q^T = TSVD_l(|Z|), with the singular values split
 * evenly between A (rows x l) and Q (cols x l); S o (A Q^T) is the member of the format nearest to Z for the
 * mask S (Theorem 1, Eq. "Ustar"), at a distance of the tail of |Z|'s spectrum (Eq. "rankl-error").  This is
 * the projection the layer-wise optimisation applies to each factor (Eq. "admm-U-prox"); applied to a factor
 * U (N x R) it yields S_a, A, Q of the stored format, and to V (M x R) it yields S_b, B, G.
 * The truncated SVD is a block subspace iteration with b = mdbf_msvid_block(l) columns (l plus 8 to 15 of
 * oversampling) started from the caller's block X0 (cols x b, row-major, linearly independent columns: e.g.
 * seeded normal deviates; the library draws no random numbers) and ended by a Rayleigh-Ritz step; `iters`
 * (0 .. 64) is the number of passes (each is one product with |Z| and one with |Z|^T).  The result is the
 * exact TSVD_l once the iteration has converged: the error A Q^T leaves exceeds the optimum by a factor that
 * falls geometrically with iters at the rate of the gap between |Z|'s singular values l and b + 1.
 *   Z_dev      rows x cols, row-major fp32, leading dimension ld >= cols
 *   S_dev      rows x cols int8 (+1 / -1), row-major, ld = cols: the input mdbf_pack takes
 *   A_dev, Q_dev   rows x l and cols x l fp32, row-major (a column of A and that of Q: up to a sign they share);  sigma_dev  b Ritz values (fp32, descending; the first l
 *              are the singular values of A Q^T)
 *   workspace_dev  caller-owned, >= mdbf_msvid_workspace_bytes (partial sums of the products and the iteration's blocks;
 *              the size has room for a copy of Z too, which is not made any more)
 * Needs b <= min(rows, cols) (else MDBF_EUNSUPPORTED), 1 <= l <= MDBF_MAX_L, pointers 16-byte aligned.
 * A Z with a NaN or an infinity in it has no projection: S is still its mask (a NaN counts as +1), the entries of A
 * and Q are zeros or NaNs and those of sigma zeros or infinities, the same ones in every call.
 * Asynchronous on `stream`; no host synchronisation, no allocation; deterministic (fixed summation orders). */
int mdbf_msvid_block(int l);
int mdbf_msvid_workspace_bytes(int rows, int cols, int l, size_t* bytes_out);
int mdbf_msvid(const float* Z_dev, int rows, int cols, int64_t ld, int l, int iters, const float* X0_dev,
               int8_t* S_dev, float* A_dev, float* Q_dev, float* sigma_dev, void* workspace_dev,
               size_t workspace_bytes, void* stream);

/* ---- attention block of a serving step ---------------------------------------------------------
 * What stands between the q, k, v projections and the output projection of a decoder layer: the new tokens' places
 * in a cache in pages (mdbf_kv_slots), norm and rotation of queries and keys (mdbf_qk_norm_rope), keys and values into
 * the cache (the same launch, or mdbf_kv_append) and attention over it (mdbf_kv_attention).
 *
 * The cache of one layer is a pool of pages of page_size tokens.  A page holds for each kv head in turn
 *     key codes    page_size x head_dim / 2 bytes      value codes   the same
 *     key scales   page_size x head_dim / 32 bytes     value scales  the same
 * (token-major; mdbf_kv_page_bytes in all).  Codes are 4-bit floating point numbers e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and
 * their negatives), the even channel in the low half of a byte; a scale byte b per 32 channels stands for 2^(b - 127),
 * and 255 for NaN throughout the block.  The smallest scale is taken that leaves the block's largest magnitude at most 7 units
 * (it may round to 6: least error at 4 bits, 11 % of a normally distributed block's norm); values round to the nearest number, ties to
 * the even code.  A block with a NaN or an infinity in it becomes NaN.  dtype bounds the scales, to 2^-23 .. 2^13 (MDBF_F16) or
 * 2^-125 .. 2^125 (MDBF_BF16), so that every stored value is a number of that type: larger magnitudes saturate.
 * (Nothing here writes other scale bytes.  Where a pool holds them, those beyond the bound are read as NaN, and values of those below it may be
 * rounded to the type.)
 * 4.25 bits a channel.  A token's place is its slot, page * page_size + offset.
 *
 * Requests are described in device memory (integer arrays need the alignment of their elements only, so that they may be
 * parts of larger ones): block tables (requests x table_width int32, row stride table_ld; entry i is the page of the
 * request's tokens i * page_size ...), cu (requests + 1 int32: the first row of each request among the step's
 * new tokens) and lengths (tokens of each request with the new ones). */
typedef struct {
  int32_t pages;       /* pages of the pool */
  int32_t kv_heads;
  int32_t head_dim;    /* 64, 128 or 256 */
  int32_t page_size;   /* tokens per page: 16, 32, 64, 128 or 256 */
  int32_t dtype;       /* MDBF_F16 or MDBF_BF16 */
} mdbf_kv_t;

/* Bytes of one page; the pool is `pages` of them, one after the other (host only). */
int mdbf_kv_page_bytes(const mdbf_kv_t* kv, size_t* bytes_out);

/* Block tables and slot map of a step from request lengths.  Request r has cached[r] tokens and gets fresh[r] new ones
 * (0 is fine); the pages that it needs beyond its first ceil(cached / page_size) are taken from the free list in the order of requests,
 * free[taken], free[taken + 1], ..., and entered in its table.  Writes
 *   lengths (requests)    cached + fresh                 cu (requests + 1)   prefix sums of fresh
 *   slots, positions (T)  of every new token, requests one after the other; -1 in the entries behind the last
 *   taken_out             taken plus the pages used      status              0, or the sum of MDBF_KV_* below
 * If status is not 0 the step is refused as a whole: tables stay as they are, taken_out = taken, lengths = cached (0 where that is negative),
 * cu is 0, slots and positions are -1 throughout, so that launches behind it do nothing.  taken_out may be taken; no other
 * output may overlap an input.  One launch, two for long steps. */
#define MDBF_KV_BAD_LENGTH 1   /* a negative count, or a length beyond 2^31 - 1 */
#define MDBF_KV_BAD_WIDTH 2    /* a request needs more pages than its table's row has room for */
#define MDBF_KV_BAD_TOKENS 4   /* more new tokens than T */
#define MDBF_KV_NO_PAGES 8     /* more pages needed than the free list holds */
int mdbf_kv_slots(int requests, int page_size, const int32_t* cached_dev, const int32_t* fresh_dev, int32_t* table_dev,
                  int64_t table_ld, int table_width, const int32_t* free_dev, int free_count, const int32_t* taken_dev,
                  int T, int32_t* lengths_dev, int32_t* cu_dev, int64_t* slots_dev, int32_t* positions_dev,
                  int32_t* taken_out_dev, int32_t* status_dev, void* stream);

/* Writes the keys and values of T tokens to their slots.  k_dev, v_dev: T rows of kv_heads x head_dim, row strides ldk,
 * ldv >= kv_heads * head_dim, elements of x_dtype.  A slot outside the pool (-1: padding) is skipped; no two tokens of a call may
 * have the same one. */
int mdbf_kv_append(const mdbf_kv_t* kv, void* cache_dev, size_t cache_bytes, const void* k_dev, int64_t ldk,
                   const void* v_dev, int64_t ldv, int x_dtype, const int64_t* slots_dev, int T, void* stream);

/* The values that T slots hold, as rows like mdbf_kv_append's (elements of y_dtype; rounded only if it is the other of
 * the two 16-bit types).  A slot outside the pool reads as zeros. */
int mdbf_kv_read(const mdbf_kv_t* kv, const void* cache_dev, size_t cache_bytes, const int64_t* slots_dev, int T,
                 void* k_dev, int64_t ldk, void* v_dev, int64_t ldv, int y_dtype, void* stream);

#define MDBF_ROPE_INTERLEAVED 1u   /* rotated pairs are channels (2 i, 2 i + 1) instead of (i, i + rot_dim / 2) */
typedef struct {
  int32_t q_heads, kv_heads, head_dim;   /* head_dim 64, 128 or 256 */
  int32_t rot_dim;                       /* channels that are rotated, the first ones: a multiple of 16 up to head_dim; 0: none */
  int32_t rope_rows;                     /* positions that the table covers */
  int32_t x_dtype, y_dtype;              /* of q, k, v as they come; of q_out, k_out */
  uint32_t flags;
  float eps;
} mdbf_rope_t;

/* For every head of q and k: x / sqrt(mean(x^2) + eps) * weight (left out where the weight is null), then the rotation by the
 * token's position, (a, b) -> (a cos - b sin, b cos + a sin), in fp32 and rounded once.
 *   q_dev, k_dev     T rows of q_heads resp. kv_heads x head_dim, row strides ldq, ldk (any, at least the row)
 *   q_weight_dev, k_weight_dev   head_dim fp32, or null
 *   rope_dev         rope_rows x rot_dim fp32: a position's rot_dim / 2 cosines, then its sines
 *   positions_dev    T int32 (neither is read where rot_dim is 0).  Negative (padding): the token's rows become zeros and nothing is cached.  At or beyond rope_rows: the rotated
 *                    channels become NaN
 *   q_out_dev        row stride ldqo; k_out_dev likewise, or null if only the cache is wanted
 * Outputs may be the inputs themselves where strides and types agree.
 * With kv (else null, like the arguments behind it) the same launch writes k, rounded to y_dtype, and v_dev (T rows
 * of kv_heads x head_dim, of x_dtype) to the cache slots: the bytes are those of mdbf_kv_append on k_out and v. */
int mdbf_qk_norm_rope(const mdbf_rope_t* desc, const void* q_dev, int64_t ldq, const void* k_dev, int64_t ldk,
                      const float* q_weight_dev, const float* k_weight_dev, const float* rope_dev,
                      const int32_t* positions_dev, int T, void* q_out_dev, int64_t ldqo, void* k_out_dev, int64_t ldko,
                      const mdbf_kv_t* kv, void* cache_dev, size_t cache_bytes, const void* v_dev, int64_t ldv,
                      const int64_t* slots_dev, void* stream);

#define MDBF_ATTN_CAUSAL 1u   /* a token sees the ones up to its own position (the new tokens are the request's last);
                                 without it all of the request */
#define MDBF_ATTN_EXACT_QUERIES 2u   /* queries are not rounded, whatever a call runs: see there */
typedef struct {
  int32_t q_heads;      /* a multiple of kv_heads: query head h reads kv head h / (q_heads / kv_heads) */
  uint32_t flags;
  int32_t window;       /* > 0 (causal only): a token sees the last `window` tokens up to itself; 0: all */
  int32_t max_fresh;    /* most new tokens of a request, and ... */
  int32_t max_length;   /* ... the longest request: launch sizes go by them.  Larger ones in cu and lengths are served as well, slowly */
  float scale;          /* of the scores, usually head_dim^-1/2; not 0 */
} mdbf_attn_t;

/* out[t, h] = sum_j softmax_j(scale q[t, h] . k_j) v_j over the tokens j of t's request that it sees, whose keys and values
 * come from the cache (the new tokens' own too: append first).  q_dev, out_dev: T rows of q_heads x head_dim of the cache's
 * dtype, row strides ldq, ldo.  Rows behind the last request's are left as they are; a token that sees nothing gets zeros.
 * What a token does not see has no influence on its row, whatever the bytes there are; a page number outside the pool reads as NaN.
 * Lengths are cut to what the table's row covers, fresh counts to T.  Scores, running maxima and sums are fp32.  Rounded are the
 * softmax's numerators, once to the cache's dtype (fp16: no finer than 2^-31 of the largest), and, in calls with many new tokens, the queries (times scale), to
 * 1.07 * 2^-14 (bf16) or 2^-18 (fp16) of the largest of each 32 channels.  With MDBF_ATTN_EXACT_QUERIES they are not: for queries with channels far
 * beyond their neighbours' (some 30 times and more); such calls take up to 15 % longer.  Repeated calls return the same bits.
 * The workspace holds partial results where the work on long caches is cut among workgroups; it may be null where 0 bytes are needed.  Its size
 * (host arithmetic only) does not depend on requests and T, and never shrinks with max_fresh and max_length: a buffer for the largest
 * call serves all of the same heads. */
int mdbf_kv_attention_workspace_bytes(const mdbf_kv_t* kv, const mdbf_attn_t* attn, int requests, int T, size_t* bytes_out);
/* What a call of these sizes runs (host only): "few rows" (16 query rows of a kv head at a time) or "prompts" (128), then
 * ", shares" where the work is cut, ", n-th row tiles" where workgroups take the row tiles that there are instead of those that there may
 * be, and ", products first" where waves that feed products have priority; "" for what a call would refuse. */
const char* mdbf_kv_attention_kernel(const mdbf_kv_t* kv, const mdbf_attn_t* attn, int requests, int T);
int mdbf_kv_attention(const mdbf_kv_t* kv, const mdbf_attn_t* attn, const void* cache_dev, size_t cache_bytes,
                      const int32_t* table_dev, int64_t table_ld, int table_width, const int32_t* cu_dev,
                      const int32_t* lengths_dev, int requests, const void* q_dev, int64_t ldq, int T, void* out_dev,
                      int64_t ldo, void* workspace_dev, size_t workspace_bytes, void* stream);

/* ---- misc ----------------------------------------------------------------------------- */
const char* mdbf_strerror(int status);
const char* mdbf_last_hip_error(void);   /* text of the last failed HIP call on this thread, or "" */
int mdbf_version(void);

#ifdef __cplusplus
}
#endif
#endif /* MDBF_H */
