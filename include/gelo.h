/*
 * gelo.h - C ABI of the GELO obfuscated-projection library for AMD MI355X (gfx950).
 *
 * GELO (Section 3.2 "Core Algorithm" of the paper) offloads a projection H*W to
 * an untrusted accelerator without showing it H:
 *
 *   trusted side      A  <- fresh random invertible n x n matrix        (step 1.2)
 *                     U  =  A * [H ; S]                                 (eq. 1, eq. 8)
 *   accelerator       Y  =  U * W                                       (eq. 2)
 *   trusted side      Z  =  A^-1 * Y, shield rows dropped               (eq. 3)
 *
 * and Z == H*W (eq. 4).  S are k secret high-norm "shield" rows (Section 3.2.1,
 * Mitigation 2); A is orthogonal (A^-1 = A^T) or a general well-conditioned
 * matrix (Mitigation 1).  Both roles run on one GPU here; U and Y are always
 * materialised in device memory because they are the messages the accelerator
 * sees (Section 3.1, the observation set O_t).
 *
 * Conventions
 *  - Every matrix pointer is a DEVICE pointer owned by the caller, row-major,
 *    16-byte aligned, with a leading dimension (in elements) that is a multiple
 *    of 8.  d and p must be multiples of 8.  The library never frees or keeps
 *    caller memory.  gelo_ctx and gelo_mixing objects are library-owned.
 *  - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *    Work is enqueued asynchronously on it; argument errors are reported
 *    synchronously and enqueue nothing.
 *  - dtype GELO_F32: H, W, U, Y, Z are float; the order of a product's sums goes by its size, so a product and the
 *    same one in parts agree to rounding and not to the bit.  GELO_BF16: they are bfloat16
 *    (upper 16 bits of a float), products accumulate in float, A is generated
 *    in float and rounded once to bfloat16 for the two mixing products.
 *  - All calls return a gelo_status; gelo_last_error() gives a message for the
 *    last failing call on a context.  No exceptions, no aborts.
 *  - A context is not thread-safe.  Sampling uses context-owned workspace, so
 *    two gelo_sample_mixing calls on one context must not overlap in time on
 *    different streams; sampling may overlap mix/project/unmix of other batches.
 *  - Memory: a context owns a factorisation workspace, a pool of mixing objects and
 *    (for gelo_qkv_forward without caller U / Y) a chain workspace.  gelo_reserve
 *    sizes all three ahead of time; a per-batch call allocates only when it meets a
 *    shape that was not reserved (first use), and only then may it synchronise the
 *    device to replace a smaller buffer.  The per-batch calls make no host allocation.
 *  - The kernels clamp out-of-range rows and columns of a ragged last tile to valid
 *    addresses and multiply them by the zero padding of A; operand rows beyond the
 *    contraction length are replaced by zeros, so a NaN or Inf in the data reaches
 *    only the outputs that mathematically depend on it.
 */
#ifndef GELO_H
#define GELO_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct gelo_ctx gelo_ctx;        /* device, Philox key (seed), workspace, record of used batch ids */
typedef struct gelo_mixing gelo_mixing;  /* the trusted side's secrets for ONE batch: A, A^-1, shield directions */

typedef enum {
    GELO_OK = 0,
    GELO_EINVAL = 1,      /* null pointer, non-positive size, bad enum value */
    GELO_ESHAPE = 2,      /* sizes outside what the kernels support (see each call) */
    GELO_EDTYPE = 3,      /* dtype of the call and of the mixing object differ */
    GELO_EALIGN = 4,      /* pointer not 16-byte aligned or leading dimension / width not a multiple of 8 */
    GELO_ENOMEM = 5,      /* device or host allocation failed */
    GELO_ECOND = 6,       /* no draw with kappa_2(A) <= cond_max within max_attempts */
    GELO_ESINGULAR = 7,   /* zero pivot met while factorising A */
    GELO_EREUSE = 8,      /* batch id already used on this context, or mixing object already consumed */
    GELO_ESTATE = 9,      /* call out of order (unmix before mix) */
    GELO_EHIP = 10        /* HIP runtime error; text in gelo_last_error() */
} gelo_status;

typedef enum { GELO_F32 = 0, GELO_BF16 = 1 } gelo_dtype;

/* How A is drawn (Section 3.2 step 1.2; Section 3.2.1).
 *  ORTHOGONAL   A = Q diag(sign r_ii) from the Householder QR of a Philox Gaussian; A^-1 = A^T.
 *  GAUSSIAN     A = G/sqrt(n); redrawn until kappa_2(A) <= cond_max; A^-1 from its QR factors.
 *  CONDITIONED  A = Q + 0.25 G2/sqrt(n): dense, A^T A != I, kappa of a few; A^-1 from its QR factors up to 128 rows
 *               (exact to its rounding); beyond by Newton's iteration from Q^T on bf16 products whose last residual takes all bits of A:
 *               |I - A A^-1| / sqrt(n) (Frobenius) is 1.0e-7 at 129 rows, 1.9e-7 at 1024, 3.8e-7 at 4096, in either dtype.
 *  STRUCTURED   A = P_3 (B D_2 P_2)(B D_1 P_1)(B D_0 P_0): Philox-drawn row permutations P_r and sign
 *               flips D_r around B, the normalised Walsh-Hadamard transform on the row blocks of the
 *               binary expansion of n.  Orthogonal (A^-1 = A^T), never formed: mix and unmix apply it in
 *               O(n log n) per column and drawing it costs O(n^2 / 64) comparisons.  The "structured
 *               orthogonal transforms" the paper's Conclusion proposes for cheaper fresh mixing, in a
 *               construction of this library's own.  It leaks what every orthogonal A leaks
 *               (Section 3.2.1 eqs. 5-6: U^T U = H^T H, the spectrum of H H^T) and comes from a finite
 *               family, 4 permutations and 3 n sign bits; its resistance to the attacks of Section 4 has
 *               not been measured by anyone.  gelo_mixing_export builds the dense A for inspection.
 *  BLOCK_ORTHOGONAL  the mixed rows are cut into blocks of at most GELO_BLOCK_ROWS rows and each block is
 *               mixed by a dense orthogonal matrix of its own (the ORTHOGONAL construction on the block's own
 *               Philox Gaussian): rows [r0, r0 + rows) of U = A_i [H[d0 : d0 + dn]; S[s0 : s0 + sn]], where
 *               of the rows up to a cut r floor(k_shield r / n) are shield rows, so every block gets its
 *               share of them.  A^-1 = A^T.  Mixing costs O(n GELO_BLOCK_ROWS (d + p)) instead of
 *               O(n^2 (d + p)) and drawing it O(n GELO_BLOCK_ROWS^2): the other route to the cheaper fresh
 *               mixing the paper's Conclusion asks for.  What it gives up: rows mix only inside their block
 *               (a block's U^T U is the Gram matrix of ITS rows of [H; S], so the leak of eq. 5 is per block,
 *               244 rows at a time here instead of all n_data), which the paper does not analyse.
 *               gelo_mixing_export builds the dense n x n matrix that acts on the stacked [H; S].
 *  REFLECTOR_PRODUCT  A = H_0 H_1 ... H_{n-1} diag(sign beta_k): the Householder reflectors of the ORTHOGONAL
 *               construction, but reflector k is built from the raw entries G[k:, k] of the Philox Gaussian (it
 *               maps them to beta_k e_0) instead of from column k of a partly factorised matrix.  In the QR that
 *               column, given the earlier reflectors, is again a vector of independent Gaussians, so A has
 *               exactly the law of the ORTHOGONAL kind (Haar; Stewart 1980) - a dense orthogonal A with
 *               A^-1 = A^T, the same leakage statement - at half the arithmetic (4/3 n^3: only the product is
 *               formed) and without the chain of dependent panels: the cheaper generation of A that Section
 *               4.2 finds wanting for n > 2048.  A different matrix than ORTHOGONAL gives for the same ids. */
typedef enum { GELO_ORTHOGONAL = 0, GELO_GAUSSIAN = 1, GELO_CONDITIONED = 2, GELO_STRUCTURED = 3,
               GELO_BLOCK_ORTHOGONAL = 4, GELO_REFLECTOR_PRODUCT = 5 } gelo_kind;

/* Row-norm statistic of H that the shield rows are scaled by. */
typedef enum { GELO_NORM_MEDIAN = 0, GELO_NORM_MEAN = 1 } gelo_norm_stat;

#define GELO_MAX_N 5120        /* largest n = n_data + k_shield the factorisation kernels take */
#define GELO_MAX_ATTEMPTS 255  /* the attempt number is one byte of the Philox counter */
#define GELO_BATCH_WINDOW 4096 /* how far below the highest batch id used so far an unused id is still accepted */
#define GELO_STATIC_MAX_N 128  /* largest n gelo_qkv_forward_static takes (and one-launch batched draws) */
#define GELO_MAX_BATCH_DRAW 48 /* mixing objects one gelo_sample_mixing_batch call draws */
#define GELO_BLOCK_ROWS 256    /* mixed rows per block of a GELO_BLOCK_ORTHOGONAL A */
#define GELO_STATIC_SCRATCH_BYTES (16u << 20)   /* size of its static device buffer, held per GPU until the process ends */

/* Creates a context on HIP device `device` with Philox key `seed`.  `allow_batch_reuse` != 0
 * switches off the check that a batch id is used at most once (for tests and benchmarks that
 * replay a batch; production callers pass 0: A must never be reused, Section 3.2 step 1.2).
 * The check keeps no growing set: with h = 1 + the highest id used so far, an id is refused
 * (GELO_EREUSE) if it was used, if it lies below the floor (gelo_set_batch_floor), or if it lies
 * more than GELO_BATCH_WINDOW below h; ids at or above h are always new.  Callers that number their
 * batches upwards (layer by layer, step by step) never meet the window. */
gelo_status gelo_create(gelo_ctx** out, int device, uint64_t seed, int allow_batch_reuse);
/* Checkpoint / resume of "never reused": A is a pure function of (seed, batch id), so the whole state
 * of a context is its seed and the ids it has used.  gelo_get_batch_floor returns the smallest id f
 * such that no id >= f has been used; a context created later with the same seed and
 * gelo_set_batch_floor(ctx, f) refuses every id below f and so never derives an A a second time.
 * The floor only moves up (GELO_EINVAL otherwise). */
gelo_status gelo_set_batch_floor(gelo_ctx* ctx, uint64_t first_unused);
gelo_status gelo_get_batch_floor(const gelo_ctx* ctx, uint64_t* first_unused);
/* Sizes the context's device memory for batches of this shape before the first of them arrives:
 * the factorisation workspace (and the side-by-side attempt buffers of GELO_GAUSSIAN with this
 * max_attempts), `mixings` pooled mixing objects, and, if p > 0, the U / Y workspace of
 * gelo_qkv_forward.  May synchronise the device and allocate; the per-batch calls that follow
 * then do neither.  Arguments as in gelo_sample_mixing. */
gelo_status gelo_reserve(gelo_ctx* ctx, gelo_kind kind, gelo_dtype dtype, int n_data, int k_shield, int d, int p,
                         int max_attempts, int mixings);
gelo_status gelo_destroy(gelo_ctx* ctx);
/* Message of the last failing call on `ctx` ("" if none).  Owned by the context. */
const char* gelo_last_error(const gelo_ctx* ctx);
const char* gelo_status_string(gelo_status s);

/* Trusted side, Section 3.2 step 1.2.  Draws the secrets of batch `batch_id`: A (n x n,
 * n = n_data + k_shield), its inverse, and k_shield Gaussian shield directions of width d.
 * A pure function of (seed, batch_id, kind, n, k_shield, d) (GELO_BLOCK_ORTHOGONAL: its blocks depend on how n
 * splits into n_data and k_shield).  cond_max and max_attempts
 * (1..GELO_MAX_ATTEMPTS) are used by GELO_GAUSSIAN only: it factorises up to four consecutive
 * attempts side by side on streams of its own (n <= 1024; one at a time beyond), reads their
 * condition estimates back (the only host synchronisation in the library) and returns the first
 * acceptable attempt in order, so the result does not depend on how many ran at once.  The
 * estimate (20 Lanczos steps) approaches kappa_2 from below, within 0.5 % as measured; an attempt
 * is accepted only if 1.01 x estimate <= cond_max, so an accepted A meets the bound itself
 * ("generate and verify", Section 3.2.1) and a draw within 1 % below it may be redrawn.
 * n <= GELO_MAX_N (GELO_STRUCTURED keeps 4 columns of all n rows in one workgroup's LDS at least,
 * which allows more rows than that on this chip), n_data >= 1,
 * k_shield >= 0, d a multiple of 8.  *out is owned by the library: release it with
 * gelo_mixing_free (which recycles its device memory inside the context). */
gelo_status gelo_sample_mixing(gelo_ctx* ctx, gelo_kind kind, int n_data, int k_shield, int d,
                               gelo_dtype dtype, double cond_max, int max_attempts,
                               uint64_t batch_id, gelo_mixing** out, void* stream);

/* Trusted side, Section 3.2 step 1.2, many batches at once: `count` mixing objects (1..GELO_MAX_BATCH_DRAW) for
 * batch ids first_batch_id .. first_batch_id + count - 1, all of one shape.  A does not depend on the data, so
 * a decode step's worth, or the next few prefill batches, can be drawn ahead together.  GELO_ORTHOGONAL,
 * GELO_REFLECTOR_PRODUCT (always by the launches for larger n below), and
 * GELO_BLOCK_ORTHOGONAL (all full blocks of all objects share the launches of one batched factorisation).
 *  n <= GELO_STATIC_MAX_N  ONE launch draws all of them (at this size a fresh A per layer-step costs more in
 *                          launch latency than in work);
 *  larger n                up to 32 factorisations share every launch of the Householder QR, each in a workspace of its own (the
 *                          chain of panel factorisations leaves most of the chip idle when one matrix is factorised alone; side
 *                          by side the strips of all of them fill it); fewer where 32 workspaces would exceed 8 GiB (one takes
 *                          0.8 MB at 200 rows, 22 at 720, 119 at 2150, 405 at 4301) or the device does not have the memory.
 * Object i is what gelo_sample_mixing returns for its batch id, bit for bit.  out: HOST array of `count`
 * pointers; on an argument error nothing is drawn and no id is consumed. */
gelo_status gelo_sample_mixing_batch(gelo_ctx* ctx, gelo_kind kind, int n_data, int k_shield, int d, gelo_dtype dtype,
                                     uint64_t first_batch_id, int count, gelo_mixing** out, void* stream);

/* Trusted side, eq. 1 / eqs. 7-8.  Shield rows S_i = g_i * shield_scale * m(H) / ||g_i||, m the
 * median or mean row 2-norm of H; then U[n x d] = A * [H ; S].  H: n_data x d (ldh), U: n x d (ldu),
 * both of type `dtype`, which must be the one the mixing object was drawn for (GELO_EDTYPE otherwise:
 * the kernels would read and write the buffers with the wrong element size).  The row counts are the
 * mixing object's (gelo_mixing_info); the caller's buffers must hold them. */
gelo_status gelo_mix(gelo_ctx* ctx, gelo_mixing* mixing, gelo_dtype dtype, const void* H, int64_t ldh,
                     float shield_scale, gelo_norm_stat stat, void* U, int64_t ldu, void* stream);

/* Accelerator side, eq. 2.  Y[n x p] = U[n x d] * W[d x p].  Touches no secret: it takes no
 * mixing object.  Also serves as the plain baseline H*W (pass H as U, n = n_data).  A bf16 product
 * of at most 96 rows whose width leaves most of the chip idle (p < 8192) cuts a long d over workgroups and
 * keeps their float partial sums in a context workspace (gelo_reserve with p sizes it): two such
 * calls on one context must not overlap in time on different streams. */
gelo_status gelo_project(gelo_ctx* ctx, gelo_dtype dtype, int n, int d, int p,
                         const void* U, int64_t ldu, const void* W, int64_t ldw,
                         void* Y, int64_t ldy, void* stream);

/* Accelerator side, eq. 2 with both operands stored as 8-bit floats (OCP FP8 E4M3, the "FP8 / INT8 quantized
 * numerics" of the paper's Conclusion): twice the matrix rate of the bf16 projection.  The weight is public and
 * static, so it is prepared once: gelo_prepare_weight_fp8 writes into the caller's DEVICE buffer Wq
 * (gelo_fp8_weight_bytes(d, p) bytes, 16-byte aligned) the codes of W^T (p x d bytes: code of
 * W[k][j] * 448 / max_k |W[k][j]| at byte j d + k, round to nearest even, saturating at 448), padded to a
 * multiple of 256 bytes, then the p column scales max_k |W[k][j]| / 448 as floats.  gelo_project_fp8 quantises
 * U (bf16, n x d) per row the same way into context workspace (allocated on first use of a size), multiplies
 * on the matrix cores with float accumulation and writes Y[i][j] = acc * su[i] * sw[j] as bf16.  d a multiple
 * of 128 (GELO_ESHAPE otherwise), p a multiple of 8.  The rounding of U and W to 3 fraction bits (relative
 * error 2^-4 per element at worst) reaches Z = A^-1 Y at about 4e-2 to 7e-2 relative Frobenius error with
 * shield rows in the batch: this call does NOT meet the 2e-2 bound of the bf16 chain; mix and unmix stay bf16. */
gelo_status gelo_fp8_weight_bytes(int d, int p, size_t* bytes);
gelo_status gelo_prepare_weight_fp8(gelo_ctx* ctx, int d, int p, const void* W, int64_t ldw, void* Wq, void* stream);
gelo_status gelo_project_fp8(gelo_ctx* ctx, int n, int d, int p, const void* U, int64_t ldu, const void* Wq,
                             void* Y, int64_t ldy, void* stream);

/* Trusted side, eq. 3 + shield drop.  Z[n_data x p] = (A^-1 * Y)[0:n_data, :]; the shield rows
 * of the product are never computed.  Y: n x p (ldy), Z: n_data x p (ldz), both of type `dtype`
 * (GELO_EDTYPE if it is not the mixing object's).  Marks the mixing consumed: a second
 * gelo_mix or gelo_unmix on it returns GELO_EREUSE. */
gelo_status gelo_unmix(gelo_ctx* ctx, gelo_mixing* mixing, gelo_dtype dtype, int p, const void* Y, int64_t ldy,
                       void* Z, int64_t ldz, void* stream);

gelo_status gelo_mixing_free(gelo_ctx* ctx, gelo_mixing* mixing);
/* gelo_mix, gelo_project and gelo_unmix (eqs. 1-3) for a mixing object drawn earlier, in one call: H (n_data x d),
 * W (d x p), Z (n_data x p), U (n x d) and Y (n x p) densely packed, all of type `dtype`; U and Y are required (they
 * are the observable messages).  The latency-bound decode path spends one host call per layer-step this way. */
gelo_status gelo_chain(gelo_ctx* ctx, gelo_mixing* mixing, gelo_dtype dtype, int p, const void* H, const void* W,
                       float shield_scale, gelo_norm_stat stat, void* Z, void* U, void* Y, void* stream);
/* Shape and type a mixing object was drawn for (any out pointer may be NULL): H is n_data x d,
 * U is (n_data + k_shield) x d, Y is (n_data + k_shield) x p, Z is n_data x p. */
gelo_status gelo_mixing_info(gelo_ctx* ctx, const gelo_mixing* mixing, int* n_data, int* k_shield, int* d,
                             gelo_dtype* dtype, gelo_kind* kind);

/* The whole chain for one batch: sample, mix, project, unmix (eqs. 1-3).  H: n_data x d, W: d x p,
 * Z: n_data x p, all densely packed (leading dimension = width).  U_opt (n x d) and Y_opt (n x p)
 * receive the two observable messages; if NULL they are written to context workspace instead. */
gelo_status gelo_qkv_forward(gelo_ctx* ctx, gelo_kind kind, gelo_dtype dtype, int n_data, int k_shield,
                             int d, int p, const void* H, const void* W, float shield_scale,
                             gelo_norm_stat stat, double cond_max, int max_attempts, uint64_t batch_id,
                             void* Z, void* U_opt, void* Y_opt, void* stream);

/* For callers that cannot allocate (code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc): gelo_qkv_forward for one decode-shaped batch with every intermediate of the
 * trusted side (A, A^-1, the factorisation workspace, shield directions and rows) in a static device
 * buffer of GELO_STATIC_SCRATCH_BYTES that each GPU the library runs on holds until the process ends.
 * Calls no hipMalloc / hipFree and creates no stream, event or pooled object.  n = n_data + k_shield
 * <= GELO_STATIC_MAX_N, and the batch's buffers (about 0.6 MB at n = 128 plus 10 bytes (bf16) or
 * 12 bytes (float) per element of the k_shield x d shield block) must fit the static buffer:
 * GELO_ESHAPE otherwise.  kind: any but GELO_GAUSSIAN.  U (n x d) and
 * Y (n x p) are required; H, W, Z, U, Y densely packed as in gelo_qkv_forward.  All calls on one GPU
 * share the one buffer, whatever their context or stream: calls that overlap in time on a GPU race;
 * issue them on one stream or order them yourself.  Same results, bit for bit, as gelo_qkv_forward
 * (a projection that cuts K over workgroups keeps its float partial sums in the static buffer too;
 * only if they do not fit behind the batch's buffers is K left whole, and Y then differs from
 * gelo_qkv_forward's in the order of summation: never for n x p up to 68 x 12288). */
gelo_status gelo_qkv_forward_static(gelo_ctx* ctx, gelo_kind kind, gelo_dtype dtype, int n_data, int k_shield,
                                    int d, int p, const void* H, const void* W, float shield_scale,
                                    gelo_norm_stat stat, uint64_t batch_id, void* Z, void* U, void* Y, void* stream);

/* ---------------------------------------------------------------------------------------------------------------
 * What the trusted side does itself between two obfuscated projections: the hidden states H of the next batch from the
 * residual stream, queries and keys rotated by their positions and kept in a paged cache, and the attention that
 * reads the cache.  All calls are asynchronous on `stream`; device arrays are read when the kernels run.
 *
 * gelo_kv_cache: K and V are arrays of n_pages pages; row r of head h of page g starts at element
 * g page_stride + h head_stride + r row_stride of either (the same strides for both, multiples of 8, row_stride at
 * most 2^24, head_dim contiguous values at each).  page_rows is a power of two from 16 on.  k and v are 16-byte aligned DEVICE pointers.
 * (gelo_rope_append fills caches of any head_dim that is a multiple of 8, gelo_attention reads those of 64, 96, 128 and 256.)
 * gelo_seq_batch: sequence s brings the rows [row_start[s], row_start[s + 1]) of the batch and has kv_len[s] rows in the
 * cache; row p of it lies in page page_table[s table_ld + p / page_rows], row p % page_rows.  row_start
 * (n_seqs + 1 ascending values from 0 to n_rows) may be NULL if every sequence brings one row (n_rows = n_seqs,
 * max_rows = 1).  All three are DEVICE arrays of 32-bit integers.  max_rows and max_kv_len bound the rows a sequence brings
 * and its kv_len, on the HOST: launches and workspaces are sized by them, so a captured launch serves all batches within its
 * bounds.  Entries of page_table behind the last used page are not read.
 * The structures are read during the call only. */
typedef struct gelo_kv_cache {
    void* k;
    void* v;
    int n_pages, n_kv_heads, page_rows, head_dim;
    int64_t page_stride, head_stride, row_stride;
} gelo_kv_cache;

typedef struct gelo_seq_batch {
    int n_seqs, n_rows, max_rows, max_kv_len;
    const int32_t* row_start;
    const int32_t* kv_len;
    const int32_t* page_table;
    int64_t table_ld;
} gelo_seq_batch;

/* Which components of a head turn together: i and i + rot_dim / 2, or 2 i and 2 i + 1. */
typedef enum { GELO_ROPE_HALF = 0, GELO_ROPE_PAIRS = 1 } gelo_rope_layout;

#define GELO_NORM_MAX_D 65536  /* widest row gelo_rms_norm takes */

/* Root-mean-square norm of the rows of h = X + R (R may be NULL: h = X):
 *   R_out = h,   y = h / sqrt(mean_j h_j^2 + eps) * gamma,   H = y,   codes = e4m3(y * 448 / max_j |y_j|), scales = max_j |y_j| / 448.
 * X, R, R_out, H: n x d of type `dtype` (ldx, ldr, ldro, ldh); gamma: d values of it.  R_out may be NULL; H (or codes and
 * scales) may be NULL, not both.  H and R_out may be X or R; but for that no output shares memory with another matrix of the call.  Everything is computed in float from the unrounded h and rounded once.  codes: n x d bytes
 * (ldq, a multiple of 8), the row quantisation of gelo_project_fp8, scales: n floats (1 for a row of zeros, 2^-126 where the largest |y| is below 1.3e-36): together the operand of
 * gelo_project_fp8_codes, which wants ldq to be a multiple of 16.  A NaN or infinity in a row makes the row's y NaN or zero as the formula does; a NaN among them gives the
 * code 0x7F and the scale NaN.  d <= GELO_NORM_MAX_D, eps >= 0, n up to 2^22 (d > 8192: 2^21). */
gelo_status gelo_rms_norm(gelo_ctx* ctx, gelo_dtype dtype, int n, int d, const void* X, int64_t ldx, const void* R, int64_t ldr,
                          const void* gamma, float eps, void* R_out, int64_t ldro, void* H, int64_t ldh,
                          uint8_t* codes, int64_t ldq, float* scales, void* stream);

/* gelo_project_fp8 whose left operand is 8-bit codes with row scales already (as gelo_rms_norm writes them): n x d bytes,
 * ldq a multiple of 16 bytes, n floats.  d a multiple of 128. */
gelo_status gelo_project_fp8_codes(gelo_ctx* ctx, int n, int d, int p, const uint8_t* codes, int64_t ldq, const float* scales,
                                   const void* Wq, void* Y, int64_t ldy, void* stream);

/* Fills the table of gelo_rope_append: table[(p - first_pos) rot_dim + 2 i] = cos(p w_i), the next float sin(p w_i), for
 * positions p = first_pos ... first_pos + n_pos - 1 and i < rot_dim / 2, from angles in double.  w_i = base^(-2 i / rot_dim),
 * stretched for contexts longer than the trained one by `factor` (1: not at all): with lambda_i = 2 pi / w_i and
 * t_i = (trained / lambda_i - low) / (high - low) cut to [0, 1], w_i becomes w_i (t_i + (1 - t_i) / factor) - waves that turn more than `high` times
 * over the trained length stay, those of less than `low` turns are stretched in full.  trained = 0: all are stretched in full
 * (linear interpolation of positions; low and high are ignored).  rot_dim a multiple of 16, table 16-byte aligned. */
gelo_status gelo_rope_table(gelo_ctx* ctx, int rot_dim, int first_pos, int n_pos, double base, double factor, double trained,
                            double low, double high, float* table, void* stream);

/* Rotates the queries and keys of the batch's rows by their positions and appends keys and values to the cache.  QKV: n_rows x
 * (n_q_heads + 2 n_kv_heads) head_dim of type `dtype` (ld), the fused Q | K | V that gelo_unmix writes as Z.  Row j of sequence s, which
 * brings n of them, has position p = kv_len[s] - n + j (kv_len counts the new rows).  The first rot_dim components
 * of every query and key head turn by the angles of `table` (row p, as gelo_rope_table writes it; positions from 0, n_table of them, at
 * least max_kv_len); the rest and the values are copied.  Q: n_rows x n_q_heads head_dim (ldq) takes the queries; it may be QKV itself
 * (ldq = ld: in place), but not share its memory otherwise.  n_q_heads = 0 (Q NULL): keys and values only, as for an encoder's states.  rot_dim = 0 (table NULL): nothing
 * turns.  A row of negative position gives zero queries and is not appended; one at or beyond max_kv_len gives NaN queries and is not
 * appended; one whose page number lies outside the cache is not appended.  rot_dim a multiple of 16 up to head_dim, head_dim a multiple of 8. */
gelo_status gelo_rope_append(gelo_ctx* ctx, gelo_dtype dtype, int n_q_heads, const void* QKV, int64_t ld, const gelo_kv_cache* cache,
                             const gelo_seq_batch* batch, gelo_rope_layout layout, int rot_dim, const float* table, int n_table,
                             void* Q, int64_t ldq, void* stream);

/* Attention over the cache: O[row, h] = sum_p softmax_p(scale Q[row, h] . K[p, h']) V[p, h'], h' = h n_kv_heads / n_q_heads
 * (n_q_heads a multiple of n_kv_heads).  causal != 0: row j of the n that sequence s brings sees the rows p <= kv_len[s] - n + j of
 * the cache (its own last; kv_len counts the new rows, which are in the cache already); causal = 0: all p < kv_len[s] (cross
 * attention to states of another length).  A row that sees nothing gives zeros (one that sees only scores of -infinity: NaN).  Q, O: n_rows x n_q_heads head_dim of type
 * `dtype` (ldq, ldo), no bytes in common; head_dim 64, 96, 128 or 256.  Rows outside [row_start[0], row_start[n_seqs]) are left as
 * they are.  kv_len beyond max_kv_len is cut to it, below zero is zero; a page number outside the cache is not followed: the
 * results of its sequence are then NaN or partly so.  Statistics, products and sums are float; GELO_BF16 holds the weights exp(s - max) in 16
 * bits for the product with V; a call where max_rows times the query heads of a key head is more than 16 may round them to bfloat16, in their sum too.  What lies in
 * cache rows that no query of the batch sees does not reach the result, NaN and infinity included.
 * Where the rows and heads are too few to fill the chip the cache's length is cut over workgroups and their parts are joined through float
 * workspace of the context (gelo_reserve_attention sizes it ahead; else the first call that needs more allocates): calls on one context must not
 * overlap in time on different streams. */
gelo_status gelo_attention(gelo_ctx* ctx, gelo_dtype dtype, int n_q_heads, const void* Q, int64_t ldq, const gelo_kv_cache* cache,
                           const gelo_seq_batch* batch, float scale, int causal, void* O, int64_t ldo, void* stream);
/* Allocates that workspace (as much as any batch of heads of this width needs): gelo_attention then allocates nothing. */
gelo_status gelo_reserve_attention(gelo_ctx* ctx, int head_dim);

/* ---------------------------------------------------------------------------------------------------------------
 * A paged cache of 4 bits: a block of 32 values of a head's row is held as codes - a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 -
 * times 2^e, e the least whole number from -110 to 125 with max |value| <= 7 2^e (125 if none is), each to nearest, ties to the even code.  No value is off by more than
 * 2^e, a seventh of the block's largest at least and below two sevenths of it, but at the ends: what lies beyond 7 2^125 (3.0e38) becomes 6 2^125, and a block whose largest is
 * 3.5 2^-110 (2.7e-33) or less has 2^-110 all the same, so that no value is off by more than 2^-111 and those of 2^-112 and less are zeros.
 * A block with a NaN or an infinity is NaN as a whole.  17/32 of a byte to a value: 2.1 GB of keys and values of bfloat16 are 0.57 GB.
 *
 * gelo_kv_cache_fp4: K and V are arrays of n_pages pages; head h of page g is a piece of gelo_fp4_page_bytes(page_rows, head_dim) bytes from byte
 * g page_stride + h head_stride of either (strides in bytes, multiples of 16, of pages below 2^31).  page_rows is a power of two from 16 on, head_dim a multiple of 32, their
 * product at most 2^28.  k and v are 16-byte aligned DEVICE pointers.  A piece is the codes of its rows, then their scale bytes (e + 127; 255: NaN; a query that
 * sees a block of another byte beyond 252 or below 17 gets what it may), as gelo_rope_append_fp4 writes them: two codes to a byte, the value of even number in the lower half; of keys row by row, of values four rows at a time: of each
 * of the four rows the first head_dim / 32 bytes of its codes, then of each the next, 16 times; and of each the first block's scale, then of each the next block's. */
typedef struct gelo_kv_cache_fp4 {
    uint8_t* k;
    uint8_t* v;
    int n_pages, n_kv_heads, page_rows, head_dim;
    int64_t page_stride, head_stride;
} gelo_kv_cache_fp4;

/* bytes = 17 page_rows head_dim / 32 */
gelo_status gelo_fp4_page_bytes(int page_rows, int head_dim, size_t* bytes);

/* gelo_rope_append into such a cache; everything said there holds.  Queries come out as there, to the bit; a key's codes are those of its rotation worked out
 * in double, a value's those of the value.  Entries of rows of the cache that the batch does not bring are left as they are. */
gelo_status gelo_rope_append_fp4(gelo_ctx* ctx, gelo_dtype dtype, int n_q_heads, const void* QKV, int64_t ld, const gelo_kv_cache_fp4* cache,
                                 const gelo_seq_batch* batch, gelo_rope_layout layout, int rot_dim, const float* table, int n_table,
                                 void* Q, int64_t ldq, void* stream);

/* The values that the batch's rows are held as: row j of sequence s, which brings n of them, is the cache's row kv_len[s] - n + j, so a batch that brings all
 * kv_len[s] rows reads whole sequences.  K, V: n_rows x n_kv_heads head_dim of type `dtype` (ldk, ldv), no bytes in common; either may be NULL.  Exact in
 * both types.  A row of negative position gives zeros; one at or beyond max_kv_len and one whose page number lies outside the cache give NaN. */
gelo_status gelo_cache_rows_fp4(gelo_ctx* ctx, gelo_dtype dtype, const gelo_kv_cache_fp4* cache, const gelo_seq_batch* batch,
                                void* K, int64_t ldk, void* V, int64_t ldv, void* stream);

/* gelo_attention over such a cache; everything said there holds, for keys and values as they are held.  They are multiplied exactly; GELO_F32 has queries
 * and weights in full.  Weights are relative to a maximum that may lag up to 2^8 behind: sums of values beyond 2^100 can overflow.
 * The workspace that such a call has used stays until the context ends, also where a later call needs a larger one: a captured call has its address. */
gelo_status gelo_attention_fp4(gelo_ctx* ctx, gelo_dtype dtype, int n_q_heads, const void* Q, int64_t ldq, const gelo_kv_cache_fp4* cache,
                               const gelo_seq_batch* batch, float scale, int causal, void* O, int64_t ldo, void* stream);

/* ---------------------------------------------------------------------------------------------------------------
 * Low-rank adapters of many requests beside one projection, on the trusted side: the shared weight is public, what a request adds to it is not.
 *
 * gelo_adapters: n_adapters of them.  The p columns are n_parts parts (the queries, keys and values of a fused projection) that end at columns
 * part_end[0] < part_end[1] < ... = p, multiples of 16 but for the last.  Adapter w has an A of n_parts rank rows of d values, row r at a + w a_stride + r lda
 * (rows k rank ... belong to part k), a B of p rows of rank values, row j at b + w b_stride + j ldb, both of the call's type, and a factor scale[w]
 * (scale NULL: 1).  rank is a multiple of 8 up to GELO_ADAPT_MAX_RANK: a smaller one is filled up with zeros.  a, b (16-byte aligned), scale: DEVICE pointers; strides
 * in values, multiples of 8, lda and ldb at most 2^24.  The structure is read during the call only. */
#define GELO_ADAPT_MAX_RANK 128
#define GELO_ADAPT_MAX_PARTS 4
typedef struct gelo_adapters {
    const void* a;
    const void* b;
    const float* scale;
    int n_adapters, rank, n_parts;
    int part_end[GELO_ADAPT_MAX_PARTS];
    int64_t a_stride, lda, b_stride, ldb;
} gelo_adapters;

/* Z[i, j] = base[i, j] + scale[w] sum_r (sum_k H[i, k] A_w[r, k]) B_w[j, r], r over the rank rows of j's part, w = which[i] (DEVICE, n 32-bit
 * integers).  A row whose number is no adapter's (-1, say) gets base[i].  H: n x d (ldh), base, Z: n x p (ldb, ldz) of type `dtype`; Z may be base itself, and
 * shares no memory with H or with base otherwise.  Sums are float, one rounding at the end; GELO_BF16 may hold the inner sum in 16 bits for the second product.  A
 * NaN or infinity in H, base or an adapter reaches only the rows it belongs to.  Rows in any order.  A row's bits do not go by the other rows; they may go by the sizes of the call, n and
 * n_adapters among them.  Calls of many rows put those that share one of the n_adapters together, which takes longer the more there are, and from 12288 on do not: each row
 * then reads its adapter for itself (4096 rows of 4096 -> 12288 columns that share eight of rank 16, us: 51 where n_adapters is 8, 60 at 64, 153 at 12287, 326 at 12288).  Where many are kept
 * it pays to describe the range of them that a batch of prompts uses.
 * The inner sums go through float workspace of the context (gelo_reserve_adapt sizes it ahead; else the first call that needs more allocates, and what it replaces stays
 * until the context ends): calls on one context must not overlap in time on different streams. */
gelo_status gelo_adapt(gelo_ctx* ctx, gelo_dtype dtype, int n, int d, int p, const void* H, int64_t ldh, const gelo_adapters* adapters, const int32_t* which,
                       const void* base, int64_t ldb, void* Z, int64_t ldz, void* stream);
/* Allocates that workspace for calls of up to so many rows, ranks, parts and adapters: gelo_adapt then allocates nothing. */
gelo_status gelo_reserve_adapt(gelo_ctx* ctx, int n, int rank, int n_parts, int n_adapters);

/* Test hook: copies the secrets of a mixing object to caller DEVICE buffers (any may be NULL):
 * A and A_inv as float n x n (dense), S as float k_shield x d (dense; valid after gelo_mix).
 * attempt / kappa are HOST pointers: the accepted attempt number and the library's estimate of
 * kappa_2(A) (1 for ORTHOGONAL and STRUCTURED).  A STRUCTURED object holds no matrix: A and A_inv
 * are built here by transforming the identity, in the context workspace that gelo_qkv_forward also
 * uses for U / Y when they are not passed in - do not run the two at the same time on one context. */
gelo_status gelo_mixing_export(gelo_ctx* ctx, const gelo_mixing* mixing, float* A, float* A_inv,
                               float* S, int* attempt, float* kappa, void* stream);

/* Test hooks for bitwise checks of the integer work.
 * gelo_debug_philox_words: words[4 i .. 4 i + 3] (DEVICE, 16-byte aligned) = the four 32-bit outputs of
 * Philox4x32-10 for counter (first_block + i, stream_id << 8 | attempt, batch id low, batch id high)
 * under the context's key; stream ids: 0 mixing Gaussian (attempt = redraw number), 1 shield
 * directions, 2 CONDITIONED perturbation, 3 sort keys of permutation r and 4 sign words of round r of
 * the structured kind (r travels in the attempt byte).
 * gelo_mixing_export_table: the (rounds + 1) x n words of a GELO_STRUCTURED object (entry j of
 * permutation r in the low 31 bits, sign flip of position j in round r in the top bit) to a DEVICE buffer. */
gelo_status gelo_debug_philox_words(gelo_ctx* ctx, uint32_t stream_id, uint32_t attempt, uint64_t batch_id,
                                    uint32_t first_block, uint32_t blocks, uint32_t* words, void* stream);
gelo_status gelo_mixing_export_table(gelo_ctx* ctx, const gelo_mixing* mixing, uint32_t* table, void* stream);
/* Measurement aid (for the caller that reports a kernel against the matrix-core peak, as Section 4.2 style
 * "fraction of peak" figures do): what the matrix cores of this device deliver when every wave issues nothing
 * but independent matrix instructions from registers - v_mfma_f32_16x16x32_bf16 (fp8 = 0, 32 accumulator tiles per
 * wave) or v_mfma_f32_32x32x64_f8f6f4 on E4M3 (fp8 = 1, eight), two waves per SIMD, as in a K
 * step of the projection kernels; no memory traffic.  Runs one warm-up launch and `launches` (1..1000) timed
 * launches of `iters` (1..2^20) loop passes each on `stream`, WAITS for them, and returns the mean time of one
 * launch (HOST double) and the floating-point operations one launch executes (HOST double).  Uses the static
 * scratch buffer of gelo_qkv_forward_static: do not overlap the two on one GPU. */
gelo_status gelo_measure_matrix_rate(gelo_ctx* ctx, int fp8, int iters, int launches, double* seconds, double* flop,
                                     void* stream);

/* Test hook: the row quantisation gelo_project_fp8 applies to U, into caller DEVICE buffers: codes n x d bytes
 * (16-byte aligned), scales n floats. */
gelo_status gelo_debug_quantize_rows_fp8(gelo_ctx* ctx, int n, int d, const void* U, int64_t ldu, uint8_t* codes,
                                         float* scales, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* GELO_H */
