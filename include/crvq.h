/*
 * crvq.h -- C ABI of libcrvq, the MI355X (gfx950) hot path of CRVQ,
 * "Channel-Relaxed Vector Quantization for Extreme Compression of LLMs"
 * (arXiv 2412.09282).
 *
 * Conventions shared by every call
 * --------------------------------
 * - Array arguments are DEVICE pointers owned by the caller.  The library
 *   never allocates, frees or retains them after the call returns.  Arrays of
 *   pointers (books, codes of several codebooks) are HOST arrays whose
 *   entries are device pointers.
 * - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *   Work is enqueued on it asynchronously; the call returns after enqueue.
 * - All arguments are validated on the host before anything is enqueued.  On
 *   a validation error nothing runs, outputs are untouched and a nonzero
 *   crvq_status is returned; crvq_last_error() gives the reason (thread-local
 *   text).  No exception crosses the ABI and the library never aborts.
 *   Launch failures return CRVQ_ERR_HIP.
 * - Device-resident indices (codes, perm, initial-codeword indices) cannot be
 *   checked on the host; every kernel bounds-checks them and treats an
 *   out-of-range entry as documented per call (it never reads out of bounds).
 * - Scratch memory comes from a caller-supplied `workspace` of at least the
 *   size the matching *_workspace_size() function returns (256-byte aligned).
 * - Layouts are row-major.  A codebook is K x d elements.  Codes are int32.
 * - A "vector set" is the paper's sub-vector partition (Sec. 3.1 Eq. 1): a
 *   matrix of n_rows rows is cut into vecs_per_row contiguous d-vectors per
 *   row; vector v = r * vecs_per_row + g starts at element r * ld + g * d of
 *   `X`.  The critical slab of a reordered matrix (its first n_crit columns,
 *   Sec. 4.3) is the vector set with vecs_per_row = n_crit / d, ld = N.
 * - Element types: CRVQ_F32 (float) and CRVQ_BF16 (bfloat16, stored as
 *   uint16 bit patterns).  Floating-point inputs must be finite.
 * - Results are deterministic: no floating-point atomics are used anywhere,
 *   so equal inputs give bitwise-equal outputs.
 */
#ifndef CRVQ_H
#define CRVQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  CRVQ_OK = 0,
  CRVQ_ERR_INVALID = 1,     /* a NULL required pointer or an out-of-range size / option */
  CRVQ_ERR_UNSUPPORTED = 2, /* a valid request outside what the library implements */
  CRVQ_ERR_WORKSPACE = 3,   /* workspace missing or smaller than the *_workspace_size() result */
  CRVQ_ERR_HIP = 4          /* the HIP runtime reported an error while enqueueing */
} crvq_status;

/* CRVQ_F64 is accepted only where a call says so (the fp64 operands of the
 * refinement calls and the fp64 output of crvq_dequant / crvq_dequant_books). */
typedef enum { CRVQ_F32 = 0, CRVQ_BF16 = 1, CRVQ_F64 = 2 } crvq_dtype;
typedef enum { CRVQ_REDUCE_SUM = 0, CRVQ_REDUCE_MAX = 1 } crvq_reduce;

#define CRVQ_MAX_K 65536   /* codewords per codebook (e <= 16 bits) */
#define CRVQ_MAX_D 16      /* sub-vector length */
#define CRVQ_MAX_BEAM 16   /* residual beam width (each lane group keeps its top-B list in registers) */
#define CRVQ_MAX_BOOKS 8   /* basic + extended codebooks */

/* Library version (major * 10000 + minor * 100 + patch). */
int crvq_version(void);

/* Text describing the last error returned on the calling thread ("" if none). */
const char* crvq_last_error(void);

/* ---------------------------------------------------------------------------
 * crvq_channel_importance -- column (input-channel) reduction.
 *
 *   out[j] = s_j * R_{i < M} (A[i*lda + j] - B[i*ldb + j])^2,   j < N
 *
 * R = sum (CRVQ_REDUCE_SUM, accumulated in fp64) or max (CRVQ_REDUCE_MAX,
 * exact); B may be NULL (treated as 0); scale may be NULL (s_j = 1).
 * The paper's channel-importance metrics are modes of this one reduction:
 *  - Hessian diagonal h_j = [X X^T]_jj (Appendix A.2 Eq. 9): A = the
 *    calibration activations stored tokens x N, B = NULL, scale = NULL, SUM.
 *  - W-only importance I_j = max_i w_ij^2 (Sec. 4.1): A = W, MAX.
 *  - W-A importance (Sec. 4.1 Eq. 7 / Appendix A.2 Eq. 10): A = W,
 *    B = the prequantized W, MAX, scale = h/2 (Eq. 10) or 1/(2[H^-1]_jj) (Eq. 7).
 *  - Energy-weighted importance I_j = h_j * sum_i w_ij^2: A = W, SUM, scale = h.
 * A, B: M x N matrices of `dtype` with leading dimensions lda, ldb >= N.
 * scale: float[N] or NULL.  out: float[N] (fp32, rounded once from fp64).
 * workspace: crvq_importance_workspace_size(M, N) bytes.
 */
size_t crvq_importance_workspace_size(int64_t M, int64_t N);
crvq_status crvq_channel_importance(const void* A, int64_t lda, const void* B, int64_t ldb, int dtype,
                                    int64_t M, int64_t N, const float* scale, int reduce, float* out,
                                    void* workspace, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * crvq_reorder -- channel reordering (Sec. 4.2, Alg. 1 ReorderChannels) and
 * its reverse (Sec. 4.3 / Fig. 3 right).
 *
 * If importance != NULL, first writes perm[N]: the channels in descending
 * importance, equal importance in ascending channel index, NaN last (a
 * stable descending sort).  Otherwise perm is an input and must hold a
 * permutation of 0..N-1.
 * Then forward (inverse == 0):  out[r*ld_out + k]       = in[r*ld_in + perm[k]]
 *      inverse (inverse != 0):  out[r*ld_out + perm[k]] = in[r*ld_in + k]
 * for r < M, k < N.  in and out are M x N of `dtype`, must not overlap.
 * in may be NULL (then only perm is computed; M is ignored).  An
 * out-of-range perm entry leaves the affected output elements unwritten.
 * workspace: crvq_reorder_workspace_size(N) bytes, needed when importance != NULL or
 * inverse != 0.  N <= 2^20.
 */
size_t crvq_reorder_workspace_size(int64_t N);
crvq_status crvq_reorder(const void* in, int64_t ld_in, void* out, int64_t ld_out, int dtype, int64_t M,
                         int64_t N, const float* importance, int32_t* perm, int inverse, void* workspace,
                         size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * crvq_assign -- nearest-codeword encoding (Sec. 3.1 Eq. 3-4; Alg. 1
 * VectorQuant):  codes[v] = argmin_k ||x_v - C_k||_2, v < n_rows*vecs_per_row.
 *
 * Exact: the chosen k minimises the fp64 squared distance
 * sum_t (x_vt - C_kt)^2 (t ascending); among equal distances the lowest k
 * wins.  dist[v] (optional) = that fp64 distance rounded to float.
 * X: vector set (see conventions) of x_dtype, d <= 16.
 * C: K x d codebook of c_dtype, 1 <= K <= 65536.
 * codes: int32[n]; dist: float[n] or NULL.
 * workspace: crvq_assign_workspace_size(n, d, K) bytes.
 */
size_t crvq_assign_workspace_size(int64_t n_vectors, int32_t d, int64_t K);
crvq_status crvq_assign(const void* X, int x_dtype, int64_t n_rows, int64_t vecs_per_row, int64_t ld,
                        int32_t d, const void* C, int c_dtype, int64_t K, int32_t* codes, float* dist,
                        void* workspace, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * crvq_assign_noalloc -- crvq_assign for callers that cannot allocate device
 * memory (code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc): the same arguments and results without a workspace.  Its
 * scratch is a fixed array of CRVQ_NOALLOC_SCRATCH_BYTES inside the library's
 * device memory, one per GPU, held until the process ends; the call allocates
 * nothing.  A request whose crvq_assign_workspace_size(n, d, K) exceeds that
 * size returns CRVQ_ERR_UNSUPPORTED before anything is enqueued (128 MiB holds
 * about 2.5 million vectors against 65536 codewords, 4.8 million against 256).  Every call on a GPU
 * shares that GPU's array: calls that overlap on one GPU (on different
 * streams or from different threads) race and must be ordered by the caller;
 * calls on one stream are ordered already.  The array's contents left by one
 * call are never read by the next (every counter is reset by the call).
 */
#define CRVQ_NOALLOC_SCRATCH_BYTES (128LL << 20)
crvq_status crvq_assign_noalloc(const void* X, int x_dtype, int64_t n_rows, int64_t vecs_per_row, int64_t ld,
                                int32_t d, const void* C, int c_dtype, int64_t K, int32_t* codes, float* dist,
                                void* stream);

/* ---------------------------------------------------------------------------
 * crvq_assign_residual_beam -- joint code choice over additive codebooks by
 * beam search (Sec. 3.1 last paragraph; Sec. 4.3; Alg. 1 BeamSearchOptimize),
 * under the squared Euclidean error of the residual.
 *
 * books[0] is the basic codebook, books[1..n_books-1] the extended ones, in
 * the order they were fitted.  For each vector, starting from one empty
 * tuple with residual x: for book t, every kept tuple (rank p, residual r)
 * is extended by every codeword c of book t; a candidate's key is
 * (sum_j (r_j - c_j)^2 in fp64, p, codeword index), the `beam` smallest keys
 * survive in key order, and a survivor's residual is r - c (fp64).  The
 * answer is the rank-0 tuple after the last book.  beam = 1 is the greedy
 * additive fit of Alg. 1's extended-codebook loop.
 * X: vector set of x_dtype.  books: host array of n_books device pointers,
 * book t is Ks[t] x d of book_dtypes[t].  codes: host array of n_books
 * device pointers; the code of vector v = r * vecs_per_row + g for book t is
 * written to codes[t][r * ldc[t] + g] (ldc = NULL means ldc[t] = vecs_per_row;
 * otherwise ldc[t] >= vecs_per_row, so the basic codes of a critical slab can
 * land directly in the full matrix's code array).  err: float[n] (final
 * squared error, vector order) or NULL.
 * 1 <= beam <= 16, 1 <= n_books <= 8.
 * workspace: crvq_beam_workspace_size(n, d, n_books, Ks, beam) bytes.
 */
size_t crvq_beam_workspace_size(int64_t n_vectors, int32_t d, int32_t n_books, const int64_t* Ks, int32_t beam);
crvq_status crvq_assign_residual_beam(const void* X, int x_dtype, int64_t n_rows, int64_t vecs_per_row,
                                      int64_t ld, int32_t d, int32_t n_books, const void* const* books,
                                      const int32_t* book_dtypes, const int64_t* Ks, int32_t beam,
                                      int32_t* const* codes, const int64_t* ldc, float* err, void* workspace,
                                      size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * crvq_kmeans_update -- one Lloyd update of a K-means codebook (Sec. 3.1
 * Eq. 2; Alg. 1 KMeansCodebook):
 *
 *   C[k] := mean{ x_v : codes[v] == k }  (fp64 sums, rounded to c_dtype
 *   round-to-nearest-even); a codeword with no members is left unchanged.
 *
 * Atomic-free and deterministic: codes are stably counting-sorted, every
 * centroid is a fixed-order fp64 reduction over its segment.  Codes outside
 * [0, K) belong to no cluster.  counts: int32[K] member counts, or NULL.
 * workspace: crvq_kmeans_workspace_size(n, d, K) bytes.
 */
size_t crvq_kmeans_workspace_size(int64_t n_vectors, int32_t d, int64_t K);
crvq_status crvq_kmeans_update(const void* X, int x_dtype, int64_t n_rows, int64_t vecs_per_row, int64_t ld,
                               int32_t d, const int32_t* codes, int64_t K, void* C, int c_dtype,
                               int32_t* counts, void* workspace, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * crvq_gather_vectors -- out[k] = x_{idx[k]} for k < count (the K-means
 * initial codewords drawn from the vector set, Alg. 1 KMeansCodebook).
 * idx: int64[count] device array; an index outside [0, n) yields a NaN row.
 * out: count x d of out_dtype (same as x_dtype, or F32 from BF16 widening).
 */
crvq_status crvq_gather_vectors(const void* X, int x_dtype, int64_t n_rows, int64_t vecs_per_row, int64_t ld,
                                int32_t d, const int64_t* idx, int64_t count, void* out, int out_dtype,
                                void* stream);

/* ---------------------------------------------------------------------------
 * crvq_dequant -- additive reconstruction, the ComputeError / Update steps of
 * Alg. 1, and the reverse reordering at inference (Sec. 4.3, Fig. 3 right).
 *
 * For an M x n_cols matrix in reordered channel order, vector (r, g), g <
 * n_cols/d, is rebuilt as
 *   R[r, g*d+t] = C_base[q_base[r*ldq_base+g]][t]
 *                 + sum_{e < n_ext, g < n_crit/d} C_ext[e][q_ext[e][r*ldq_ext+g]][t]
 * summed in fp64 in book order.  Then
 *   minuend != NULL (residual mode):  out[r*ld_out + c] = minuend[r*ld_min + c] - R[r, c]
 *   perm != NULL (reverse reorder):   out[r*ld_out + perm[c]] = R[r, c]
 *   otherwise:                        out[r*ld_out + c] = R[r, c]
 * each rounded once to out_dtype (CRVQ_F64 allowed when perm is NULL: the
 * residual of the refinement calls, minuend - R exact up to one fp64 rounding).
 * perm and minuend are mutually exclusive.
 * n_crit is a multiple of d, 0 <= n_crit <= n_cols.  A code outside its
 * codebook yields NaN for that vector.
 * workspace: crvq_dequant_workspace_size(n_cols) bytes (only used with perm).
 */
size_t crvq_dequant_workspace_size(int64_t n_cols);
crvq_status crvq_dequant(int64_t M, int64_t n_cols, int32_t d, int64_t n_crit, const int32_t* q_base,
                         int64_t ldq_base, const void* C_base, int base_dtype, int64_t K_base, int32_t n_ext,
                         const int32_t* const* q_ext, int64_t ldq_ext, const void* const* C_ext,
                         const int32_t* ext_dtypes, const int64_t* K_ext, const int32_t* perm,
                         const void* minuend, int minuend_dtype, int64_t ld_min, void* out, int out_dtype,
                         int64_t ld_out, void* workspace, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * crvq_dequant_books -- crvq_dequant for a layout with n_base >= 1 basic
 * codebooks (the additive basic VQ with m > 1 books of Sec. 3.2 and Sec. 6.4,
 * e.g. m = 2 books on d = 16 vectors) followed by n_ext extended books:
 *   R[r, g*d+t] = sum_{b < n_base} C[b][q[b][r*ldq_base+g]][t]
 *                 + sum_{n_base <= b < n_base+n_ext, g < n_crit/d} C[b][q[b][r*ldq_ext+g]][t]
 * summed in fp64 in book order, then written exactly as by crvq_dequant
 * (residual mode with minuend, reverse reorder with perm, else plain), each
 * element rounded once.  q, C, dtypes, Ks: host arrays of n_base + n_ext
 * entries (device pointers for q and C).  n_base + n_ext <= 8.  crvq_dequant is
 * this call with n_base = 1.  A code outside its codebook yields NaN for
 * that vector.  workspace: crvq_dequant_workspace_size(n_cols) bytes (only
 * used with perm).
 */
crvq_status crvq_dequant_books(int64_t M, int64_t n_cols, int32_t d, int64_t n_crit, int32_t n_base, int32_t n_ext,
                               const int32_t* const* q, int64_t ldq_base, int64_t ldq_ext, const void* const* C,
                               const int32_t* dtypes, const int64_t* Ks, const int32_t* perm, const void* minuend,
                               int minuend_dtype, int64_t ld_min, void* out, int out_dtype, int64_t ld_out,
                               void* workspace, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * crvq_bits_per_weight -- average storage per weight of a quantized layer
 * (Sec. 3.2 Eq. 6 and Appendix A.1 Eq. 8, counted for the exact layout):
 *
 *   bits = [ sum_{b < n_base} (rows*cols/d) * e_b
 *            + sum_{n_base <= b < n_base+n_ext} (rows*n_crit/d) * e_b
 *            + sum_b Ks[b] * d * codeword_bits + cols * perm_bits ] / (rows*cols)
 *
 * with e_b = ceil(log2 Ks[b]), the code width that indexes book b (0 for a
 * one-codeword book).  The paper stores codewords in FP16 (codeword_bits =
 * 16) and the channel permutation as 16-bit indices (perm_bits = 16, or 0 to
 * leave it out as Eq. 8 does).  With n_crit = lambda*cols this is Eq. 8 with
 * all m = n_base + n_ext codebooks counted in the codebook term; with
 * n_ext = 0 and perm_bits = 0 it is Eq. 6.
 * Host-only: Ks is a host array of n_base + n_ext entries, out a host double.
 * Needs rows, cols >= 1, d in [1, 16] dividing cols, n_crit a multiple of d in
 * [0, cols], n_base >= 1, n_ext >= 0, n_base + n_ext <= 8, Ks[b] in
 * [1, 65536], codeword_bits in [1, 64], perm_bits in [0, 64].
 */
crvq_status crvq_bits_per_weight(int64_t rows, int64_t cols, int32_t d, int64_t n_crit, int32_t n_base, int32_t n_ext,
                                 const int64_t* Ks, int32_t codeword_bits, int32_t perm_bits, double* out);

/* ===========================================================================
 * Loss-driven refinement (Alg. 1: QuantLoss, FineTuneCodebook,
 * BeamSearchOptimize at width 1).  A layer is taken in reordered channel order
 * (critical channels first).  With calibration activations X stored
 * tokens x N, H = X^T X is the paper's X X^T, R = W - W_hat, and
 *   QuantLoss = ||W X^T - W_hat X^T||_F^2 = sum_r R_r H R_r^T,
 *   d QuantLoss / d W_hat = -2 R H.
 * All refinement arithmetic is fp64; codebooks being tuned are fp32.
 * ------------------------------------------------------------------------- */

/* crvq_gram -- H = X^T X (Appendix A.2: the Hessian proxy X X^T of Eq. 9-10,
 * full matrix).  X: n_rows x n_cols of x_dtype (F32 or F64), row stride ld.
 * H: n_cols x n_cols fp64, row stride ldh >= n_cols.  Products are exact in
 * fp64 for fp32 input; sums are fused multiply-adds in row order. */
crvq_status crvq_gram(const void* X, int x_dtype, int64_t n_rows, int64_t n_cols, int64_t ld, double* H, int64_t ldh,
                      void* stream);

/* crvq_hessian_inverse_diagonal -- the denominator of the W-A channel
 * importance of Sec. 4.1 Eq. 7, [(X X^T)^-1]_jj, for every channel j:
 *
 *   hinv[j]  = [(H + delta I)^-1]_jj,   delta = damp * (sum_j H_jj) / N,
 *   scale[j] = float(1 / (2 hinv[j]))   (Eq. 7's factor, rounded once),
 *
 * so that crvq_channel_importance(W, B = the prequantized W, scale, MAX)
 * gives Eq. 7's I_j.  The damping (damp >= 0; 0.01 is the usual choice)
 * makes the proxy invertible when the calibration set has fewer tokens than
 * channels or a channel is never active.  H: N x N fp64, row stride ldh >= N,
 * symmetric; only its lower triangle (j <= i) is read.  hinv: double[N] and
 * scale: float[N], device memory, either may be NULL (not both).  Computed in
 * fp64 by a blocked Cholesky factorization A = L L^T with the inverse factor
 * T = L^-1 formed alongside ([A^-1]_jj = sum_i T_ij^2); deterministic.  If
 * the damped matrix is not positive definite (a pivot <= 0, NaN or infinite),
 * every hinv[j] and scale[j] is NaN: the status does not report it, since the
 * check runs on the device.  N <= 65536.
 * workspace: crvq_hessian_inverse_workspace_size(N) bytes (about 16 N^2).
 */
size_t crvq_hessian_inverse_workspace_size(int64_t N);
crvq_status crvq_hessian_inverse_diagonal(const double* H, int64_t ldh, int64_t N, double damp, double* hinv,
                                          float* scale, void* workspace, size_t ws_bytes, void* stream);

/* crvq_hessian_product -- G = R H[:, 0:n_out] (so -2 G is the gradient of
 * QuantLoss w.r.t. W_hat on those columns) and, when row_loss != NULL (needs
 * n_out == N), row_loss[r] = sum_j R[r][j] G[r][j], the QuantLoss of row r
 * (Alg. 1 QuantLoss).  When loss_total != NULL (needs row_loss), loss_total[0]
 * = sum_r row_loss[r], the layer's QuantLoss, summed on the device in a fixed
 * order (so a caller's loop guard needs no host-side reduction).
 * R: M x N fp64 (stride ldr), H: N x N fp64 (stride ldh), G: M x n_out fp64
 * (stride ldg >= n_out); loss_total: one fp64 device value.  Deterministic. */
crvq_status crvq_hessian_product(int64_t M, int64_t N, int64_t n_out, const double* R, int64_t ldr, const double* H,
                                 int64_t ldh, double* G, int64_t ldg, double* row_loss, double* loss_total,
                                 void* stream);

/* crvq_code_sums -- sums[k] = sum of the vectors x_v with codes[v] == k, in
 * fp64, and counts[k] their number (the per-codeword gradient of
 * FineTuneCodebook when X holds -2 R H, or plain cluster sums).  X: vector set
 * (see conventions) of CRVQ_F64 elements; codes: int32[n]; codes outside
 * [0, K) belong to no code.  sums: K x d fp64; counts: int32[K] or NULL.
 * 1 <= K <= 65536.  Deterministic: every code's members are added in vector
 * order per block, the blocks in block order (K > 1024: the vectors are first
 * grouped by the high byte of their code, and a code's members are added in
 * vector order per chunk of its group, the chunks in order).
 * workspace: crvq_code_sums_workspace_size(n, d, K) bytes. */
size_t crvq_code_sums_workspace_size(int64_t n_vectors, int32_t d, int64_t K);
crvq_status crvq_code_sums(const double* X, int64_t n_rows, int64_t vecs_per_row, int64_t ld, int32_t d,
                           const int32_t* codes, int64_t K, double* sums, int32_t* counts, void* workspace,
                           size_t ws_bytes, void* stream);

/* crvq_adam_step -- one Adam step (Kingma & Ba, with bias correction; the
 * paper fine-tunes codebooks with beta1 = 0.9, beta2 = 0.95) on n fp32
 * parameters C with gradient g = grad_scale * grad (fp64):
 *   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
 *   C = C - lr * (m / (1 - b1^step)) / (sqrt(v / (1 - b2^step)) + eps)
 * in fp64 (each operation rounded on its own), C rounded once to fp32.
 * m, v: fp64 state of n entries (zero before step 1).  step >= 1. */
crvq_status crvq_adam_step(float* C, const double* grad, double grad_scale, double* m, double* v, int64_t n,
                           int64_t step, double lr, double beta1, double beta2, double eps, void* stream);

/* crvq_adam_step_bf16 -- the same step for a bf16 codebook C (bit patterns)
 * tuned through an fp32 master copy (n floats, state like m and v): at step 1
 * the master is first set to C (exact); the master then moves as
 * crvq_adam_step moves an fp32 codebook, and C becomes the master rounded to
 * bf16, nearest-even (Alg. 1 FineTuneCodebook, as read for bf16 layers). */
crvq_status crvq_adam_step_bf16(uint16_t* C, float* master, const double* grad, double grad_scale, double* m,
                                double* v, int64_t n, int64_t step, double lr, double beta1, double beta2, double eps,
                                void* stream);

/* crvq_refine_codes -- BeamSearchOptimize of Alg. 1 at the paper's width 1,
 * under QuantLoss, for one codebook C (K x d, F32 or BF16) covering the
 * column groups 0 .. n_cols/d - 1 of an M x N layer (n_cols = N for a basic
 * book, n_crit for an extended one).  For every group in column order and
 * every row independently, the group's code becomes the k minimising QuantLoss
 * with all other codes fixed (lowest k among equal values); the residual
 * R (M x N fp64, stride ldr, in/out) and codes (int32, row stride ldq >=
 * n_cols/d, in/out) are updated as it goes.  H: N x N fp64.  The loss change
 * of candidate k in group g is evaluated as
 *   c_k^T H_gg c_k - 2 c_k . ((R H)_g + H_gg c_cur) (minus the same at c_cur),
 * with (R H) kept current as codes move: within a block of 64 columns by
 * delta^T H[g rows, block columns] per change, and for the later columns by one
 * product (the block's deltas) x H per block.  A code outside [0, K) leaves
 * that row's group unchanged.  1 <= K <= 65536: a codebook that fits a CU's
 * LDS (K d <= 8192) is searched from LDS by each workgroup's rows, group after
 * group; a larger one one group at a time over all rows, in codebook slices
 * merged per row (the same values and choices either way).
 * workspace: crvq_refine_workspace_size(M, N, n_cols) bytes. */
size_t crvq_refine_workspace_size(int64_t M, int64_t N, int64_t n_cols);
crvq_status crvq_refine_codes(int64_t M, int64_t N, int32_t d, int64_t n_cols, double* R, int64_t ldr, const double* H,
                              int64_t ldh, const void* C, int c_dtype, int64_t K, int32_t* codes, int64_t ldq,
                              void* workspace, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * crvq_dequant_gemv -- matrix-vector product with a CRVQ-quantized layer, the
 * inference step the paper times (Sec. 4.3, Fig. 3 right; Table 7):
 *
 *   y = W_hat x,   W_hat[:, perm[k]] = R[:, k]   (W_hat = R when perm is NULL),
 *   R[r, 8g+t] = C_base[q_base[r*ldq_base+g]][t]
 *                + sum_{e < n_ext, g < n_crit/8} C_ext[e][q_ext[e][r*ldq_ext+g]][t]
 *
 * for an M x N layer stored as 8-bit codes (every book has K <= 256, d = 8),
 * x of N elements (x_dtype), y of M floats.  N must be a multiple of 64;
 * q_base 8-byte aligned with ldq_base a multiple of 8 and >= N/8; n_crit a
 * multiple of 8 in [0, N].  Products are formed in fp32 (codeword elements and
 * x widened exactly; per column group an 8-term fp32 dot product), partial sums
 * in fp32 over at most 1024 columns and in fp64 across them: |y - W_hat x| is
 * within a few times 2^-24 * sum_j |W_hat_rj x_j|.  A code outside its book or
 * a perm entry outside [0, N) makes y_r NaN.  M = 0 is a no-op.  Deterministic.
 * workspace: crvq_gemv_workspace_size(M, N, K_base) bytes.
 */
size_t crvq_gemv_workspace_size(int64_t M, int64_t N, int64_t K_base);
crvq_status crvq_dequant_gemv(int64_t M, int64_t N, int64_t n_crit, const uint8_t* q_base, int64_t ldq_base,
                              const void* C_base, int base_dtype, int64_t K_base, int32_t n_ext,
                              const uint8_t* const* q_ext, int64_t ldq_ext, const void* const* C_ext,
                              const int32_t* ext_dtypes, const int64_t* K_ext, const int32_t* perm, const void* x,
                              int x_dtype, float* y, void* workspace, size_t ws_bytes, void* stream);

/* ===========================================================================
 * The attention block of a decoder on quantized data: projections in 4 bits
 * (crvq_w4_*) and a paged cache of keys and values in 8 bits (crvq_kv_*).
 *
 * The cache.  Pages of `page` tokens (16, 32, 64, 128 or 256) of Hkv heads of
 * D elements (a multiple of 16 up to 256), n_pages of them:
 *   k_cache  int8 [n_pages][Hkv][page][D]      key of slot s:   k_scale * k_cache[.][h][s][:]
 *   v_cache  int8 [n_pages][Hkv][D][page]      value of slot s: v_scale * v_cache[.][h][:][s]
 *   k_scale, v_scale  float [n_pages][Hkv]     one scale for a head's tokens in a page
 * (values are stored transposed, so that both products of attention read
 * their operand along the contracted index).  Both arrays 16-byte aligned;
 * scales are not negative.
 * Token t of sequence b is in slot t % page of page block_table[b * ld_table +
 * t / page].  A page may belong to several sequences as long as no call
 * appends to it.
 *
 * A batch of B sequences with new tokens: rows start[b] .. start[b+1] - 1 of
 * the n_tokens rows of q, k, v are sequence b's new tokens (start: int32[B+1],
 * device), and kv_len[b] (int32, device) is its number of tokens in the cache
 * with the new ones included: they are the last ones, token i of n being at
 * place kv_len[b] - n + i.  max_new and max_kv (host) are upper bounds of the
 * rows and of kv_len over the batch.  q is n_tokens x Hq x D, k and v n_tokens x
 * Hkv x D with strides (in elements) between tokens and between heads, the D
 * elements of a head contiguous; Hq is a multiple of Hkv, and query heads
 * h * Hq/Hkv .. share key head h.  Element type CRVQ_F32 or CRVQ_BF16.
 * ------------------------------------------------------------------------- */
#define CRVQ_KV_MAX_D 256
#define CRVQ_KV_MAX_LEN (1 << 30) /* tokens of a sequence; a longer kv_len counts as one past its block table */

/* crvq_kv_append -- rotates, quantizes and stores the new keys and values, and
 * rotates the queries, in one launch.
 *
 * Rotation (cos != NULL; rot even, 0 < rot <= D): pair j < rot/2 is elements
 * (j, j + rot/2), or (2j, 2j+1) when interleaved, and becomes (a c - b s,
 * b c + a s) with c = cos[p*rot/2 + j], s = sin[..] (float, n_angles rows) of
 * row p = the token's place in its sequence, or positions[row] (int32, device)
 * when given; fp32, every operation rounded on its own.  The other elements
 * stay.  A place outside the table makes the rotated elements NaN.  q (may be
 * NULL) goes to q_out the same way, rounded to dtype; q_out may be q itself.
 * Quantization of a head's tokens in a page, for k and v alike: with m the
 * largest magnitude among its new tokens, s = max(m / 127, 2^-100).  If the
 * page holds tokens from before the call, the larger of s and its old scale
 * becomes the scale, and if that is s the old codes c become
 * rint(c * (old / s)) (a growth costs an old code up to half a step); otherwise
 * the scale is s.  A new element x becomes min(max(rint(x / scale), -127), 127).
 * A NaN or infinity among the new tokens makes the scale NaN (and the page's
 * head NaN for every reader) with new codes 0.
 * A sequence whose rows are not within [0, n_tokens], that has more than
 * max_new of them or more than kv_len[b], or whose kv_len[b] exceeds ld_table *
 * page, is left out; so are tokens whose page is outside [0, n_pages).
 * Results depend on how tokens are grouped into calls only through the scales'
 * growth. */
crvq_status crvq_kv_append(int32_t B, int32_t Hq, int32_t Hkv, int32_t D, int32_t page, int64_t n_pages, int8_t* k_cache,
                           int8_t* v_cache, float* k_scale, float* v_scale, const int32_t* block_table,
                           int64_t ld_table, const int32_t* start, const int32_t* kv_len, int32_t max_new,
                           int64_t n_tokens, int dtype, const void* k, int64_t k_tok, int64_t k_head, const void* v,
                           int64_t v_tok, int64_t v_head, const void* q, int64_t q_tok, int64_t q_head, void* q_out,
                           int64_t qo_tok, int64_t qo_head, const float* cos, const float* sin, int64_t n_angles,
                           int32_t rot, const int32_t* positions, int interleaved, void* stream);

/* crvq_kv_read -- the values the cache holds for the last start[b+1] - start[b]
 * tokens of every sequence (all of them when that is kv_len[b]): k_out and
 * v_out (either may be NULL), n_tokens x Hkv x D of dtype, each element
 * scale * code rounded once.  Sequences that crvq_kv_append would leave out
 * leave their rows unwritten; tokens whose page is outside [0, n_pages) read
 * NaN. */
crvq_status crvq_kv_read(int32_t B, int32_t Hkv, int32_t D, int32_t page, int64_t n_pages, const int8_t* k_cache,
                         const int8_t* v_cache, const float* k_scale, const float* v_scale, const int32_t* block_table,
                         int64_t ld_table, const int32_t* start, const int32_t* kv_len, int32_t max_new,
                         int64_t n_tokens, int dtype, void* k_out, int64_t k_tok, int64_t k_head, void* v_out,
                         int64_t v_tok, int64_t v_head, void* stream);

/* crvq_kv_attention -- attention of the new tokens over the cache:
 *
 *   out_i = sum_t p_t V_t,  p = softmax over the visible t < kv_len[b] of scale * q_i . K_t
 *
 * with token i of n at place P_i = kv_len[b] - n + i.  causal != 0: t <= P_i is
 * visible, and with window > 0 only t > P_i - window; causal == 0: every t (window must
 * be 0).  n may exceed kv_len[b] (places then start below 0).  A row that sees nothing is
 * 0.  lse (float [n_tokens][Hq] or NULL) = log sum_t exp(scale q_i . K_t), -inf
 * for a row that sees nothing.  out: n_tokens x Hq x D of q's type, its own
 * strides; it may be q itself (same strides), and may not overlap it otherwise.
 * Arithmetic: a query row is held to 24 bits below its largest element (many
 * CRVQ_BF16 rows: as fp16 relative to a power of two), and its products with the
 * key codes are exact; softmax statistics and sums are fp32; weights enter the product with the values
 * with 24 bits (CRVQ_F32), or rounded to 22 (CRVQ_BF16, max_new * Hq / Hkv <= 16; those below 2^-10 of the
 * row's largest keep fewer, at least 11) or to 11 bits (CRVQ_BF16, more rows).
 * A row with a NaN or infinite query element is NaN, as is a row that sees a
 * page outside [0, n_pages) or a page with a scale that is negative or not finite.  Rows of a sequence
 * with kv_len[b] < 0 or > ld_table * page are NaN, as are the first max_new rows of one
 * with more than max_new; a sequence whose rows are not within [0, n_tokens] is
 * left out.  Deterministic.
 * workspace: crvq_kv_attention_workspace_size(...) bytes. */
size_t crvq_kv_attention_workspace_size(int32_t B, int32_t Hq, int32_t Hkv, int32_t D, int32_t max_new, int32_t max_kv);
crvq_status crvq_kv_attention(int32_t B, int32_t Hq, int32_t Hkv, int32_t D, int32_t page, int64_t n_pages,
                              const int8_t* k_cache, const int8_t* v_cache, const float* k_scale, const float* v_scale,
                              const int32_t* block_table, int64_t ld_table, const int32_t* start, const int32_t* kv_len,
                              int32_t max_new, int32_t max_kv, int64_t n_tokens, int dtype, const void* q, int64_t q_tok,
                              int64_t q_head, void* out, int64_t o_tok, int64_t o_head, float scale, int causal,
                              int32_t window, float* lse, void* workspace, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Drafted tokens over the cache.  A tree of drafted tokens is appended like any
 * new tokens (crvq_kv_append with the places of crvq_tree_mask as positions), verified in
 * one call, and the accepted ones are moved behind the context (crvq_kv_gather).
 * ------------------------------------------------------------------------- */

/* crvq_tree_mask -- what the drafted tokens of a tree see.  parents[row]
 * (int32[n_tokens], device) is the index of the token's parent among its
 * sequence's new tokens, below its own, or -1 for a token that follows the
 * context itself; start, kv_len and max_new as in a batch.
 *   mask (uint64 [n_tokens][ld_mask], 64 ld_mask >= max_new, or NULL): bit j of
 *     row i is 1 for j = i and every ancestor j (of those the `window` nearest, i among
 *     them, where window > 0)
 *   places (int32[n_tokens], or NULL) = kv_len - n + depth - 1: a token's place
 *     behind the context, n being the sequence's new tokens
 * A token with a parent that is neither -1 nor below its child, its own or an
 * ancestor's, gets a mask of zeros and the place -1 (which crvq_kv_append turns into NaN
 * queries).  Rows of a sequence that is not within [0, n_tokens] or has more than max_new are left out. */
crvq_status crvq_tree_mask(int32_t B, const int32_t* parents, const int32_t* start, const int32_t* kv_len, int32_t max_new,
                           int64_t n_tokens, int32_t window, uint64_t* mask, int64_t ld_mask, int32_t* places, void* stream);

/* crvq_kv_tree_attention -- crvq_kv_attention (its batch, arithmetic, lse, NaN and
 * left-out rules) with a mask of its own among the new tokens: token i of a
 * sequence's n sees the context, t < kv_len[b] - n, and new token j where bit
 * j % 64 of word mask[row i][j / 64] is 1; bits from n on do not matter.  Any mask will
 * do; a row that sees nothing is 0.  window > 0: of the context only t > P_i - window, P_i =
 * places[row i] (int32, device), or kv_len[b] - n + i where places is NULL;
 * new tokens are seen as the mask says.  At most 2^16 query heads a key head, and 2^30 rows of them.
 * workspace: crvq_kv_tree_attention_workspace_size(...) bytes. */
size_t crvq_kv_tree_attention_workspace_size(int32_t B, int32_t Hq, int32_t Hkv, int32_t D, int32_t max_new, int32_t max_kv);
crvq_status crvq_kv_tree_attention(int32_t B, int32_t Hq, int32_t Hkv, int32_t D, int32_t page, int64_t n_pages,
                                   const int8_t* k_cache, const int8_t* v_cache, const float* k_scale, const float* v_scale,
                                   const int32_t* block_table, int64_t ld_table, const int32_t* start, const int32_t* kv_len,
                                   int32_t max_new, int32_t max_kv, int64_t n_tokens, int dtype, const void* q, int64_t q_tok,
                                   int64_t q_head, void* out, int64_t o_tok, int64_t o_head, float scale, const uint64_t* mask,
                                   int64_t ld_mask, int32_t window, const int32_t* places, float* lse, void* workspace,
                                   size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * The cache within a budget: the attention weight every cached token receives is
 * added up (crvq_kv_weights, after the attention of the same rows), the tokens with the most
 * are kept (crvq_kv_select) and moved to other pages (crvq_kv_gather); the old
 * pages are free then.  Weights: float [B][Hkv][ld], token t of sequence b's
 * cache and key head h at (b * Hkv + h) * ld + t.
 * ------------------------------------------------------------------------- */

/* crvq_kv_weights -- for every sequence that brings rows, key head and token t < kv_len[b]:
 *
 *   after[t] = decay * before[t] + sum_{i, h: row i of head h sees t} exp(scale q_ih . K_t - lse_ih)
 *
 * over the query heads of the key head; the sequence's new tokens have no
 * `before`, and before = NULL is 0 for all; after may be before.  q, lse (as
 * crvq_kv_attention or crvq_kv_tree_attention returned it), scale, causal and
 * window are those of the attention; mask != NULL: of a tree, with places (causal is not
 * looked at).  Rows whose lse is infinite or NaN add nothing, nor do tokens whose page is
 * outside [0, n_pages) or whose scale is negative or not finite.  Sequences
 * that bring no rows, whose rows are not within [0, n_tokens] or more than
 * max_new, or with kv_len[b] < 0, > max_kv or > ld_table * page, and tokens from kv_len[b] on, stay as they were in `after`.
 * Products are exact (CRVQ_F32 queries as three bf16 terms; down to 2^-110), sums fp32 in a
 * fixed order.  ld >= max_kv; B * Hkv is at most 65535, and rows as in crvq_kv_tree_attention.
 * workspace: crvq_kv_weights_workspace_size(...) bytes. */
size_t crvq_kv_weights_workspace_size(int32_t B, int32_t Hq, int32_t Hkv, int32_t D, int32_t max_new, int32_t max_kv);
crvq_status crvq_kv_weights(int32_t B, int32_t Hq, int32_t Hkv, int32_t D, int32_t page, int64_t n_pages, const int8_t* k_cache,
                            const float* k_scale, const int32_t* block_table, int64_t ld_table, const int32_t* start,
                            const int32_t* kv_len, int32_t max_new, int32_t max_kv, int64_t n_tokens, int dtype, const void* q,
                            int64_t q_tok, int64_t q_head, const float* lse, float scale, int causal, int32_t window,
                            const uint64_t* mask, int64_t ld_mask, const int32_t* places, float decay, const float* before,
                            float* after, int64_t ld, void* workspace, size_t ws_bytes, void* stream);

/* crvq_kv_select -- the min(kv_len[b], budget) tokens of every key head that are
 * kept: the first `sinks`, the last `recent` (sinks + recent <= budget), and of
 * the others those with the largest weights, the lower index first where they are equal; NaN counts as
 * less than everything.  keep (int32 [B][Hkv][ld_keep], ld_keep >= min(budget,
 * ld)) gets them in order, kept_weights ([B][Hkv][ld_keep] or NULL) their weights, kept_len (int32[B]) their number,
 * the same for all heads; 0 where kv_len[b] < 0 or > ld.  Entries from kept_len[b] on stay as they were.
 * workspace: crvq_kv_select_workspace_size(B, Hkv, ld) bytes. */
size_t crvq_kv_select_workspace_size(int32_t B, int32_t Hkv, int64_t ld);
crvq_status crvq_kv_select(int32_t B, int32_t Hkv, const int32_t* kv_len, const float* weights, int64_t ld, int32_t budget,
                           int32_t sinks, int32_t recent, int32_t* keep, int64_t ld_keep, int32_t* kept_len, float* kept_weights,
                           void* workspace, size_t ws_bytes, void* stream);

/* crvq_kv_gather -- moves tokens to other pages: slot j % page of page
 * to_table[b * ld_to + j / page] becomes token keep[b][h][j] (int32 [B][keep_heads][ld_keep],
 * keep_heads = Hkv, or 1 for the same tokens of every head) of sequence b, for
 * j < kept_len[b] <= max_keep (host).  A new page's scale is the largest of its tokens' old ones
 * and a code becomes rint(c * (old / new)), in fp32: tokens that shared a page
 * keep their codes, the others lose up to half a step.  Slots of the last page from
 * kept_len[b] on become 0.  The new pages must be none that the call reads and in
 * one place of to_table (otherwise their contents are undefined; nothing outside the cache is
 * touched).  A token outside [0, kv_len[b]), or whose page is outside [0, n_pages)
 * or has a scale that is negative or not finite, makes the new page's head NaN with codes 0.  A
 * sequence with kept_len[b] above ld_keep or ld_to * page, and new pages outside [0, n_pages), are
 * left out. */
crvq_status crvq_kv_gather(int32_t B, int32_t Hkv, int32_t D, int32_t page, int64_t n_pages, int8_t* k_cache, int8_t* v_cache,
                           float* k_scale, float* v_scale, const int32_t* block_table, int64_t ld_table, const int32_t* kv_len,
                           const int32_t* keep, int64_t ld_keep, int32_t keep_heads, const int32_t* kept_len, int32_t max_keep,
                           const int32_t* to_table, int64_t ld_to, void* stream);

/* ---------------------------------------------------------------------------
 * 4-bit matrices.  An M x N matrix as codes c in 0 .. 15 with a scale s and a
 * zero point z for every `group` (32, 64, 128 or 256) consecutive columns of a row:
 *   W[r][j] = s[r][j/group] * (c[r][j] - z[r][j/group]),   z = 8 when zeros is NULL.
 * codes: uint8, column 2i in the low and 2i+1 in the high half of byte i of
 * its row; 16-byte aligned, row stride ld bytes, a multiple of 16 with 2 ld >= N.
 * scales: CRVQ_F32 or CRVQ_BF16, row stride ld_s >= ceil(N / group).  zeros:
 * uint8, row stride ld_z, or NULL.  The last group of a row may be shorter.
 * ------------------------------------------------------------------------- */

/* crvq_w4_quantize -- the codes, scales (and zero points) of W (M x N of dtype,
 * row stride ldw) rounded to nearest, group by group.  zeros NULL: s = max|w| / 7,
 * z = 8.  Otherwise lo = min(0, min w), hi = max(0, max w), s = (hi - lo) / 15,
 * z = min(max(rint(-lo / s), 0), 15).  s is at least 2^-100 and is rounded to its stored type
 * first; c = min(max(rint(w / s) + z, 0), 15).  A NaN or infinity in a group makes its
 * scale NaN (codes 0, zero point 0 or 8).  The last bytes of a row up to a multiple of 16 bytes get zero
 * codes past column N. */
crvq_status crvq_w4_quantize(int64_t M, int64_t N, int32_t group, const void* W, int64_t ldw, int dtype, uint8_t* codes,
                             int64_t ld, void* scales, int scale_dtype, int64_t ld_s, uint8_t* zeros, int64_t ld_z,
                             void* stream);

/* crvq_w4_dequant -- out (M x N of dtype, row stride ldo) = the values, rounded once. */
crvq_status crvq_w4_dequant(int64_t M, int64_t N, int32_t group, const uint8_t* codes, int64_t ld, const void* scales,
                            int scale_dtype, int64_t ld_s, const uint8_t* zeros, int64_t ld_z, void* out, int64_t ldo,
                            int dtype, void* stream);

/* crvq_w4_gemv -- y[t] = W x[t] for T >= 0 vectors: x is T x N of x_dtype (row
 * stride ldx), y is T x M of y_dtype (row stride ldy).  Products are exact
 * (bf16 x as it is, fp32 x as the sum of three bf16 terms), sums fp32 per group and across groups in units of
 * 2^-12 (results below 2^-114 are held to multiples of 2^-137 times a scale), rounded
 * once.  Every finite x has the result of its sums; an infinite or NaN element of x[t] makes y[t] NaN.  y may not overlap x.  Deterministic.
 * Meant for few vectors: codes are read again for every 5 to 32 of them.  Many go in several launches, so that the
 * workspace stays within 64 MiB, or what one such pass needs where that is more.
 * workspace: crvq_w4_gemv_workspace_size(M, N, T) bytes. */
size_t crvq_w4_gemv_workspace_size(int64_t M, int64_t N, int64_t T);
crvq_status crvq_w4_gemv(int64_t M, int64_t N, int64_t T, int32_t group, const uint8_t* codes, int64_t ld,
                         const void* scales, int scale_dtype, int64_t ld_s, const uint8_t* zeros, int64_t ld_z,
                         const void* x, int64_t ldx, int x_dtype, void* y, int64_t ldy, int y_dtype, void* workspace,
                         size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * 8-bit matrices: `rows` rows of N columns as codes c in -127 .. 127 with a
 * scale for each row (a channel of a weight, a token of activations),
 *   X[i][j] = scales[i] * c[i][j].
 * codes: int8, 16-byte aligned, row stride ld bytes, a multiple of 16 and at
 * least N; what lies past column N up to a multiple of 16 belongs to the row's
 * storage.  scales: float[rows].  1 <= N <= CRVQ_ROW_MAX_N.
 * ------------------------------------------------------------------------- */
#define CRVQ_ROW_MAX_N 65536 /* elements of a row: registers hold it (crvq_norm, crvq_w8_*) */

/* crvq_w8_quantize -- the codes and scales of X (rows x N of dtype, row stride
 * ldx): s = max(max|x| / 127, 2^-100), c = min(max(rint(x / s), -127), 127),
 * fp32, every operation rounded on its own.  A NaN or infinity in a row makes
 * its scale NaN and its codes 0.  The bytes of a row past N up to a multiple of
 * 16 become 0. */
crvq_status crvq_w8_quantize(int64_t rows, int64_t N, const void* X, int64_t ldx, int dtype, int8_t* codes, int64_t ld,
                             float* scales, void* stream);

/* crvq_w8_gemm -- y[t][r] = x_scales[t] * scales[r] * sum_j x_codes[t][j] * codes[r][j]
 * for an M x N matrix and T rows of x, y T x M of y_dtype (row stride ldy).  The
 * sum is exact (32-bit integers; codes of -128 are taken as they are), its
 * product with the two scales' product is fp32, each operation rounded on its own,
 * and rounded once to y_dtype.  Columns from N on are not read into the sums.  M = 0 or
 * T = 0 is a no-op.  y may not overlap an input.  Deterministic.
 * workspace: crvq_w8_gemm_workspace_size(M, N, T) bytes. */
size_t crvq_w8_gemm_workspace_size(int64_t M, int64_t N, int64_t T);
crvq_status crvq_w8_gemm(int64_t M, int64_t N, int64_t T, const int8_t* codes, int64_t ld, const float* scales,
                         const int8_t* x_codes, int64_t ldx, const float* x_scales, void* y, int64_t ldy, int y_dtype,
                         void* workspace, size_t ws_bytes, void* stream);

/* crvq_norm -- what lies between two blocks of a decoder, for T rows of N
 * elements in one pass: the norm after a block, its gate and scale, the residual
 * sum, and the norm before the next block:
 *
 *   u = post ? n(x) w_post + b_post : x,   r' = r + alpha (gate u),   h = n(r') w_pre + b_pre
 *   n(x) = x / sqrt(mean x^2 + eps)                     (CRVQ_NORM_RMS)
 *   n(x) = (x - mean x) / sqrt(mean (x - mean x)^2 + eps)   (CRVQ_NORM_LAYER)
 *
 * x, gate and h are of dtype, r and r_out (r') of r_dtype, the weights (N
 * elements each) of w_dtype; ldx, ldg, ldr, ldro and ldh are row strides.
 * NULL: gate and a w are 1, r and a b are 0, r_out and h are not wanted (one of the two
 * has to be).  ldg = 0: one gate of N elements for every row.
 * h_scales != NULL: h is int8 with a scale for each row, as crvq_w8_quantize
 * makes it of the unrounded h (its layout and rules), ready for crvq_w8_gemm.
 * Sums, means and roots are fp64, the rest fp32; h is computed from r' before
 * its rounding to r_dtype.  r_out may be r or x and h may be x or r, of the same type and
 * row stride; outputs overlap nothing otherwise.  T = 0 is a no-op.
 * Deterministic; a row's result does not depend on the other rows. */
typedef enum { CRVQ_NORM_RMS = 0, CRVQ_NORM_LAYER = 1 } crvq_norm_kind;
crvq_status crvq_norm(int64_t T, int64_t N, int kind, const void* x, int64_t ldx, int dtype, int post, const void* w_post,
                      const void* b_post, const void* gate, int64_t ldg, double alpha, const void* r, int64_t ldr,
                      void* r_out, int64_t ldro, int r_dtype, const void* w_pre, const void* b_pre, int w_dtype,
                      double eps, void* h, int64_t ldh, float* h_scales, void* stream);

/* ---------------------------------------------------------------------------
 * crvq_workspace_size -- one entry for every call's workspace size: the value
 * the per-call *_workspace_size function above returns for the same shape.
 * op selects the call; each op reads only the arguments listed (others are
 * ignored and may be 0 / NULL):
 *   CRVQ_OP_IMPORTANCE  M, N                         (crvq_channel_importance)
 *   CRVQ_OP_REORDER     N                            (crvq_reorder)
 *   CRVQ_OP_ASSIGN      n_vectors, d, K              (crvq_assign)
 *   CRVQ_OP_BEAM        n_vectors, d, n_books, Ks, beam  (crvq_assign_residual_beam)
 *   CRVQ_OP_KMEANS      n_vectors, d, K              (crvq_kmeans_update)
 *   CRVQ_OP_DEQUANT     N = n_cols                   (crvq_dequant, crvq_dequant_books)
 *   CRVQ_OP_CODE_SUMS   n_vectors, d, K              (crvq_code_sums)
 *   CRVQ_OP_REFINE      M, N, n_cols                 (crvq_refine_codes)
 *   CRVQ_OP_GEMV        M, N, K = K_base             (crvq_dequant_gemv)
 *   CRVQ_OP_HINV        N                            (crvq_hessian_inverse_diagonal)
 *   CRVQ_OP_KV_ATTENTION  n_vectors = B, d = D, M = Hq, N = Hkv, K = max_new,
 *                       n_cols = max_kv              (crvq_kv_attention)
 *   CRVQ_OP_W4_GEMV     M, N, K = T                  (crvq_w4_gemv)
 *   CRVQ_OP_W8_GEMM     M, N, K = T                  (crvq_w8_gemm)
 *   CRVQ_OP_KV_WEIGHTS, CRVQ_OP_KV_TREE_ATTENTION  as CRVQ_OP_KV_ATTENTION
 *                                                    (crvq_kv_weights, crvq_kv_tree_attention)
 *   CRVQ_OP_KV_SELECT   n_vectors = B, N = Hkv, n_cols = ld  (crvq_kv_select)
 * Returns 0 for an unknown op or a shape the call rejects (and for calls that
 * need no workspace at that shape).  Ks is a host array of n_books entries.
 */
typedef enum {
  CRVQ_OP_IMPORTANCE = 0,
  CRVQ_OP_REORDER = 1,
  CRVQ_OP_ASSIGN = 2,
  CRVQ_OP_BEAM = 3,
  CRVQ_OP_KMEANS = 4,
  CRVQ_OP_DEQUANT = 5,
  CRVQ_OP_CODE_SUMS = 6,
  CRVQ_OP_REFINE = 7,
  CRVQ_OP_GEMV = 8,
  CRVQ_OP_HINV = 9,
  CRVQ_OP_KV_ATTENTION = 10,
  CRVQ_OP_W4_GEMV = 11,
  CRVQ_OP_W8_GEMM = 12,
  CRVQ_OP_KV_WEIGHTS = 13,
  CRVQ_OP_KV_TREE_ATTENTION = 14,
  CRVQ_OP_KV_SELECT = 15
} crvq_op;
size_t crvq_workspace_size(int op, int64_t n_vectors, int64_t K, int32_t beam, int32_t n_books, int32_t d,
                           const int64_t* Ks, int64_t M, int64_t N, int64_t n_cols);

/* ---------------------------------------------------------------------------
 * crvq_pack_codes_u8 -- 8-bit storage of codes (the e = 8 code width of Sec. 3.2
 * Eq. 6 / Appendix A.1): out[i] = codes[i] & 255 for i < n.  Codes produced
 * against a book of K <= 256 codewords lie in [0, K) and are stored exactly.
 */
crvq_status crvq_pack_codes_u8(const int32_t* codes, int64_t n, uint8_t* out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CRVQ_H */
