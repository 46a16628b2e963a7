/*
 * atomo.h - C ABI of the MI355X (gfx950) ATOMO gradient encoder / decoder.
 *
 * ATOMO ("ATOMO: Communication-efficient Learning via Atomic Sparsification",
 * arXiv 1806.04090) writes a stochastic gradient in an atomic decomposition
 * g = sum_i lambda_i a_i with unit-norm atoms (Section 3), draws independent
 * t_i ~ Bernoulli(p_i) and sends only the kept atoms, rescaled:
 *
 *     g_hat = sum_i (lambda_i t_i / p_i) a_i                       (eq. (vhat))
 *
 * with the p that minimises the variance under a sparsity budget sum p_i = s
 * (eq. (opt_prob1), solved by Algorithm 1).  Two decompositions are built:
 * entry-wise (a_i = e_i, lambda_i = g_i) and, for a gradient viewed as a
 * matrix, the singular value decomposition (atoms u_i v_i^T, lambda_i =
 * sigma_i; Section 5, "Spectral-ATOMO").
 *
 * Conventions for every entry point
 *  - All data pointers are DEVICE pointers (HIP global memory on the device the
 *    context was created for) unless a parameter says "host".  Descriptor
 *    structs (atomo_mat, atomo_svd_msg, atomo_ew_msg) and arrays of them are
 *    HOST memory; they are read during the call and may be freed afterwards.
 *  - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *    Work is enqueued on it; calls do not wait for the results.  Results are
 *    valid once the stream has reached the end of the enqueued work.
 *    Descriptor tables travel to the device through a ring of eight pinned
 *    staging buffers owned by the context: a call that needs a buffer whose
 *    previous copy (eight uploads ago) has not been executed yet waits for
 *    that copy, and for nothing else.  The SVD encoder, the SVD decoder and
 *    atomo_probabilities each keep the four sets of tables used last on the device, and skip the
 *    upload when a call, on the same stream, describes exactly the buffers of
 *    one of them (a training loop, or one that takes a few sets of buffers in
 *    turn): the tables hold addresses and sizes, never data.
 *  - The caller owns every input, output and message buffer.  Inputs are never
 *    modified.  The context owns a device workspace that grows on demand
 *    (growing it allocates, which synchronises the device; atomo_reserve
 *    pre-sizes it).  One context must not be used from two streams at once.
 *  - Return value: ATOMO_OK or a negative atomo_status.  Nothing throws, exits
 *    or prints.  Conditions that are only known on the GPU (a message that did
 *    not fit its capacity, a Jacobi run that hit the sweep limit) do not fail
 *    the call; they are latched on the device and read back by atomo_status.
 *  - Random numbers: Philox4x32-10 (Salmon et al., SC'11).  Atom i of a call
 *    with (seed, stream_id) uses output word i mod 4 of the block with counter
 *    (i div 4 [64 bit], stream_id [64 bit]) and key seed [64 bit];
 *    u = (word >> 8) * 2^-24 and the atom is kept iff u < p_i, compared in
 *    single precision.  The paper fixes only t_i ~ Bernoulli(p_i) (Section 3).
 */
#ifndef ATOMO_H
#define ATOMO_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum atomo_status_code {
    ATOMO_OK = 0,
    ATOMO_EINVAL = -1,     /* null pointer, non-positive size, s <= 0 or NaN, inconsistent shapes  */
    ATOMO_ECAPACITY = -2,  /* (atomo_status only) more atoms were kept than a message could hold    */
    ATOMO_ENOCONV = -3,    /* (atomo_status only) the Jacobi SVD stopped at the sweep limit         */
    ATOMO_EHIP = -4,       /* a HIP runtime call failed; atomo_last_hip_error gives its code        */
    ATOMO_ENOMEM = -5,     /* the workspace, or host memory for the plan of a call, could not be allocated */
    ATOMO_ETOOLARGE = -6   /* atomo_encode_entrywise_noalloc: n exceeds what its fixed scratch holds */
} atomo_status_code;

enum { ATOMO_KIND_SVD = 0, ATOMO_KIND_ENTRYWISE = 1, ATOMO_KIND_LQ = 2 };

typedef struct atomo_ctx atomo_ctx;   /* opaque: device, workspace, latched device-side flags */

/* A gradient viewed as a matrix (Section 5; Fig. 1: a conv gradient [out,in,k,k] is the row-major
 * out x (in*k*k) matrix it already is in memory).  rows x cols, row stride ld >= cols, float32. */
typedef struct atomo_mat {
    int32_t rows, cols;
    int64_t ld;
    const float* data;               /* device */
} atomo_mat;

/* One Spectral-ATOMO message: the kept singular triplets of one matrix with their weights (what a worker
 * sends to the parameter server in Section 6).  Atom index 0 is the largest singular value.
 * All pointers are caller-owned device memory. */
typedef struct atomo_svd_msg {
    int32_t rows, cols;              /* shape of the encoded matrix                                   */
    int32_t capacity;                /* room for this many kept atoms, 1 <= capacity                 */
    int32_t* count;                  /* [1]  number of atoms kept (may exceed capacity: see status)  */
    int32_t* idx;                    /* [capacity] atom indices, ascending                           */
    float*   w;                      /* [capacity] weights sigma_i / p_i; NULL selects the folded form below */
    float*   U;                      /* [capacity][rows]  U[k*rows + i] = (u of k-th kept atom)_i, unit norm;  */
                                     /* folded form (w == NULL): (sigma_i / p_i) u, the weight carried by the   */
                                     /* left vector (Section 6), rows + cols reals per atom as in the cost      */
                                     /* s(n+m) of Table "matrix_sparse"                                         */
    float*   V;                      /* [capacity][cols]  V[k*cols + j] = (v of k-th kept atom)_j, unit norm */
} atomo_svd_msg;

/* One entry-wise ATOMO message: kept coordinates, ascending, with values g_i / p_i. */
typedef struct atomo_ew_msg {
    int64_t n;                       /* length of the encoded gradient, 0 < n < 2^32                 */
    int64_t capacity;                /* room for this many pairs                                     */
    int64_t* count;                  /* [1]  number of pairs kept (may exceed capacity: see status)  */
    uint32_t* idx;                   /* [capacity] kept coordinates, ascending: decoding searches them */
    float* val;                      /* [capacity] g_i / p_i                                         */
} atomo_ew_msg;

/* One l_q-quantised gradient (Section 4: L_q(g)_i = |g|_q sign(g_i) zeta_i; q = 2 is 1-bit QSGD, q = inf
 * TernGrad): the kept coordinates with their signs, and the one magnitude they all share. */
typedef struct atomo_lq_msg {
    int64_t n;                       /* length of the encoded gradient, 0 < n < 2^31                 */
    int64_t capacity;                /* room for this many kept coordinates                          */
    int64_t* count;                  /* [1]  number kept (may exceed capacity: see status)           */
    uint32_t* idx;                   /* [capacity] kept coordinates, ascending, in bits 0..30; bit 31 is set where g_i < 0 */
    float* norm;                     /* [1]  |g|_q                                                   */
} atomo_lq_msg;

/* Options of the SVD encoder; pass NULL for the defaults.
 *
 * Matrices of 33 .. 640 vectors on the shorter side, with a budget s of at most 32 atoms, are first solved directly: the
 * Gram matrix in double precision, its eigenvalues, and singular vectors of the kept atoms only.  The Jacobi iteration
 * that the options below describe takes over for a matrix with singular values at or under twice the fp32 floor (3.8e-6 of the
 * largest; gradients of low rank, other than through rows that are zero) or with kept atoms whose vectors it cannot
 * separate (singular values that agree to eight digits, fewer digits for values far below the largest); for every other
 * size and budget; and for every matrix of a call that sets stop_cosine, max_inner_sweeps, inner_reduction, full_period or
 * block_order, or a max_sweeps under the default. */
typedef struct atomo_svd_options {
    int32_t max_sweeps;              /* default 16 (0 = default).  Noise-dominated gradients take 5 to 7 sweeps,   */
                                     /* exactly low-rank ones (rank 128 in 600 x 700) 12, singular values graded   */
                                     /* over two decades 11, three 14, five 16; a matrix half of whose rows are    */
                                     /* copies of the other half 16.  Every sweep allowed costs launches even when */
                                     /* unused (they return at once, about 0.08 ms per sweep for 512-row           */
                                     /* matrices).  Hitting the limit reports ATOMO_ENOCONV; the message is then   */
                                     /* still an exact decomposition of the input, with atoms that are not yet     */
                                     /* orthogonal to the tolerance.                                               */
                                     /* No effect on matrices with min(rows, cols) <= 32 (the [x*y/2, 2*k*k]        */
                                     /* reshape of Section 6): two passes over the data, the r x r problem solved  */
                                     /* in double precision by one workgroup                                       */
    float   stop_cosine;             /* default 1e-4 (0 = default): stop after the first sweep whose largest */
                                     /* |<a_i,a_j>| / (|a_i||a_j|), measured before rotating, is below; matrices   */
                                     /* that iterate on their Gram matrix stop once the Gram matrix formed afresh  */
                                     /* from the rotated data has no cosine above it                               */
    int32_t max_inner_sweeps;        /* most Jacobi sweeps per 64x64 block-pair problem; 0 = default: 1 for the   */
                                     /* matrices that iterate on their Gram matrix (481 or more vectors on the    */
                                     /* shorter side), 2 for the others                                            */
    float   inner_reduction;         /* a block-pair problem stops sweeping once its largest |cos| is below        */
                                     /* inner_reduction x the value it started at; 0 = default: 0.1 (0.01 for the  */
                                     /* matrices that iterate on their Gram matrix, which matters only with        */
                                     /* max_inner_sweeps above 1)                                                  */
    int32_t full_period;             /* default 12 (0 = default): a block-pair problem rotates all 2016 index    */
                                     /* pairs in the rounds of an outer sweep whose number is a multiple of this */
                                     /* and only the 1024 pairs that couple its two blocks in the other rounds;  */
                                     /* 1: all 2016 pairs in every round                                         */
    int32_t block_order;             /* matrices with 481 or more vectors on the shorter side (they iterate on the */
                                     /* r x r Gram matrix): 0 (default) pairs the 32-row blocks of every round by  */
                                     /* the weight of their off-diagonal blocks, heaviest first (dynamic ordering  */
                                     /* of the parallel block-Jacobi method; a matrix falls back to the tournament */
                                     /* once a row has shrunk by 1e-5, as in gradients of low rank); 1 keeps the   */
                                     /* fixed round-robin tournament that the smaller matrices use throughout.     */
                                     /* Either order gives the same result from call to call                      */
    const uint64_t* stream_ids;      /* HOST array of n_mats Philox stream ids, or NULL for stream_base + j: lets */
                                     /* one call encode the gradients of several workers (stream = worker, layer) */
                                     /* and produce the messages that separate calls would                        */
    int32_t adaptive;                /* 0 (default): the launches of all max_sweeps sweeps are enqueued.  k > 0:  */
                                     /* for a training loop that encodes the same layer set step after step. The  */
                                     /* context remembers how many sweeps the matrices of earlier calls with the  */
                                     /* same shapes took (the most recent call that has finished; at most four    */
                                     /* such calls are in flight: a fifth waits for the oldest before it is       */
                                     /* enqueued) and enqueues that many + k, at most max_sweeps, separately for  */
                                     /* the matrices that iterate on their Gram matrix and for the others; a call */
                                     /* that used up such a reduced limit is followed by one with the full limit. */
                                     /* A matrix that needs more sweeps than were enqueued is reported through    */
                                     /* ATOMO_ENOCONV exactly as at max_sweeps (its message is still an exact,    */
                                     /* unbiased decomposition); gradients change slowly from step to step, so    */
                                     /* k = 1 or 2 rarely meets that.  The matrices that iterate on their Gram     */
                                     /* matrix confirm convergence on a Gram matrix formed afresh from the rotated */
                                     /* data, at a sweep boundary; the context also remembers after how many sweeps */
                                     /* the first of them asked for that, and a call enqueues those launches only  */
                                     /* from k sweeps before: a matrix that is ready sooner sweeps on until then.  */
                                     /* A matrix that was solved directly in that earlier call gets no iteration   */
                                     /* enqueued.  One that would have needed it is reported through ATOMO_ENOCONV, */
                                     /* and the call after it enqueues both; its message holds the direct result,  */
                                     /* or, if a kept vector of that was not accepted, atoms of another exact      */
                                     /* decomposition: the vectors of the shorter side, e_i (a_i / |a_i|)^T, drawn  */
                                     /* with Algorithm 1 on their norms, so it is still an unbiased estimate.  A   */
                                     /* matrix that was not solved directly iterates without another attempt in    */
                                     /* the next eight calls                                                       */
} atomo_svd_options;

/* -------- context ------------------------------------------------------------------------------ */

/* Creates a context on HIP device `device`.  *out is set on success.
 * A context owns one workspace and (for the SVD encoder) three helper streams that are forked from and joined
 * back into the caller's stream inside a call that uses them: calls that share a context must be issued from one host
 * thread at a time and onto one stream, or onto streams the caller has ordered among themselves; use one
 * context per concurrent stream. */
int atomo_create(atomo_ctx** out, int device);
int atomo_destroy(atomo_ctx* ctx);

/* Makes sure the workspace holds at least `bytes`; atomo_svd_workspace_bytes /
 * atomo_entrywise_workspace_bytes say how much a call will need (host-side arithmetic only).  An SVD encode
 * that cannot get that much does without the direct solution, which takes up to twice what the iteration does;
 * atomo_reserve makes it try again. */
int atomo_reserve(atomo_ctx* ctx, size_t bytes);
int atomo_svd_workspace_bytes(const atomo_mat* mats /*host*/, int n_mats, size_t* bytes /*host*/);
int atomo_entrywise_workspace_bytes(int64_t n, size_t* bytes /*host*/);

/* Waits for `stream`, then reports and clears what the GPU latched since the last call:
 * ATOMO_OK, ATOMO_ECAPACITY, ATOMO_ENOCONV, ATOMO_EINVAL (an entry-wise or l_q message whose coordinates do not ascend
 * was decoded: the output is not its sum; or a token named no row of its table) or ATOMO_EHIP.  If sweeps is not NULL it receives the
 * largest number of Jacobi sweeps any matrix of the last atomo_encode_svd took. */
int atomo_status(atomo_ctx* ctx, void* stream, int32_t* sweeps /*host, optional*/);
int atomo_last_hip_error(const atomo_ctx* ctx);

/* Waits for `stream`, then copies the number of Jacobi sweeps each matrix of the last
 * atomo_encode_svd took into sweeps[0 .. n_mats) (HOST) and, if refreshes is not NULL, how many
 * times the full Gram matrix of the matrix was formed from the data (matrices of 33 .. 480 rows
 * iterate directly on the data: 0 below 225 rows, from there on the number of whole-matrix
 * convergence checks near the end).  A matrix that was solved directly, or has at most 32 rows or columns, counts as one sweep and two passes over
 * the data (the Gram matrix, and the vectors of the longer side).  n_mats must match that call; the counts stay readable until the
 * next atomo_encode_svd on the context. */
int atomo_svd_sweeps(atomo_ctx* ctx, void* stream, int32_t* sweeps /*host*/, int32_t* refreshes /*host, optional*/,
                     int n_mats);
const char* atomo_strerror(int status);

/* -------- the method --------------------------------------------------------------------------- */

/*
 * Algorithm 1 ("ATOMO probabilities", Section 3; closed form in the KKT appendix, eq. (p_i)).
 * For each of n_seg independent segments lambda[offsets[k] .. offsets[k+1]) computes
 *     p = argmin sum lambda_i^2 / p_i   s.t.  0 <= p_i <= 1,  sum p_i = s
 * i.e. p_i = 1 for the n_s largest |lambda_i| and p_i = |lambda_i| (s - n_s) / sum_{rest} |lambda_j|
 * for the rest, n_s the smallest count that keeps every p_i <= 1.  lambda may be in any order and
 * of any sign; p comes back in the same order.  lambda_i = 0 gets p_i = 0; if s >= #nonzeros every
 * nonzero gets 1 (then sum p < s).
 *   lambda, p : device float32 [offsets[n_seg]]      offsets : HOST int64 [n_seg + 1], ascending
 *   s > 0 (a real number, the same for every segment)
 */
int atomo_probabilities(atomo_ctx* ctx, const float* lambda, const int64_t* offsets /*host*/, int n_seg,
                        double s, float* p, void* stream);

/*
 * Spectral-ATOMO encode (Section 5; eq. (vhat) on the singular value decomposition).
 * For each matrix j: thin SVD  G_j = sum_i sigma_i u_i v_i^T  (sigma descending), p = Algorithm 1
 * on sigma with budget s, t_i ~ Bernoulli(p_i) from Philox stream (seed, stream_base + j), and the
 * message = kept atoms (index, sigma_i / p_i, u_i, v_i) in ascending index.
 *   mats, msgs : HOST arrays of n_mats descriptors; msgs[j].rows/cols must equal mats[j].rows/cols.
 *   sigma_out, p_out : optional device float32, all matrices concatenated, min(rows, cols) values
 *                      each, descending sigma order (atom order).  Pass NULL to skip.
 * Supported shapes: min(rows, cols) <= 2048, max(rows, cols) <= 2^30.
 */
int atomo_encode_svd(atomo_ctx* ctx, const atomo_mat* mats, int n_mats, double s,
                     uint64_t seed, uint64_t stream_base, const atomo_svd_options* opt /*host, optional*/,
                     const atomo_svd_msg* msgs, float* sigma_out, float* p_out, void* stream);

/*
 * Entry-wise ATOMO encode (Section 3 with the standard basis; Section 4 shows 1-bit QSGD and
 * TernGrad are this with s = |g|_1/|g|_2 and s = |g|_1/|g|_inf).  lambda_i = g_i, p = Algorithm 1,
 * coordinate i is kept iff u_i < p_i (Philox stream (seed, stream_id)) and stored as
 * (i, g_i / p_i), ascending in i.
 *   g : device float32 [msg->n];  p_out : optional device float32 [msg->n].
 */
int atomo_encode_entrywise(atomo_ctx* ctx, const float* g, double s, uint64_t seed, uint64_t stream_id,
                           const atomo_ew_msg* msg /*host*/, float* p_out, void* stream);

/*
 * atomo_encode_entrywise for callers that cannot allocate device memory: code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc.  Same arguments, same message, bit for bit; the scratch
 * memory of the kernels (water-level search state, per-chunk counts, keep and undecided bits) is a fixed array
 * of 5 MiB that the library holds on every GPU it runs on until the process ends, instead of the context's
 * growable workspace.  The call allocates nothing (no hipMalloc, hipFree, event or stream creation), on any
 * path.
 *   n = msg->n is limited to 2^24 = 16,777,216 elements; a longer gradient returns ATOMO_ETOOLARGE and
 *   nothing is enqueued.
 *   All calls on one GPU share that GPU's array, whatever their context or stream: two such calls whose
 *   kernels overlap in time race on it.  Issue them on one stream, or order the streams.  The array keeps
 *   the previous call's contents; the call clears what it needs cleared itself, with a kernel.
 *   atomo_create looks up the array's address on the context's device, so this call does no set-up of its own.
 *   Event bracketing (atomo_profile_enable) does not cover this call.
 */
int atomo_encode_entrywise_noalloc(atomo_ctx* ctx, const float* g, double s, uint64_t seed, uint64_t stream_id,
                                   const atomo_ew_msg* msg /*host*/, float* p_out, void* stream);

/*
 * l_q quantisation (Section 4, Theorem (lqgrad)): p_i = |g_i| / |g|_q, the variance-optimal entry-wise
 * probabilities for the budget s = |g|_1 / |g|_q, computed without Algorithm 1 (every g is balanced for
 * that budget).  Coordinate i is kept iff u_i < p_i (Philox stream (seed, stream_id)); a kept coordinate
 * decodes to sign(g_i) |g|_q.  q > 0; pass INFINITY for the maximum norm (TernGrad), 2 for 1-bit QSGD.
 *   g : device float32 [msg->n];  p_out : optional device float32 [msg->n].
 */
int atomo_encode_lq(atomo_ctx* ctx, const float* g, double q, uint64_t seed, uint64_t stream_id,
                    const atomo_lq_msg* msg /*host*/, float* p_out, void* stream);

/*
 * Decode (eq. (vhat)): out = scale * sum over the n_msgs messages of sum_k w_k a_k.  With
 * scale = 1/P and the P workers' messages this is the parameter server's averaged gradient
 * (Section 2).  `out` is overwritten.
 *   kind = ATOMO_KIND_SVD:       msgs is a HOST array of n_msgs atomo_svd_msg with equal rows/cols;
 *                                out is the dense rows x cols row-major matrix with row stride ld.
 *   kind = ATOMO_KIND_ENTRYWISE: msgs is a HOST array of n_msgs atomo_ew_msg with equal n;
 *                                out is the dense vector of n floats (ld is ignored).
 *   kind = ATOMO_KIND_LQ:        msgs is a HOST array of n_msgs atomo_lq_msg with equal n; out as above.
 * A message whose count exceeds its capacity contributes its first `capacity` atoms.  The coordinates of
 * an entry-wise or l_q message have to ascend, as encoders write them; others are reported by atomo_status.
 * The sum is formed in a fixed order (entry-wise and l_q messages one after the other, in the order
 * given), so the same messages decode to the same bits in every run.
 */
int atomo_decode(atomo_ctx* ctx, int kind, const void* msgs, int n_msgs, float scale,
                 float* out, int64_t ld, void* stream);

/*
 * Batched form of the SVD decode for a whole layer set: for each of n_out outputs, the messages
 * msgs[first[o] .. first[o+1]) are summed into outs[o] as atomo_decode does, in one launch.
 *   msgs : HOST array;  first : HOST int32 [n_out + 1];  outs : HOST array of n_out device pointers;
 *   lds  : HOST int64 [n_out].
 */
int atomo_decode_svd_batch(atomo_ctx* ctx, const atomo_svd_msg* msgs, const int32_t* first, int n_out,
                           float scale, float* const* outs, const int64_t* lds, void* stream);

/*
 * The parameter server's step (Section 2: w_{k+1} = w_k - gamma g_hat; Section 6: the PS combines the
 * workers' messages and updates the model with the average gradient) without materialising the gradient:
 *     params[o] += alpha * sum over msgs[first[o] .. first[o+1]) of sum_k w_k u_k v_k^T
 * for each of n_out parameter matrices, in one launch; alpha = -gamma / P for P workers.  Arguments as for
 * atomo_decode_svd_batch, except that params[o] (device, rows x cols, row stride lds[o]) is read and updated.
 */
int atomo_apply_svd_batch(atomo_ctx* ctx, const atomo_svd_msg* msgs, const int32_t* first, int n_out,
                          float alpha, float* const* params, const int64_t* lds, void* stream);

/* -------- the training step around the method ------------------------------------------------------
 *
 * What stands before and behind an encode / decode in the training of a language model: the embedding lookup with its
 * gradient, which is a sum of row atoms e_token dy^T from the start, and the optimizer's step on the decoded gradients.
 * The paper's own step is plain SGD (atomo_apply_svd_batch).
 *
 * Buffers that a call writes may not overlap others of that call.  Pointers need the alignment of their element type
 * only.  All calls below may be captured into a graph, atomo_adamw_create and atomo_adamw_destroy apart.  Those that need the context's
 * workspace (atomo_embedding_grad) do not grow it then: reserve it before (ATOMO_ENOMEM otherwise).  A block of
 * workspace that a captured call uses stays allocated until atomo_destroy, also when a later call makes the context
 * take a larger one; graphs of one context share it and must not run at the same time.  A captured call holds the
 * numbers it was given; those that change from replay to replay come from device memory (step_dev, lr_dev). */

enum { ATOMO_F32 = 0, ATOMO_BF16 = 1, ATOMO_F16 = 2 };

/* A row-major matrix of ATOMO_F32 / BF16 / F16 elements: row stride ld >= cols elements (an input's may also be 0: every
 * row the same; the stride of a single row is not looked at). */
typedef struct atomo_rows {
    int64_t rows;                    /* < 2^31 - 1; 0 rows only where stated                          */
    int32_t cols, type;              /* 1 <= cols <= 2^30                                             */
    int64_t ld;
    void* data;                      /* device                                                        */
} atomo_rows;

/* A flat list of tokens, row numbers of the table.  Tokens that equal `padding` (any number, also one outside of the
 * table) stand for no row. */
typedef struct atomo_tokens {
    int64_t n;                       /* 0 <= n < 2^31                                                 */
    const void* data;                /* device: int32 or int64 [n]                                    */
    int32_t bytes;                   /* 4 or 8 per token                                              */
    int64_t padding;
} atomo_tokens;

/*
 * Embedding lookup: out[t] = scale * table[tokens[t]], formed in fp32 and rounded once; zeros for padding.
 *   out : tokens->n rows (at least; rows behind stay as they are) of table->cols columns, any of the types.
 * A token outside of the table that is not padding gives zeros as well, and atomo_status reports ATOMO_EINVAL.
 */
int atomo_embedding(atomo_ctx* ctx, const atomo_rows* table /*host*/, const atomo_tokens* tokens /*host*/, float scale,
                    const atomo_rows* out /*host*/, void* stream);

/*
 * Its gradient: grad[r] = (accumulate ? grad[r] : 0) + scale * sum over the t with tokens[t] = r of dy[t], summed in
 * fp32 and rounded once to grad's type.  Without accumulate every row of grad is written, those that no token names as
 * zeros; with it such rows are not touched.  The order of the sum depends on the sizes, types and tokens alone, so the
 * same call gives the same bits in every run.
 *   dy : tokens->n rows (at least) of grad->cols columns.
 * Tokens outside of the table are left out, and reported as by atomo_embedding.
 */
int atomo_embedding_grad(atomo_ctx* ctx, const atomo_tokens* tokens /*host*/, const atomo_rows* dy /*host*/, float scale,
                         const atomo_rows* grad /*host*/, int accumulate, void* stream);

/* Workspace of an atomo_embedding_grad of n_tokens into rows x cols. */
int atomo_embedding_workspace_bytes(int64_t n_tokens, int64_t rows, int32_t cols, size_t* bytes /*host*/);

/*
 * AdamW over many tensors.  One step, t = 1, 2, ...:
 *     g' = c g,  c = grad_scale * min(1, max_norm / *grad_norm)             (c = grad_scale without a norm to clip to)
 *     m = beta1 m + (1 - beta1) g'        v = beta2 v + (1 - beta2) g' g'
 *     param -= lr lr_mult / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps) + lr lr_mult weight_decay param
 * in fp32 (eps rounded to it), every product and sum of m and v rounded by itself; and, if it has one, copy = param rounded to
 * copy_type.  0 / 0, of an element without a gradient so far where eps is 0, counts as 0.
 * Where *grad_norm is not finite the step does nothing at all (the caller counts t on only where it was finite).
 *
 * States m and v are float32, or 8 bits per element with a scale for each block of 128 consecutive elements.  The scale
 * is a byte S, the biased fp32 exponent of the block's largest finite |m| (v); E = max(S, 1) - 127.  m is a code of
 * sign, 4 exponent bits (bias 7) and 3 mantissa bits times 2^(E - 7), its NaN being 0x7f; v, which is never negative, has
 * 5 exponent bits (bias 15) and 3 mantissa bits, times 2^(E - 15), its NaN being 0xff.  Both are rounded at random such
 * that their expectation is the value itself (to the nearest code, v could not follow: a step moves it by a
 * thousandth, a code by an eighth): of an |x| that lies f steps of 2^-16 above a code, the next one is taken iff
 * r + f >= 2^16, r uniform in 0 .. 2^16 - 1.  A v that is not zero keeps a code that is not zero.  Infinite and NaN
 * values become NaN.  Element i of the tensor whose predecessors in the plan fill b blocks takes word i mod 4 of the Philox block with
 * counter (32 b + i div 4, t) and key seed: r is its low half for m, its high half for v.  These are the words that an encoder
 * draws for the coordinates of a message with the same seed and stream_id = t.  A coordinate that it keeps with probability p has
 * a word below p 2^32, so that the r of its v would be below p 2^16, and its v rounded down but for a share of p: the expectation holds only
 * if the seed is none of those of the messages that the gradients come from (whose stream ids may equal t).  Where a program has one seed for all,
 * this one is ATOMO_ADAMW_SEED ^ that seed.
 */
#define ATOMO_ADAMW_SEED 0x6164616d775f6d76ull

typedef struct atomo_adamw_tensor {
    int64_t n;                       /* elements, 0 < n < 2^40                                        */
    float* param;                    /* [n]; NULL (in every tensor of a plan): atomo_adamw_grad_norm only */
    const void* grad;                /* [n] of grad_type                                              */
    void* m;                         /* [n] float32, or codes (uint8) if the scales are not NULL      */
    void* v;
    uint8_t* m_scale;                /* [ceil(n / 128)], or NULL, both                                */
    uint8_t* v_scale;
    void* copy;                      /* [n] of copy_type, or NULL                                     */
    int32_t grad_type, copy_type;
    float lr_mult, weight_decay;     /* finite, not negative                                          */
} atomo_adamw_tensor;

typedef struct atomo_adamw_options {
    double lr, beta1, beta2, eps;    /* lr >= 0, 0 <= beta < 1, eps >= 0, finite                      */
    int64_t step;                    /* t >= 1 (not looked at if step_dev is not NULL)                */
    const int64_t* step_dev;         /* device [1], optional: t (below 1 is taken for 1)              */
    const float* lr_dev;             /* device [1], optional: taken instead of lr                     */
    const float* grad_norm;          /* device [1], optional: see above                               */
    float max_norm;                  /* > 0: clip to it (needs grad_norm); 0: do not clip             */
    float grad_scale;                /* finite                                                        */
    uint64_t seed;                   /* of the rounding of 8-bit states: not one of an encoder's      */
} atomo_adamw_options;

typedef struct atomo_adamw atomo_adamw;   /* opaque: the tensors of a model, described once on the device */

/* Describes the tensors (HOST array of n, read during the call) on the context's device; waits for the device.  Memory that a
 * step writes may overlap nothing else in the plan: ATOMO_EINVAL, as for more than 1.6e7 pieces of at most 2048 elements (3.4e10
 * elements).  Contents stay the caller's: nothing of them is kept.
 * One plan must not be used from two streams at once.  Destroy it before its context, and after the graphs that hold its
 * calls. */
int atomo_adamw_create(atomo_ctx* ctx, const atomo_adamw_tensor* tensors /*host*/, int n, atomo_adamw** out);
int atomo_adamw_destroy(atomo_ctx* ctx, atomo_adamw* plan);

/* norm[0] = |grad_scale| * the Euclidean norm of all gradients of the plan, summed in double precision in a fixed order.
 * norm : device [1]. */
int atomo_adamw_grad_norm(atomo_ctx* ctx, const atomo_adamw* plan, float grad_scale, float* norm, void* stream);

int atomo_adamw_step(atomo_ctx* ctx, const atomo_adamw* plan, const atomo_adamw_options* opt /*host*/, void* stream);

/* What 8-bit states stand for: out[i] = code times scale, formed in fp32 and rounded to `type` (what a step has
 * written is exact in ATOMO_F32, and in ATOMO_BF16 down to its smallest normal number).  n elements from the start of a block, 0 < n < 2^34. */
enum { ATOMO_STATE_M = 0, ATOMO_STATE_V = 1 };
int atomo_state8_unpack(atomo_ctx* ctx, int which, const uint8_t* codes, const uint8_t* scales, int64_t n, int type,
                        void* out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ATOMO_H */
