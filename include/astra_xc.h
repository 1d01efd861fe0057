/*
 * astra_xc.h -- C ABI of the MI355X (gfx950) classifier-layer hot path of ASTRA
 * (arXiv 2409.20156): hard-negative mining by exact top-k inner product, the
 * hard+uniform negative mixture, and the sampled BCE training step with a sparse
 * SGD update of the classifier rows; dropout of the embeddings that enter a step,
 * the scores of all labels from 8-bit integers or 4-bit floating point, the check of
 * drafted labels against the classifier's probabilities, log probabilities of labels
 * under the soft-max of the scores, and the loss against a teacher's top labels.
 *
 * Conventions shared by every call
 *   - Every data pointer is a DEVICE pointer owned by the caller.  The library
 *     allocates nothing; temporary memory is a caller-provided workspace whose
 *     size is asked for first (xc_*_workspace).  Workspaces and all arrays must
 *     be 16-byte aligned, unless a call says otherwise.
 *   - Work is enqueued on the HIP stream passed as `stream` (a hipStream_t cast
 *     to void*, NULL = the default stream).  No call synchronises; results,
 *     including scalars, appear in device memory in stream order.
 *   - W is row-major L x d (one label per contiguous row), Z row-major B x d,
 *     both of type `t`.  Label ids are int32 in [0, L); any id outside that
 *     range (-1 by convention) is padding and is ignored.
 *   - Return value: XC_OK or a negative xc_status.  Shape and pointer errors are
 *     detected on the host before anything is launched; nothing is written then.
 *     After XC_EHIP, xc_last_hip_error() gives the hipError_t of this thread.
 */
#ifndef ASTRA_XC_H
#define ASTRA_XC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { XC_F32 = 0, XC_BF16 = 1 } xc_dtype;            /* storage of Z and W; sums are fp32 */
typedef enum { XC_LOSS_BCE = 0, XC_LOSS_SOFTMAX = 1 } xc_loss;

typedef enum {
    XC_OK = 0,
    XC_EINVAL = -1,      /* null or misaligned pointer, bad loss kind or margin   */
    XC_ESHAPE = -2,      /* unsupported or inconsistent sizes                     */
    XC_EWORKSPACE = -3,  /* workspace smaller than xc_*_workspace reports         */
    XC_EHIP = -4,        /* a HIP runtime call failed; see xc_last_hip_error()    */
    XC_EDTYPE = -5,      /* element type that is neither XC_F32 nor XC_BF16       */
    XC_ESCRATCH = -6     /* xc_step_static: the step's temporaries exceed
                            XC_STATIC_SCRATCH_BYTES                               */
} xc_status;

/* limits checked by the host side of every call */
#define XC_MAX_K_MINE 128      /* k_h accepted by xc_mine_negatives                */
#define XC_MAX_K_SAMPLE 1024   /* k_h accepted by xc_sample_negatives              */
#define XC_MAX_ROW_BYTES 4096  /* d * sizeof(element) accepted by xc_step          */
#define XC_MAX_CANDIDATES 16384 /* k_p + n_neg accepted by xc_step                 */
#define XC_MAX_KP 256          /* k_p accepted by xc_step                          */
#define XC_STATIC_SCRATCH_BYTES (32u << 20)  /* temporaries xc_step_static can hold    */
#define XC_MAX_D_QUANTIZED 131072 /* d accepted by the 8-bit calls: |sum| <= 127^2 d < 2^31 */
#define XC_MAX_DRAFTS 1024     /* n accepted by xc_verify_drafts                   */
#define XC_MAX_GIVEN 256       /* n accepted by xc_label_logprobs                  */
#define XC_MAX_TOP 128         /* k accepted by xc_label_logprobs                  */
#define XC_MAX_TEACHER 256     /* K accepted by xc_distill                         */

const char* xc_strerror(int status);
int xc_last_hip_error(void);
int xc_version(void);

/* ---------------------------------------------------------------------------
 * Mining (Alg. 1, the "ANNS refresh" step; Sec. 2.1 score f_l(x) = <w_l, z>).
 * Exact search stands in for the ANNS index, which the paper itself ran as a
 * control (Sec. 5.2.1 a).  For each of the Zq query rows of Z:
 *   shortlist[i*k_h + r] = id of the label with the r-th largest <z_i, w_l>,
 *   l in [0, L); equal scores are ordered by smaller id.
 *   scores[i*k_h + r]    = that inner product (fp32), if scores != NULL.
 * Products are accumulated in fp32.  The Zq x L score matrix is never stored.
 * Requires 1 <= k_h <= min(L, XC_MAX_K_MINE), d*sizeof(element) a multiple of 16.
 * A score that is NaN is never selected; a query with fewer than k_h finite
 * scores gets id -1 and score -inf in the remaining slots.
 * Every kernel sums a score's products in the same order, so ids and scores do
 * not depend on which one a call takes, bit for bit.
 * Two environment variables, read at every call, only choose between kernels
 * (for A/B timing and tests): XC_MINE_GENERAL=1
 * sends every shape through the general tile kernel; XC_MINE_ROWS=narrow or
 * wide fixes the work-item width of the kernel for bf16 rows of 128..512 bytes
 * (with either set, the kernels for few queries, the 8-bit filter and the fp16 copies of fp32 rows stay out).
 * xc_mine_workspace includes room for the 8-bit filter where a search takes it
 * (bf16 rows of 256 or 512 bytes, at least 4096 queries and 2^20 labels: up to
 * 545 MB), and for fp16 copies where a search of fp32 rows sweeps the labels on these
 * first (more than 256 queries, rows of up to 8 KB: up to 512 MiB and the queries);
 * a workspace without that room is accepted as before, and the search
 * then runs on the rows themselves throughout.
 * ------------------------------------------------------------------------- */
int xc_mine_workspace(int64_t Zq, int64_t L, int d, int k_h, xc_dtype t, size_t* bytes);
int xc_mine_negatives(const void* Z, const void* W, int64_t Zq, int64_t L, int d, int k_h,
                      xc_dtype t, int32_t* shortlist /* [Zq*k_h] out */,
                      float* scores /* [Zq*k_h] out, or NULL */,
                      void* ws, size_t ws_bytes, void* stream);

/* The same search, with the same result (bit for bit) in every case, started from the thresholds that the previous
 * search with this workspace left in it: Alg. 1 repeats the search every tau_r steps on a classifier that
 * has moved little, so the k_h-th score of a query, lowered by rel_margin * |score|, is a threshold
 * that its new k_h best labels almost always pass.  One sweep over the labels with these thresholds
 * and one selection replace the phased search.  If a query comes out of the sweep with fewer than
 * k_h candidates (the classifier moved further than the margin, or the workspace held nothing
 * useful), a flag is raised on the device for its tile of 256 queries and the call repeats the full
 * search for the flagged tiles; whatever the workspace holds, the result is exact and only the time
 * differs.  One sweep takes less time than the phases, except where the search from scratch has the
 * 8-bit filter (see above), which this one does not take: 16 384 queries on 120 M rows of 512 bytes take
 * 0.67 s from thresholds and 0.38 s from scratch.  rel_margin >= 0.  The first 32-bit word of the
 * workspace is 1 after the call if some tile needed the full search, else 0 (device memory; read it
 * after synchronising the stream). */
int xc_mine_negatives_warm(const void* Z, const void* W, int64_t Zq, int64_t L, int d, int k_h,
                           xc_dtype t, float rel_margin, int32_t* shortlist /* [Zq*k_h] out */,
                           float* scores /* [Zq*k_h] out, or NULL */,
                           void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Negative sampling (Alg. 1, hard+random step; Sec. 3.1 Idea 2; p under Eq. 2).
 * For query i of the batch, neg[i*(k_h+k_r) + ...]:
 *   slots 0..k_h-1   the shortlist row of the query, copied verbatim, logq = 0
 *                    (taken with probability one, weight 1 in Eq. 2);
 *   slots k_h..      k_r independent uniform draws from [0,L) minus H_i, H_i the
 *                    distinct in-range ids of the row (u_i of them; u_i = k_h for
 *                    a mined shortlist), logq = log(k_r / (L - u_i)): the log of
 *                    the expected number of copies of a label, so exp(-logq) is
 *                    the 1/(p k_r) factor of Eq. 2.
 * shortlist == NULL selects the warm-up phase (Alg. 1, t < tau_s): all k_h+k_r
 * slots are uniform draws from [0,L) and logq = log((k_h+k_r)/L).
 * Draw j of query i is element r = floor(u*M / 2^64) of the complement, M its
 * size, u = fmix(fmix(seed ^ K1*(i+1)) + K2*(j+1)) with fmix the splitmix64
 * finaliser, K1 = 0x9E3779B97F4A7C15, K2 = 0xD1B54A32D192ED03 (64-bit wrapping).
 * Integer arithmetic only: the ids depend on (seed, i, j, shortlist row) and on
 * nothing else.  Requires 0 <= k_h <= XC_MAX_K_SAMPLE, k_h < L, k_h + k_r >= 1.
 * ------------------------------------------------------------------------- */
int xc_sample_negatives(const int32_t* shortlist /* [B*k_h] or NULL */, int64_t B, int k_h,
                        int k_r, int64_t L, uint64_t seed,
                        int32_t* neg /* [B*(k_h+k_r)] out */,
                        float* logq /* [B*(k_h+k_r)] out */, void* stream);

/* ---------------------------------------------------------------------------
 * Negative sampling from the mixture proposal itself (Sec. 3.1, Idea 2:
 * P = (1-r) P_imp + r P_unif with P_imp proportional to the sigmoid of the stale score,
 * r = k_r/(k_h+k_r)), in stratified form.  shortlist and scores are [B*M], M >= k_h wide
 * (for example the M best labels and their scores from xc_mine_negatives).  For query i:
 *   slots 0..k_h-1   independent draws of a shortlist slot m with probability w_m / T,
 *                    w_m an integer image of 2^32*sigmoid(score) (about 1e-4 relative; the
 *                    exact recipe is in the sampler's source), T the sum over the row;
 *                    slots whose id is outside [0,L) or whose score is NaN have weight 0;
 *   slots k_h..      independent uniform draws from all of [0,L);
 *   logq             for every slot, log(k_h*W_l/T + k_r/L), W_l the total weight of the
 *                    slots holding that label: the log of the expected number of copies,
 *                    so pairs weighted by exp(-logq) estimate the sum over all L labels
 *                    without bias.  A row without any weight: all slots uniform,
 *                    logq = log((k_h+k_r)/L).
 * Random words as in xc_sample_negatives (draw j of query i); the importance draw is
 * floor(u*T/2^64) located in the running sums of the weights in slot order.  Integer
 * arithmetic only for the ids.  Requires 1 <= M <= XC_MAX_K_SAMPLE, k_h + k_r >= 1.
 * ------------------------------------------------------------------------- */
int xc_sample_negatives_mixture(const int32_t* shortlist /* [B*M] */, const float* scores /* [B*M] */,
                                int64_t B, int M, int k_h, int k_r, int64_t L, uint64_t seed,
                                int32_t* neg /* [B*(k_h+k_r)] out */, float* logq /* [B*(k_h+k_r)] out */,
                                void* stream);

/* ---------------------------------------------------------------------------
 * Hard negatives SAMPLED WITHOUT REPLACEMENT from a wider stale shortlist, a slot with probability
 * proportional to the sigmoid of its stale score (Sec. 3.1: the importance distribution of
 * Observation 2 inside the mixture of Idea 2; the paper then retrieves the top scoring labels
 * instead, which xc_sample_negatives does).  shortlist and scores are [B*M] as above, weights w_m
 * as in xc_sample_negatives_mixture.  For query i, k = min(k_h, number of slots with weight) slots
 * are chosen with inclusion probability pi_m = min(1, k' w_m / T'):
 *   - slots with k' w_m >= T' (k' slots still to choose, T' the remaining total weight) are taken
 *     for certain, all at once, and the test is repeated with what remains;
 *   - the others by systematic sampling: on the axis of the running sums of the remaining weights,
 *     in slot order and scaled by k', the points U + j T' (j < k') are marked, U = floor(u T' / 2^64)
 *     with u the query's draw 0; a slot is taken when a point falls into its interval.  No slot is
 *     taken twice and exactly k' are taken.
 *   slots 0..k-1     the labels of the chosen slots, in slot order;
 *   slots k..        independent uniform draws from all of [0,L) (draw j for slot j);
 *   logq             log(sum of pi_m over the slots holding the label + (k_h + k_r - k) / L): the
 *                    log of the expected number of copies, so pairs weighted by exp(-logq) estimate
 *                    the sum over all L labels without bias.  A row without any weight: all slots
 *                    uniform.
 * Integer arithmetic only for the ids.  Requires 1 <= M <= XC_MAX_K_SAMPLE, 0 <= k_h <=
 * XC_MAX_K_SAMPLE, k_h + k_r >= 1.
 * ------------------------------------------------------------------------- */
int xc_sample_negatives_pps(const int32_t* shortlist /* [B*M] */, const float* scores /* [B*M] */,
                            int64_t B, int M, int k_h, int k_r, int64_t L, uint64_t seed,
                            int32_t* neg /* [B*(k_h+k_r)] out */, float* logq /* [B*(k_h+k_r)] out */,
                            void* stream);

/* ---------------------------------------------------------------------------
 * One training step of the classifier layer (Alg. 1: scores on positives and
 * sampled negatives, loss of Eq. 2, SGD on W; loss averaged over the batch).
 * Per query i with score s = <z_i, w_l> on the pre-update W:
 *   BCE      loss_i = sum_{l in pos_i} log(1+e^-s)
 *                   + sum_{j} m_ij e^{-logq_ij} (s + log(1+e^-s)),
 *            m_ij = 0 if neg_ij is padding or one of pos_i (the (1-y_l) factor);
 *   SOFTMAX  logits s - logq over pos_i and the unmasked negatives,
 *            loss_i = mean over pos_i of -log softmax (a query without a
 *            positive is skipped).
 *   loss[0] = (1/B) sum_i loss_i;  dZ = d loss / d Z (fp32, [B*d]);
 *   w_l <- w_l - lr * d loss / d w_l for every label in an unmasked pair;
 *   a label in several pairs gets the summed gradient, added in a fixed order
 *   (results are bitwise reproducible run to run), and is written once (rounded
 *   to nearest even for bf16).
 *   touched[0..n_touched[0]) = those labels, ascending; no other row changes.
 *   W_rows_out, if not NULL, receives the updated rows in that order.
 *   (How: the pairs are sorted by label first.  For the BCE loss a label with a single
 *   unmasked pair gets its row updated while that pair's score is computed, w - lr g z
 *   rounded once; the other labels are summed over their pairs in pair order afterwards.
 *   After the call the first 32-bit word of the workspace holds the number of rows of
 *   the first kind, for measurements.)
 * Z and dZ must not alias.  Requires B >= 1, 0 <= k_p <= XC_MAX_KP, n_neg >= 0,
 * 1 <= k_p + n_neg <= XC_MAX_CANDIDATES, B*(k_p+n_neg) < 2^31,
 * d*sizeof(element) a multiple of 16 and <= XC_MAX_ROW_BYTES.
 * The workspace size does not depend on L.
 * ------------------------------------------------------------------------- */
int xc_step_workspace(int64_t B, int d, int k_p, int n_neg, xc_dtype t, size_t* bytes);
int xc_step(const void* Z /* [B*d] */, void* W /* [L*d], updated in place */, int64_t B,
            int64_t L, int d, const int32_t* pos /* [B*k_p] */, int k_p,
            const int32_t* neg /* [B*n_neg] */, const float* logq /* [B*n_neg] */, int n_neg,
            float lr, xc_loss kind, xc_dtype t, float* loss /* [1] out */,
            float* dZ /* [B*d] out */, int32_t* touched /* [B*(k_p+n_neg)] out */,
            int32_t* n_touched /* [1] out */, void* W_rows_out /* [B*(k_p+n_neg)*d] or NULL */,
            void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * xc_step for callers that cannot allocate device memory and have no workspace to hand over:
 * code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same
 * arguments, results and error behaviour as xc_step, without `ws`/`ws_bytes`: the step's
 * temporaries (sort pairs, coefficients, histograms, segment starts, partial sums) live in an
 * array of XC_STATIC_SCRATCH_BYTES that is part of the library's device image, one per GPU, held
 * until the process ends.  The call allocates and frees nothing; its first call on a device asks
 * the runtime once for the array's address there.  A shape for which xc_step_workspace reports
 * more than XC_STATIC_SCRATCH_BYTES is refused with XC_ESCRATCH before anything is launched
 * (the c2 and c3 benchmark shapes fit, c4 and c5 do not).  All calls on one GPU share that
 * GPU's array: calls that overlap in time on one GPU (two streams, two threads) race and give
 * wrong results; calls on one stream, or ordered by events, are safe.  Nothing needs clearing
 * between calls: every temporary is written before it is read.
 * ------------------------------------------------------------------------- */
int xc_step_static(const void* Z /* [B*d] */, void* W /* [L*d], updated in place */, int64_t B,
                   int64_t L, int d, const int32_t* pos /* [B*k_p] */, int k_p,
                   const int32_t* neg /* [B*n_neg] */, const float* logq /* [B*n_neg] */, int n_neg,
                   float lr, xc_loss kind, xc_dtype t, float* loss /* [1] out */,
                   float* dZ /* [B*d] out */, int32_t* touched /* [B*(k_p+n_neg)] out */,
                   int32_t* n_touched /* [1] out */, void* W_rows_out /* [B*(k_p+n_neg)*d] or NULL */,
                   void* stream);

/* ---------------------------------------------------------------------------
 * Rows in 8 bits.  Row i of X (d elements of type t) becomes
 *   scale[i] = m / 127 (fp32), m the row's largest magnitude;
 *   Q[i*pitch + j] = 127 x_ij / m to the nearest integer, halves to the even one,
 *   decided exactly; zeros for d <= j < pitch, pitch = d rounded up to 16.
 * A row of zeros gets scale 0; a row with an element that is not a finite number
 * gets zeros and a scale that is not a number.
 * ids == NULL: all N rows.  Else only rows ids[0..m), or ids[0..min(m, count[0]))
 * if count (device memory) is not NULL, for example the `touched` and `n_touched`
 * of the step that changed them; ids outside [0,N) are ignored, an id may occur
 * several times, the other rows of Q and scale keep their values.
 * Requires N >= 1, m >= 0, d*sizeof(element) a multiple of 16, d <= XC_MAX_D_QUANTIZED;
 * Q and scale may overlap neither each other nor an input (XC_EINVAL).
 * ------------------------------------------------------------------------- */
int xc_quantize_rows(const void* X /* [N*d] */, int64_t N, int d, xc_dtype t,
                     const int32_t* ids /* [m] or NULL */, int64_t m, const int32_t* count /* [1] or NULL */,
                     int8_t* Q /* [N*pitch] out */, float* scale /* [N] out */, void* stream);

/* ---------------------------------------------------------------------------
 * The scores of all labels from 8-bit integers: the rows of Z (type t) are brought
 * to integers p and scales a as above, and
 *   out[i*L + l] = (<p_i, q_l> * a_i) * scale[l],
 * <p, q> exact in 32-bit integers, then rounded to fp32, multiplied in fp32 and
 * rounded to out_t at the end.  Q and scale are what xc_quantize_rows gives for the
 * classifier (or for a contiguous range of its rows, from a multiple of 4 on: scale is
 * aligned to 16 bytes as all arrays are).  The workspace holds the integers of Z; it is
 * written before it is read.
 * A score does not depend on how many queries or labels are scored with it, bit for bit.
 * Requires B >= 1, 1 <= L < 2^31, B*L <= 2^40, d as above; out and the workspace may
 * overlap neither each other nor an input (XC_EINVAL).
 * ------------------------------------------------------------------------- */
int xc_scores_workspace(int64_t B, int d, size_t* bytes);
int xc_scores_quantized(const void* Z /* [B*d] */, int64_t B, int d, xc_dtype t,
                        const int8_t* Q /* [L*pitch] */, const float* scale /* [L] */, int64_t L,
                        xc_dtype out_t, void* out /* [B*L] out */, void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Rows in 4-bit floating point with shared scales (the OCP microscaling format MXFP4).  32
 * neighbouring elements of a row are a block; with m its largest magnitude,
 *   scale byte s = floor(log2 m) - 2 + 127 (0 where that is less, and for a block of zeros);
 *   element    x / 2^(s - 127) to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, halves to the
 *              neighbour whose code is even; what lies beyond 6 is 6.
 * A code is a sign, two bits of exponent and one of mantissa; element j of a row is in the low
 * (j even) or high half of byte j / 2.  Q[N * pitch / 2], scale[N * pitch / 32], pitch = d
 * rounded up to 128; zeros behind column d.  A block with an element that is not a finite number
 * gets zeros and scale 255, which makes every score with its row not a number.
 * ids, m, count as in xc_quantize_rows.  Requires 1 <= N < 2^31, m >= 0, d*sizeof(element) a
 * multiple of 16, d <= XC_MAX_D_QUANTIZED; Q and scale may overlap neither each other nor an
 * input (XC_EINVAL).  scale has to be aligned to 4 bytes only: any range of rows may be written.
 * ------------------------------------------------------------------------- */
int xc_microscale_rows(const void* X /* [N*d] */, int64_t N, int d, xc_dtype t,
                       const int32_t* ids /* [m] or NULL */, int64_t m, const int32_t* count /* [1] or NULL */,
                       uint8_t* Q /* [N*pitch/2] out */, uint8_t* scale /* [N*pitch/32] out */, void* stream);

/* ---------------------------------------------------------------------------
 * The scores of all labels from 4-bit floating point: the rows of Z (type t) are brought to 4 bits
 * as above, and
 *   out[i*L + l] = sum over blocks of 2^(s_i + s_l - 254) * (sum over the block of p_i q_l),
 * sums in fp32 in an order that depends on d alone, rounded to out_t at the end: a score does not
 * depend on how many queries or labels are scored with it, bit for bit.  Q and scale are what
 * xc_microscale_rows gives for the classifier (or a contiguous range of its rows, from any row on:
 * scale has to be aligned to 4 bytes only).  The workspace holds the 4-bit rows of Z; it is written
 * before it is read.
 * Requires B >= 1, 1 <= L < 2^31, B*L <= 2^40, d as above; out and the workspace may
 * overlap neither each other nor an input (XC_EINVAL).
 * ------------------------------------------------------------------------- */
int xc_scores_microscaled_workspace(int64_t B, int d, size_t* bytes);
int xc_scores_microscaled(const void* Z /* [B*d] */, int64_t B, int d, xc_dtype t,
                          const uint8_t* Q /* [L*pitch/2] */, const uint8_t* scale /* [L*pitch/32] */, int64_t L,
                          xc_dtype out_t, void* out /* [B*L] out */, void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Log probabilities of labels under the soft-max of their scores.  X is B rows of V scores, ld >= V
 * elements apart; a score of -infinity is a label that is not there.  With T the temperature,
 * per row: m the largest score, S = sum_v exp((x_v - m) / T),
 *   logp[b*n + j]     (x_v - m) / T - log S of label v = labels[b*n + j]; 0 for padding;
 *   entropy[b]        of the soft-max, in nats;
 *   norm[2*b], [2*b+1]  m and log S (their log-sum-exp is m / T + log S);
 *   top[b*k + r]      the label with the r-th largest score, the lower one of equal ones first;
 *   top_logp[b*k + r] its log probability.  Where the row has fewer than k labels: -1 and -infinity.
 * A row without any label: m, log S and every logp are -infinity, its entropy is 0.  A row with a
 * score that is not a number, or +infinity: log S, entropy and logp are not numbers; a score that
 * is not a number is never among the top ones.
 * Sums are fp32, in an order that depends on (B, V, k, t) and on where a row lies relative to 16 bytes.
 * Requires B >= 1, 1 <= V < 2^31, B*ld <= 2^44, 0 <= n <= XC_MAX_GIVEN, 0 <= k <= min(V, XC_MAX_TOP),
 * 1e-6 <= T <= 1e6.  labels and logp may be NULL if n = 0, top and top_logp if k = 0.  What is written
 * may overlap nothing else of the call (XC_EINVAL).
 * ------------------------------------------------------------------------- */
int xc_label_logprobs_workspace(int64_t B, int64_t V, int k, xc_dtype t, size_t* bytes);
int xc_label_logprobs(const void* X /* [B*ld] */, int64_t ld, int64_t B, int64_t V, xc_dtype t, float temperature,
                      const int32_t* labels /* [B*n] */, int n, int k, float* logp /* [B*n] out */,
                      float* entropy /* [B] out */, float* norm /* [B*2] out */, int32_t* top /* [B*k] out */,
                      float* top_logp /* [B*k] out */, void* ws, size_t ws_bytes, void* stream);

/* The gradient for the scores, from those for logp and (dentropy, or NULL) for the entropy:
 *   dX_v = (sum of dlogp over v's places in the list - p_v (G + dentropy (log p_v + entropy))) / T,
 * G the row's sum of dlogp over labels that are no padding; norm and entropy (NULL without dentropy) as
 * xc_label_logprobs gave them.  dX has rows ldd elements apart and type out_t; formed in fp32, rounded
 * once.  A row without any label gets zeros.  dX may be X if types and row distances are the same;
 * otherwise it may overlap nothing else of the call (XC_EINVAL).  Limits as above. */
int xc_label_logprobs_grad(const void* X /* [B*ld] */, int64_t ld, int64_t B, int64_t V, xc_dtype t, float temperature,
                           const int32_t* labels /* [B*n] */, int n, const float* dlogp /* [B*n] */,
                           const float* norm /* [B*2] */, const float* entropy /* [B] or NULL */,
                           const float* dentropy /* [B] or NULL */, void* dX /* [B*ldd] out */, int64_t ldd,
                           xc_dtype out_t, void* stream);

/* ---------------------------------------------------------------------------
 * The loss of scores X (as above) against a teacher of which the top labels are given, and its gradient.
 * labels[b*K ..] and teacher[b*K ..] are K labels (padding is ignored) and their logits at the temperature
 * T, that is already divided by it.  p is the soft-max of x / T over all V labels.
 *   tail = 0: q_k is the soft-max of the teacher's values over the list;
 *   tail = 1: they are log probabilities, q_k = exp(teacher_k), and the labels that are not listed are one more
 *             outcome: q_r = max(0, 1 - sum_k q_k), p_r the sum of p over them (q_r = 0 if none of them is there).
 *   loss[b] = w_b T^2 (sum_k q_k (log q_k - log p_k) + q_r (log q_r - log p_r)),
 *   dX      = its derivative: w_b T (Q p_v - q_v) for a listed label, w_b T (Q p_r - q_r) p_v / p_r for any
 *             other one, Q = sum_k q_k + q_r.
 * Terms with q = 0 are 0.  A label that occurs several times in a list is one label with the sum of its q, in the
 * loss as well as in the gradient.  weight is [B] or NULL (all 1); a row of weight 0 counts for nothing, whatever it
 * holds: loss and gradient 0; so does a row without a label in its list, or (tail = 0) with teacher values of -infinity
 * alone.  A row of scores without any label has loss infinity where q > 0, and p counts as 0 in its gradient.  Where
 * scores or teacher values are not numbers, the loss is not a number.  Sums over a row are fp32, what is formed from
 * them 64 bits.
 * dX (or NULL: the loss alone) has rows ldd elements apart and type out_t; it may be X if types and row distances
 * are the same.  Otherwise what is written may overlap nothing else of the call (XC_EINVAL).
 * Requires B, V, ld, T as above, 1 <= K <= XC_MAX_TEACHER.
 * ------------------------------------------------------------------------- */
int xc_distill_workspace(int64_t B, int64_t V, xc_dtype t, size_t* bytes);
int xc_distill(const void* X /* [B*ld] */, int64_t ld, int64_t B, int64_t V, xc_dtype t, float temperature,
               const int32_t* labels /* [B*K] */, const float* teacher /* [B*K] */, int K, int tail,
               const float* weight /* [B] or NULL */, float* loss /* [B] out */, void* dX /* [B*ldd] out, or NULL */,
               int64_t ldd, xc_dtype out_t, void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Drafted labels checked against the classifier's probabilities, so that what is
 * kept is distributed as if it had been drawn from these.  Sequence b has drafts
 * x_0, x_1, ... (the first of drafts[b*n ..] that lies outside [0,V) ends them),
 * drawn from the rows of draft_probs [B*n*V]; target is [B*(n+1)*V], one row per
 * draft and one behind the last; u [B*(n+1)] are uniform random numbers in [0,1).
 *   Draft i stands if u[b,i] * draft_probs[b,i,x_i] < target[b,i,x_i] (decided exactly).
 *   accepted[b] = a, the drafts before the first that falls, or all of them;
 *   tokens[b*(n+1) + i] = x_i for i < a; one more label at i = a; -1 behind it.
 * That label is the first v at which the running sum of w passes u[b,n] times the
 * sum of all w (the last v with w > 0 if none does), with
 *   w_v = max(0, target[b,a,v] - draft_probs[b,a,v])  where a draft fell,
 *   w_v = target[b,a,v]                               where all of them stand, or where the former are all zero;
 * -1 if these are all zero too.  Entries (or differences) that are negative,
 * infinite or not a number have w = 0.  Sums are held in 64 bits and added in an
 * order that depends on V alone.
 * draft_probs == NULL: drafts that were looked up, not drawn (probability 1 each):
 * draft i stands if u[b,i] < target[b,i,x_i], and w_v of a fallen one is the
 * target's without x_a.
 * Requires B >= 1, 0 <= n <= XC_MAX_DRAFTS, 1 <= V < 2^31; drafts may be NULL if n = 0.
 * tokens, accepted and the workspace may overlap neither each other nor an input
 * (XC_EINVAL).
 * ------------------------------------------------------------------------- */
int xc_verify_workspace(int64_t B, int64_t V, size_t* bytes);
int xc_verify_drafts(const int32_t* drafts /* [B*n] */, int64_t B, int n, int64_t V,
                     const void* target /* [B*(n+1)*V] */, const void* draft_probs /* [B*n*V] or NULL */, xc_dtype t,
                     const float* u /* [B*(n+1)] */, int32_t* tokens /* [B*(n+1)] out */,
                     int32_t* accepted /* [B] out */, void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Dropout without a stored mask: Y_ij = X_ij * 65536 / (65536 - T) or, if dropped, 0
 * (whatever X_ij is), with T = floor(65536 rate + 1/2).  Element (i, j) is dropped if
 * field j mod 4 (16 bits each, the lowest first) of word g = j / 4 (rounded down) is less than T,
 *   word = fmix(fmix((seed ^ K3) ^ K1*(row0+i+1)) + K2*(g+1)),
 * fmix, K1, K2 as in xc_sample_negatives, K3 = 0x64726F706F757431 (a step may use one
 * seed for its samples and its dropout).  The gradient of dropout is the same map with
 * the same rate, seed and row0, applied to the gradient.  The product is formed in
 * fp32 and rounded once.  X and Y may be the same array if their types are; arrays
 * that overlap otherwise are refused.
 * Requires B >= 1, 1 <= d < 2^31, B*d <= 2^40, rate >= 0, T <= 65535, row0 >= 0.
 * ------------------------------------------------------------------------- */
int xc_dropout(const void* X /* [B*d] */, xc_dtype t, int64_t B, int64_t d, float rate, uint64_t seed,
               int64_t row0, void* Y /* [B*d] out */, xc_dtype out_t, void* stream);

/* ---------------------------------------------------------------------------
 * Measurement aid (no passage of the paper: used by the benchmark to time each
 * kernel with HIP events on the stream it is launched on).  While enabled, every
 * kernel launch of the calls above is bracketed by a pair of events.
 * xc_profile_collect() waits for the recorded events (host-side wait), adds the
 * elapsed times to per-kernel totals and returns the number of kernel names;
 * xc_profile_get(i, ...) reads total milliseconds and launch count of name i;
 * xc_profile_reset() clears the totals.  Off by default; when off the calls
 * above record no events.  Not thread-safe against concurrent launches.
 * ------------------------------------------------------------------------- */
int xc_profile_enable(int on);
int xc_profile_collect(void);
int xc_profile_get(int i, const char** name, double* total_ms, int64_t* launches);
int xc_profile_reset(void);

/* Measurement aid: a plain device-to-device copy kernel (reads `bytes`, writes `bytes`;
 * both pointers device memory, 16-byte aligned, `bytes` a multiple of 16, buffers must not
 * overlap).  The benchmark launches it beside the library's kernels in hardware-counter runs
 * so that the traffic counters can be scaled by a kernel of known size.  Asynchronous on
 * `stream`.  XC_EINVAL on null or misaligned arguments. */
int xc_copy_probe(void* dst, const void* src, size_t bytes, void* stream);

/* Measurement aid: a register-resident loop of bf16 MFMA instructions (no memory traffic) on
 * 256 workgroups of 8 waves, `iters` (1 .. 2^20) rounds of 8 products per wave.  With
 * random_operands != 0 the operands are pseudo-random bf16 values, else zero: the rate the chip
 * sustains depends on the operand values through its power limit, and the benchmark reports it
 * beside the published peak.  `out` is device memory for 256*512 floats (a checksum, so that the
 * loop is not removed); `*flop` (host pointer, may be NULL) receives the floating-point
 * operations of one launch.  Asynchronous on `stream`. */
int xc_mfma_probe(float* out, int iters, int random_operands, double* flop, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ASTRA_XC_H */
