/*
 * grim_lm.h -- operators of a recurrent language model around the BCR products of grim_bcr.h: the layer norm between
 * layers, a gated linear recurrence that trains over long sequences and serves token by token, distillation of a pruned
 * student from its teacher's top logits, and the rules applied to the logits of a served step.
 *
 * Conventions of grim_bcr.h: functions return a grim_status and never throw or abort; *_dev pointers are device memory of
 * the current GPU, owned by the caller; a call only enqueues kernels on hip_stream (NULL = the default stream), allocates
 * nothing, never synchronises and may be captured into a graph.  Argument errors are found before anything is enqueued.
 * Calls that need scratch memory take a workspace of at least the number of bytes that the matching *_workspace function
 * returns (0 for sizes that the call refuses), 16-byte aligned, contents irrelevant before and after; calls that overlap in
 * time need workspaces of their own.
 *
 * Tensors are rows of tokens: element (n, c) at n * ld + c, any ld >= the row's length, aligned to an element.  dt is the
 * element type of activations and their gradients (fp32, fp16, bf16); parameters, their gradients, states and statistics are
 * fp32.  Sums, statistics and states are held in fp32, results rounded once (nearest even).  No kernel uses floating-point
 * atomics: a call repeated on the same inputs gives the same bits.  Zero rows are a valid call (row pointers may then be NULL).
 * Outputs overlap no other operand but where a call says that it works in place, which it does from the same address with the
 * same leading dimension (another one is refused: SHAPE).
 */
#ifndef GRIM_LM_H
#define GRIM_LM_H

#include "grim_bcr.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Layer norm over the C features of each of N rows:
 *     m = sum(x) / C     s = 1 / sqrt(sum((x - m)^2) / C + eps)     y = (x - m) * s * gamma + beta
 *   gamma_dev, beta_dev   C fp32, or NULL (1 and 0)
 *   y_dev                 element type dt, rows of ldy; may be x_dev itself with ldy = ldx
 *   mean_dev, rstd_dev    N fp32 each (m and s, what the backward pass reads), or NULL
 * Backward, for the gradient dy of y (d = dy * gamma, xh = (x - m) * s):
 *     dx = s * (d - sum(d) / C - xh * sum(d * xh) / C)     dgamma = sum over rows of dy * xh     dbeta = sum over rows of dy
 *   dx_dev                element type dt, or NULL; may be dy_dev itself (same ld) but must not overlap x_dev otherwise
 *   dgamma_dev, dbeta_dev C fp32, overwritten (zeros for N = 0), or NULL
 *   workspace             grim_layer_norm_workspace(N, C) bytes, or NULL if neither dgamma nor dbeta is asked for
 * Errors: NULL, SHAPE (N < 0, N >= 2^31, C < 1, C > 16776960 in the backward pass, leading dimension too small, eps negative or not
 * finite, workspace too small), DTYPE, DEVICE.
 */
grim_status grim_layer_norm(const void *x_dev, grim_dtype dt, int64_t ldx, const float *gamma_dev, const float *beta_dev,
                            float eps, int64_t N, int64_t C, void *y_dev, int64_t ldy, float *mean_dev, float *rstd_dev,
                            void *hip_stream);
int64_t grim_layer_norm_workspace(int64_t N, int64_t C);
grim_status grim_layer_norm_backward(const void *dy_dev, int64_t lddy, const void *x_dev, int64_t ldx, grim_dtype dt,
                                     const float *gamma_dev, const float *mean_dev, const float *rstd_dev, int64_t N,
                                     int64_t C, void *dx_dev, int64_t lddx, float *dgamma_dev, float *dbeta_dev,
                                     void *workspace, int64_t workspace_bytes, void *hip_stream);

/*
 * Gated linear recurrence over packed sequences.  Row n of the gates holds the pre-activations [forget u | candidate c |
 * output v] of one token, 3H values; with the biases added,
 *     f = sigmoid(u)     h_t = f * h_(t-1) + (1 - f) * c     y_t = sigmoid(v) * h_t
 * in fp32 (1 - f is formed as sigmoid(-u), so gates that are almost open keep their digits).
 *   gates_dev      N x 3H of element type dt, rows of ldg >= 3H
 *   bias_dev       3H fp32, or NULL
 *   h0_dev         nseq x H fp32: the states before the first tokens, or NULL (zeros)
 *   seq_start_dev  nseq + 1 int32: sequence s is rows seq_start[s] .. seq_start[s+1] - 1 (empty ones allowed);
 *                  seq_start[0] = 0, ascending, seq_start[nseq] = N.  NULL: one sequence of all rows (nseq = 1).
 *                  The values are read on the GPU only; others than these give undefined results, inside the buffers.
 *   y_dev          N x H of element type dt, rows of ldy; must not overlap the gates
 *   h_last_dev     nseq x H fp32, the states after the last tokens (of an empty sequence: its h0), or NULL; must not overlap
 *                  h0 (unlike a step, the call cannot work in place: sequences end and start in different workgroups)
 *   states_dev     grim_glr_states(N, H) bytes of fp32 states for the backward pass, or NULL
 *   workspace      grim_glr_workspace(N, H) bytes, for either direction
 * Backward, for the gradients dy of y and dh_last of h_last (nseq x H fp32, or NULL: zeros): the states are
 * recomputed from states_dev a few tokens at a time.
 *     G_t = dy_t * sigmoid(v_t) + f_(t+1) * G_(t+1) (after the last token: dh_last)
 *     du = G f (1 - f) (h_(t-1) - c)     dc = G (1 - f)     dv = dy h sigmoid(v) (1 - sigmoid(v))     dh0 = f_0 G_0
 *   dgates_dev     N x 3H of element type dt, rows of lddg; must not overlap the inputs
 *   dbias_dev      3H fp32: column sums of the gates' gradient before its rounding, overwritten; or NULL
 *   dh0_dev        nseq x H fp32, overwritten (of an empty sequence: its dh_last); or NULL; must not overlap dh_last
 * Infinities and NaN of one sequence do not reach another.
 * grim_glr_step is one token for `batch` callers at once, in the layout of grim_lstm_cell: gates 3H x batch fp32 as
 * grim_bcr_spmv leaves them (ldg >= batch), states H x batch fp32 (h_new_dev may be h_dev itself, same ld), y H x batch of element
 * type dt (what the next product reads), or NULL.
 * Errors: NULL, SHAPE (N < 0, N > 2^30, H < 1, H > 2^21, nseq < 1, nseq > 1 without starts, leading dimension or a buffer too small; of
 * the step: H < 1, batch < 0, H * batch > 2^32 - 256, leading dimension too small), DTYPE, DEVICE, UNSUPPORTED (h_last over h0,
 * dh0 over dh_last).
 */
int64_t grim_glr_states(int64_t N, int64_t H);
int64_t grim_glr_workspace(int64_t N, int64_t H);
grim_status grim_glr_sequence(const void *gates_dev, grim_dtype dt, int64_t ldg, const float *bias_dev, const float *h0_dev,
                              const int32_t *seq_start_dev, int32_t nseq, int64_t N, int64_t H, void *y_dev, int64_t ldy,
                              float *h_last_dev, void *states_dev, void *workspace, int64_t workspace_bytes,
                              void *hip_stream);
grim_status grim_glr_sequence_backward(const void *gates_dev, grim_dtype dt, int64_t ldg, const float *bias_dev,
                                       const float *h0_dev, const int32_t *seq_start_dev, int32_t nseq, int64_t N, int64_t H,
                                       const void *states_dev, const void *dy_dev, int64_t lddy, const float *dh_last_dev,
                                       void *dgates_dev, int64_t lddg, float *dbias_dev, float *dh0_dev, void *workspace,
                                       int64_t workspace_bytes, void *hip_stream);
grim_status grim_glr_step(const float *gates_dev, int64_t ldg, const float *bias_dev, const float *h_dev, int64_t ldh,
                          float *h_new_dev, int64_t ldh_new, void *y_dev, grim_dtype dt, int64_t ldy, int64_t H,
                          int32_t batch, void *hip_stream);

/*
 * Distillation from a teacher's top logits.  Row n of the student's logits z has V entries; the teacher lists k of them,
 * words top_ids[n * ldt + i] with logits top_logits[n * ldt + i].  With the temperature tau,
 *     p = softmax over the listed entries of top_logits / tau        log q = log softmax over all V of z / tau
 *     loss_n = weight_n * tau^2 * sum_i p_i * (log p_i - log q[id_i])
 *     dz_n[j] = weight_n * tau * (q_j - sum of p_i with id_i = j)        (the gradient of sum over n of loss_n)
 *   z_dev          N x V of element type dt, rows of ldz
 *   top_ids        int32; an entry outside 0 .. V-1 is absent (a row may list fewer than k).  A word listed twice counts twice.
 *   weight_dev     N fp32 (the mean's 1/N, a loss scale, 0 for padding), or NULL (1).  Rows of weight 0 and rows without
 *                  any entry (or whose listed logits are all -infinity) have loss 0 and gradient 0, whatever z holds.
 *   loss_dev       N fp32
 *   dz_dev         N x V of element type dt, rows of lddz, may be z_dev itself (same ld); NULL: the loss alone
 *   workspace      grim_distill_topk_workspace(N, V) bytes
 * The loss is a difference of logarithms in fp32, off by some 2^-20 of weight tau^2: at temperatures far above the spread of
 * the logits that is more than what is left of a loss whose teacher lists all words.
 * z may hold -infinity (words that cannot come: q = 0); a row that holds nothing else, or +infinity or NaN, gives NaN, as does a
 * listed logit of +infinity or NaN.
 * Errors: NULL, SHAPE (N < 0, N >= 2^31, V < 1, V >= 2^31, k < 1, leading dimension too small, tau outside 1e-30 .. 1e30,
 * workspace too small), DTYPE, DEVICE, UNSUPPORTED (k > 1024).
 */
int64_t grim_distill_topk_workspace(int64_t N, int64_t V);
grim_status grim_distill_topk(const void *z_dev, grim_dtype dt, int64_t ldz, const float *top_logits_dev,
                              const int32_t *top_ids_dev, int32_t k, int64_t ldt, float temperature,
                              const float *weight_dev, int64_t N, int64_t V, float *loss_dev, void *dz_dev, int64_t lddz,
                              void *workspace, int64_t workspace_bytes, void *hip_stream);

/*
 * The rules applied to the logits of a served step, for `batch` callers at once, in this order:
 *     1. repetition  a word of the caller's history: z > 0 ? z / repetition : z * repetition
 *     2. frequency, presence   z - frequency * (how often the word occurs in the history) - presence * (it occurs at all)
 *     3. bias        z + the values that the caller's list gives for the word (added in the list's order)
 *     4. grammar     words that are not allowed: -infinity
 * Zero-initialise, then set what is used; a NULL pointer leaves its rule out.
 */
typedef struct grim_logit_rules {
    const int32_t *history;       /* batch rows of ld_history >= max_history words; words outside 0 .. V-1 are ignored */
    const int32_t *history_len;   /* batch: how many of them count (clamped to 0 .. max_history); NULL: max_history */
    int64_t ld_history;
    int32_t max_history;
    int32_t nbias;                /* entries of each caller's bias list */
    const float *repetition;      /* batch, > 0 each */
    const float *frequency;       /* batch */
    const float *presence;        /* batch */
    const int32_t *bias_ids;      /* batch rows of ld_bias >= nbias words; words outside 0 .. V-1 are ignored */
    const float *bias_values;     /* the same rows of values */
    int64_t ld_bias;
    const uint32_t *allowed;      /* batch rows of ld_allowed >= ceil(V / 32) words; bit v % 32 of word v / 32: word v is allowed */
    int64_t ld_allowed;
} grim_logit_rules;

/*
 *   z_dev, out_dev   element type dt; columns = 0: batch x V, a row per caller (ld >= V); columns = 1: V x batch, a column
 *                    per caller, as grim_bcr_spmv leaves logits (ld >= batch).  out_dev may be z_dev itself (same ld).
 * Arithmetic in fp32, rounded once.
 * Errors: NULL, SHAPE (V < 1, V >= 2^31, batch < 0, leading dimension too small, max_history or nbias negative), DTYPE,
 * DEVICE, UNSUPPORTED (nbias > 1024, max_history > 2^20).
 */
grim_status grim_apply_logit_rules(const void *z_dev, grim_dtype dt, int32_t columns, int64_t ldz, int64_t V, int32_t batch,
                                   const grim_logit_rules *rules, void *out_dev, int64_t ldo, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* GRIM_LM_H */
