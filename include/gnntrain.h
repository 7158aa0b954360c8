/*
 * gnntrain — the epoch loop of Algorithm 1 around gnnstage handles, on one MI355X (gfx950).  C ABI.
 *
 * One epoch: draw the chunk order (Section 3.4, first technique: shuffled at the beginning of every
 * epoch); every stage, first to last, takes all chunks in that order (gnnstage_forward_pass; chunk by chunk through all
 * stages where a stage's level-0 history is the level below it), then the loss head all rows; the
 * backward pass walks the stages from the last to the first, chunks in the reverse order; the weights are updated
 * (Algorithm 1, last line: the plain gradient step; Section 5 trains with Adam, learning rate 0.001);
 * the historical embeddings are refreshed after the epochs alpha, 2 alpha, ... (Section 3.4, second
 * technique: epoch t reads the embeddings of epoch alpha * floor((t - 1) / alpha)).
 *
 * The stages run back to back on this GPU: level L of stage s must be the same DEVICE buffer as level 0
 * of stage s + 1, and stage s + 1 must have been created with need_input_grad (its grad_in rows are the
 * upstream gradient of stage s).  On a pipeline of several GPUs each stage would sit on its own device
 * and this loop would be its schedule; here it is the sequential schedule, which computes the same values.
 *
 * The paper does not print its loss.  The head taken here is the usual one for node classification: a
 * linear classifier on the last level, logits = h W_o + b_o, and the mean softmax cross-entropy over the
 * labelled vertices.
 *
 * Ownership as in gnnstage.h: everything the descriptor points to stays with the caller, HOST arrays are
 * copied at create time, the library allocates no device memory (its state lives in the workspace).
 * Every function returns GNNSTAGE_OK or a negative GNNSTAGE_E* code.
 */
#ifndef GNNTRAIN_H
#define GNNTRAIN_H

#include "gnnstage.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct gnntrain gnntrain_t; /* opaque, owned by the library */

enum { GNNTRAIN_SGD = 0, GNNTRAIN_ADAM = 1, GNNTRAIN_ADAMW = 2 };

/* One trainable tensor.  The optimiser works on the fp32 master copy; after every step it also writes the
 * copy the kernels read when that is a different buffer (bf16 stages: W[j] of gnnstage_desc, head_W). */
typedef struct {
  float *master;         /* DEVICE fp32, count elements; holds the initial value at create time */
  void *compute;         /* DEVICE, count elements of compute_dtype; NULL when the kernels read master */
  int32_t compute_dtype; /* GNNSTAGE_F32 or GNNSTAGE_BF16 */
  float *grad;           /* DEVICE fp32, count elements; zeroed by the loop at the start of every epoch */
  int64_t count;
} gnntrain_param;

/* New fields come at the end, and zero keeps what was: clear the struct before filling it in, and build callers against the header of their library (it has no size field). */
typedef struct {
  int32_t n_stages;
  gnnstage_t *const *stages; /* HOST array, first to last; same graph size and chunks for all */
  /* loss head on level L of the last stage (n x d_top, that stage's dtype) */
  int32_t n_classes;
  const void *head_W;        /* DEVICE d_top x n_classes, dtype of the last stage */
  const float *head_b;       /* DEVICE fp32 n_classes */
  float *head_dW;            /* DEVICE fp32 d_top x n_classes, "+=" over the rows */
  float *head_db;            /* DEVICE fp32 n_classes */
  const int32_t *labels;     /* DEVICE, one class id in [0, n_classes) per vertex */
  const uint8_t *train_mask; /* DEVICE, one byte per vertex (non-zero = labelled); NULL = all vertices */
  /* parameters of all stages and of the head, in the order they are stepped */
  int32_t n_params;
  const gnntrain_param *params; /* HOST array */
  int32_t optimizer;            /* GNNTRAIN_SGD: p -= lr (g + wd p);  GNNTRAIN_ADAM: Kingma & Ba, Algorithm 1 (wd p is added to g);
                                   GNNTRAIN_ADAMW: gnntrain_adamw_step (wd apart from g, the same for every parameter: biases
                                   and norm vectors too; buffers of parameters may then not overlap) */
  float lr, beta1, beta2, eps, weight_decay;
  int32_t shuffle;    /* 0: chunks in index order every epoch */
  uint64_t seed;      /* of the chunk shuffling, and of the dropout decisions of stages that have dropout: stage s
                         gets gnnstage_set_dropout_seed(SplitMix64(seed + (epoch + 1) * 0x9E3779B97F4A7C15) + s) */
  int32_t alpha_hist; /* refresh period of the historical embeddings, >= 1 */
  int32_t history_swap; /* non-zero: refresh with gnnstage_update_history_swap (the level buffers of a stage trade places,
                           nothing but level 0 is copied) instead of update_history; the stages' level pointers then
                           come from gnnstage_level_buffers */
  void *workspace;    /* DEVICE, 256-byte aligned, >= gnntrain_workspace_size() bytes */
  size_t workspace_bytes;
  int32_t head_fused; /* non-zero: the head is gnntrain_head_xent, which keeps neither logits nor their gradients of all vertices; n_classes may then be up to
                         2^24 (otherwise 65,536).  Takes less memory from about 16 classes on where the last level is bf16 and 64, 128 or 256 wide (its rows are read in
                         place); otherwise packed rows are kept, of up to 2^20 vertices (fp32, or wider than 256: 131,072, with fp32 sums and logits), and it is the
                         classes beyond a row's width that make it smaller: 89,250 x 100 fp32, 7 classes 78 MB for 6 */
  int32_t state_8bit;  /* GNNTRAIN_ADAMW: non-zero keeps its states in 8 bits (2.06 bytes per parameter of the workspace instead of 8; draws from seed).
                          Must be zero with another optimizer */
} gnntrain_desc;

/* Device bytes the loop needs: optimiser moments, logits of up to 131,072 vertices, gradient of the logits and
 * gradient rows of the last level for all vertices, per-vertex losses, staged head weights, split-reduction
 * scratch (head_fused: gnntrain_head_xent's workspace in the place of logits, their gradients, weights and scratch).  Host-only; 0 on an invalid descriptor
 * (why: gnntrain_last_error(NULL)), also where the head refuses the last level's width or its product with n_classes. */
size_t gnntrain_workspace_size(const gnntrain_desc *desc);

/* Validates the descriptor against the stage handles (chaining of the level buffers, label range),
 * clears the optimiser state and synchronises.  *out is NULL on failure. */
int gnntrain_create(const gnntrain_desc *desc, gnntrain_t **out);

/* Runs epoch `epoch` (0-based; epochs must be run in order for the history schedule to mean what the
 * paper says, but the function itself only uses the number for the chunk order and the refresh test).
 * loss: HOST, receives the mean cross-entropy of this epoch's forward pass; with a non-NULL loss the call
 * synchronises the stream before returning, with NULL it is asynchronous. */
int gnntrain_epoch(gnntrain_t *tr, int64_t epoch, float *loss, void *hip_stream);

/* The chunk order the last epoch used (HOST, n_chunks entries). */
int gnntrain_last_order(const gnntrain_t *tr, int32_t *order);

int gnntrain_destroy(gnntrain_t *tr);
/* Of this handle, or, with NULL, of the calling thread's last failed call without one (readable until that thread's next one). */
const char *gnntrain_last_error(const gnntrain_t *tr);

/* ---- the steps of the loop, exported one by one ------------------------------------------------- */

/* Section 3.4, first technique.  order: HOST, n_chunks entries.  Epoch e owns the SplitMix64 stream (Steele,
 * Lea, Flood 2014) that starts at state seed + (e + 1) * 0x9E3779B97F4A7C15; draw i is the generator's
 * output for state start + (i + 1) * 0x9E3779B97F4A7C15; a Fisher-Yates pass from the last position down
 * swaps position i with position draw mod (i + 1).  Host only. */
int gnntrain_chunk_order(uint64_t seed, int64_t epoch, int32_t n_chunks, int32_t shuffle, int32_t *order);

/* Softmax cross-entropy of `rows` vertices.  logits: DEVICE fp32 rows x ld (n_classes valid columns); bias
 * (DEVICE fp32, may be NULL) is added to them first.  For a labelled row: row_loss = log sum_c exp(z_c) -
 * z_label and dlogits_c = (softmax_c - [c = label]) * inv_n_train; an unlabelled row gets loss 0 and a zero
 * gradient.  dlogits: DEVICE rows x dl_ld of dl_dtype, columns [n_classes, dl_ld) are written as zeros.
 * labels / mask are indexed by row (pass pointers to the first row).  Asynchronous. */
int gnntrain_softmax_xent(const float *logits, int32_t ld, const float *bias, const int32_t *labels,
                          const uint8_t *mask, int64_t rows, int32_t n_classes, float inv_n_train, void *dlogits,
                          int32_t dl_dtype, int32_t dl_ld, float *row_loss, void *hip_stream);

/* The loss head over many classes: what a linear classifier, gnntrain_softmax_xent and the classifier's gradients compute, without
 * the logits of all rows and classes in memory: those of bf16 rows of up to 256 columns never leave the registers, of others at most 2^26 are there at a time,
 * with their gradients.  z = h_r W + bias; for a labelled row: row_loss = log sum_c
 * exp(z_c) - z_label, g_c = (softmax_c - [c = label]) * inv_n_train; dh = g W^T, dW += h^T g, db += column sums of g.  A row is
 * labelled when mask (NULL: all rows) is non-zero and its label is in [0, n_classes); any other row has loss 0 and a zero row of
 * dh, takes no part in dW and db whatever it holds, and may hold anything.
 * h: DEVICE rows x d, leading dimension ld_h >= d; W: DEVICE d x n_classes, both of dtype; bias: DEVICE fp32 n_classes or NULL
 * (minus infinity leaves a class out; a row whose every logit is minus infinity has loss and gradients NaN).  labels, mask, row_loss: DEVICE, by row.
 * dh (of dtype, leading dimension ld_dh), dW (fp32 d x n_classes), db (fp32 n_classes): DEVICE, each may be NULL; all NULL: the losses
 * alone.  Outputs may not overlap inputs (dh == h is refused).  d in [1, 65534], n_classes in [1, 2^24], d * n_classes at most 2^33.
 * bf16 products have fp32 sums.  Their factors: in dh every g is the sum of two bf16 numbers (2^-16 of itself), but of up to 256 columns a probability
 * of less than 1/32 of its row's others may be one (2^-8 of itself, where what the weights have in common cancels all the same); the g in dW's
 * are the sum of two (2^-16), and where a slab of 2^20 rows has at most 16,384 labelled ones, or fewer than 128 a class, of three (all bits) in blocks of 32 rows and
 * 32 classes in which some |g| is above inv_n_train / 64; wider rows' g in dW's have all bits.  Sums are added in a fixed order: the same call gives the same bits.
 * workspace: DEVICE, 256-byte aligned, of gnntrain_head_xent_workspace_size(); written by the call, nothing in it has to be
 * cleared or kept.  Calls that overlap in time need workspaces of their own, and so do graphs that are replayed side by side.
 * The call only launches kernels (asynchronous, may be captured).  Message of an error: gnntrain_last_error(NULL). */
size_t gnntrain_head_xent_workspace_size(int64_t rows, int32_t d, int32_t n_classes, int32_t dtype, int32_t want_grads);
int gnntrain_head_xent(const void *h, int64_t ld_h, const void *W, int32_t dtype, const float *bias, const int32_t *labels,
                       const uint8_t *mask, int64_t rows, int32_t d, int32_t n_classes, float inv_n_train, float *row_loss, void *dh,
                       int64_t ld_dh, float *dW, float *db, void *workspace, size_t workspace_bytes, void *hip_stream);

/* What logits answer, per row, with z = logits + bias:
 *   logp     log softmax(z) at the row's class ids[r] (0 where that is outside [0, n_classes)); needs ids
 *   entropy  -sum_c p_c log p_c, p = softmax(z), in nats
 *   norm     (largest z that is a number, log sum_c exp(z_c - largest z)): what gnntrain_logprobs_grad takes, rows x 2
 *   top_ids, top_logp  the n_top classes of the largest z in their order, of equals the lower class first, and their log softmax, rows x n_top
 * Each output but the last two, which n_top > 0 asks for, may be NULL.  Sums are fp32; a row that is sure of its given class has a log probability with all its digits.
 * Where it is sure of another class, log sum (with entropy and top_logp, which have it in them) is off by up to 2^-24 next to 1: the top_logp of a probability within that of 1 is 0.
 * A logit of minus infinity is a class left out: probability 0, last in the order.  A row whose every logit is minus infinity, or with infinity or a NaN among
 * them, has NaN for every number but norm's first; a NaN is in no order, and ids that are not there are -1.  A row whose mask byte is 0 (mask NULL: none) takes
 * no part, whatever it holds (its memory may be read all the same): it gets zeros, classes -1 and their log probabilities minus infinity.
 * logits: DEVICE rows x n_classes of dtype, leading dimension ld >= n_classes, aligned to its elements; bias: DEVICE fp32 n_classes or NULL; ids, mask: DEVICE, by row, or NULL.
 * n_classes in [1, 2^24], n_top in [0, 64] and n_classes at most.  workspace: DEVICE, 256-byte aligned, of gnntrain_logprobs_workspace_size(), nothing in it
 * has to be cleared or kept; calls that overlap in time need workspaces of their own, and so do graphs that are replayed side by side.  Outputs may not
 * overlap inputs.  The call only launches kernels (asynchronous, may be captured); the same call gives the same bits.  Message of an error: gnntrain_last_error(NULL). */
size_t gnntrain_logprobs_workspace_size(int64_t rows, int32_t n_classes, int32_t n_top);
int gnntrain_logprobs(const void *logits, int32_t dtype, int64_t ld, const float *bias, const int32_t *ids, const uint8_t *mask, int64_t rows, int32_t n_classes,
                      int32_t n_top, float *logp, float *entropy, float *norm, int32_t *top_ids, float *top_logp, void *workspace, size_t workspace_bytes,
                      void *hip_stream);

/* Gradient of the logits from those of logp and entropy (g_logp, g_entropy: DEVICE fp32 by row; NULL: zeros):
 *   dlogits_c = g_logp ([c = id] - p_c) - g_entropy p_c (log p_c + entropy);  dbias_c += sum over the rows of dlogits_c before it is rounded
 * logits, bias, ids, mask as in the forward call, logp (with g_logp), entropy (with g_entropy) and norm what it gave.  A row without a class in [0, n_classes) has
 * no part in g_logp; a row whose mask byte is 0 gets zeros, whatever it holds (it may be read).  dlogits: DEVICE rows x n_classes of dl_dtype, leading dimension ld_dl >= n_classes (columns
 * behind n_classes stay as they are); it may be logits, with the same type and leading dimension.  dbias: DEVICE fp32 n_classes or NULL.  Sums in a fixed order.
 * workspace as above, of gnntrain_logprobs_grad_workspace_size(). */
size_t gnntrain_logprobs_grad_workspace_size(int64_t rows, int32_t n_classes);
int gnntrain_logprobs_grad(const void *logits, int32_t dtype, int64_t ld, const float *bias, const int32_t *ids, const uint8_t *mask, int64_t rows, int32_t n_classes,
                           const float *logp, const float *entropy, const float *norm, const float *g_logp, const float *g_entropy, void *dlogits, int32_t dl_dtype,
                           int64_t ld_dl, float *dbias, void *workspace, size_t workspace_bytes, void *hip_stream);

/* out[0] = scale * sum of x[0 .. n), added in a fixed order (reproducible).  scratch: DEVICE, 1024 floats. */
int gnntrain_sum(const float *x, int64_t n, float scale, float *scratch, float *out, void *hip_stream);

/* gnntrain_sum for callers that cannot allocate or bring a scratch buffer: code under HIP graph capture, tight
 * serving loops, harnesses that forbid allocation.  Same kernels, same order of additions, same result bit for
 * bit; the 1024 block sums go to an array that lives inside the library's device image (4 KB on every GPU the
 * library runs on, held until the process ends).  Calls no allocating routine.  Its address on the current device
 * is looked up at the first call on that device.  n may be at most GNNTRAIN_SUM_STATIC_MAX_N, beyond that the
 * call returns GNNSTAGE_ENOTSUP (gnntrain_last_error(NULL) says why; also for EINVAL and EHIP).  Nothing in the
 * array has to be cleared between calls (the first launch writes every slot the second reads), but every call on
 * one GPU uses the same array: calls that overlap in time on one GPU (two streams) race.  x, out: DEVICE. */
#define GNNTRAIN_SUM_STATIC_MAX_N 2147483647LL
int gnntrain_sum_static(const float *x, int64_t n, float scale, float *out, void *hip_stream);

/* One optimiser step on one tensor (t = 1, 2, ... for Adam's bias correction).  compute may be NULL. */
int gnntrain_adam_step(float *p, const float *g, float *m, float *v, void *compute, int32_t compute_dtype,
                       int64_t count, float lr, float beta1, float beta2, float eps, float weight_decay, int64_t t,
                       void *hip_stream);
/* One AdamW step (Loshchilov & Hutter, ICLR 2019, Algorithm 2) over all tensors of a model at once:
 *   g' = grad_scale g;  m = beta1 m + (1 - beta1) g';  v = beta2 v + (1 - beta2) g'^2;
 *   p = p (1 - lr weight_decay) - lr c1 m / (sqrt(c2 v) + eps),  c = 1 / (1 - beta^t);  compute = p, rounded
 * state_bits 32: m and v are fp32.  state_bits 8: m and the root of v are kept in blocks of 32 elements, a factor 2^e each (the byte e + 127 in
 * m_scale / v_scale, (count + 31) / 32 bytes) and a byte per element, the finite numbers of OCP's e4m3 (MXFP8): a value is rounded to one of its two
 * neighbours, at most 1/8 of itself apart from 2^-14 of the block's largest value on, by a draw that keeps its mean (nearest rounding would not: a step moves v by 1 - beta2 of
 * itself); what is above zero in v stays so.  The mean of v itself, the square of what is kept, is not: the draws' variance makes it larger by less than 14 % (3 to 4 % for normal
 * gradients, 6 % for such that come in one step of fifty: steps 2 and 3 % smaller), and an element's root scatters by 13 to 17 % around its own.  Far below the block's largest root it is
 * more: at 2^-15 of it v is 11 % too large, at 2^-17 68 %, and less than the least code, 2^-17 to 2^-18 of it, is held there (16 times v at 2^-19).  Tensors whose neighbouring elements
 * differ by so much are better kept in 32 bits.  All bytes zero are states of zero.  A block with a NaN, an infinity or 2^127 among its values is all NaN (byte 255).
 * The draws come from seed, t, the tensor's place in the list and the element's in the tensor (see SplitMix64 at gnntrain_chunk_order): with o(x) the
 * generator's output for state x, gamma its constant, tensor k has the key o(o(seed + t gamma) + (k + 1) gamma), its elements 2 j and 2 j + 1 the low and high half of
 * o(key + (j + 1) gamma), of which the low 16 bits are m's and the high ones v's.  The same call gives the same bits.
 * tensors: HOST, n of them, read during the call.  p (fp32), g (of g_dtype), compute (of compute_dtype, or NULL, or p): DEVICE, count elements, at any multiple of
 * their elements' size; m, v: DEVICE, count floats or bytes, at multiples of four bytes.  Buffers that are written may not overlap any other (gradients may
 * be shared).  count in [0, 2^35].  t = 1, 2, ...: a host number, as lr and seed are, so that a captured call repeats its step:
 * the same bias correction, and with 8-bit states the same draws every time, whose mean then is not kept (an element whose draw is low never moves up: replays that train need 32 bits,
 * or a graph per step).  grad_scale: DEVICE, one
 * float in no buffer that is written (what clips the gradients' norm, say), or NULL: 1.  beta1, beta2 in [0, 1).  Asynchronous, needs no workspace.
 * Message of an error: gnntrain_last_error(NULL). */
typedef struct {
  float *p;
  const void *g;
  int32_t g_dtype;       /* GNNSTAGE_F32 or GNNSTAGE_BF16 */
  int32_t compute_dtype; /* the same; read only with compute */
  void *compute;
  void *m, *v;
  uint8_t *m_scale, *v_scale; /* state_bits 8 */
  int64_t count;
  float weight_decay;
} gnntrain_adamw_tensor;
int gnntrain_adamw_step(const gnntrain_adamw_tensor *tensors, int32_t n, int32_t state_bits, float lr, float beta1, float beta2, float eps,
                        const float *grad_scale, int64_t t, uint64_t seed, void *hip_stream);

int gnntrain_sgd_step(float *p, const float *g, void *compute, int32_t compute_dtype, int64_t count, float lr,
                      float weight_decay, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* GNNTRAIN_H */
