/*
 * vcas_train.h -- what a training step does before and behind the sampled backward of its linear layers
 * (vcas.h): attention over packed sequences, the log probabilities of given tokens with the gradient that
 * starts the backward pass, and the optimizer step that takes the weight gradients.  The paper trains with these
 * (Sec. 6, App. F: transformers, cross-entropy, AdamW) without describing them.
 *
 * The conventions of vcas.h hold: every call returns VCAS_OK or a negative vcas_status, never throws, aborts or
 * prints; pointers are DEVICE pointers owned by the caller unless "host" is said; work is enqueued on the caller's
 * stream and is asynchronous; only the _create, _destroy and _status calls allocate or synchronise.  Results do not
 * depend on the order in which CTAs run: two calls with the same inputs give the same bits.  A call
 * with a handle runs on the handle's device, whichever is current; its stream and tensors must be that
 * device's.  A handle owns one workspace: its calls must not overlap on the GPU (two streams, two captured graphs
 * replayed at once); use a handle each.
 */
#ifndef VCAS_TRAIN_H_
#define VCAS_TRAIN_H_

#include "vcas.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ attention over packed sequences ---- */
/*
 * Self-attention of N sequences that lie one behind the other: sequence n is the tokens starts[n] .. starts[n+1]-1
 * (starts [N+1] int32, device, ascending; starts[N] <= total).  Query head h uses key/value head
 * h / (heads_q / heads_kv).  Per sequence and head, with scale s:
 *   S = s Q K^T,  causal: S_ij = -inf for j > i,  P = softmax(S) by rows,  O = P V,  lse_i = log sum_j exp(S_ij);
 *   dV = P^T dO,  dP = dO V^T,  dS = P (dP - rowsum(dO O)),  dQ = s dS K,  dK = s dS^T Q,
 * dK and dV summed over the query heads that share them.  Sums, softmax statistics and lse are fp32; in bf16 layers P and dS
 * are rounded to bf16 where they enter a product (on the tensor cores to a sum of two bf16 where a sequence's first rows, of
 * 64 keys or less, are concerned), O and the gradients once when stored.
 * A sequence may be empty.  Rows from starts[N] on are neither read nor written.  starts that descend, are negative
 * or pass `total` are not followed: those sequences are left out (nothing is written to their rows) and vcas_attn_status
 * reports VCAS_ERR_BAD_ARG.  The results of sequences that such starts make overlap, and of those listed behind them, are unspecified,
 * and rows of sequences that a backward drops may then be left unwritten.
 * A NaN or infinity in a row of q, k or v reaches that sequence's results only.
 * Beyond 128 sequences the time to find their tiles grows with the square of their number.
 */
typedef struct vcas_attn_s* vcas_attn;

typedef struct {
  int32_t max_tokens, max_seqs;       /* the largest `total` and N of a call */
  int32_t heads_q, heads_kv;          /* heads_q a multiple of heads_kv */
  int32_t head_dim;                   /* a multiple of 8, at most 128 */
  int32_t dtype;                      /* vcas_dtype of q, k, v, o and their gradients */
  int32_t causal;                     /* non-zero: a token sees itself and those before it */
  float scale;                        /* 0: 1 / sqrt(head_dim) */
} vcas_attn_desc;

/* A [total, heads, head_dim] tensor: element (t, h, d) is ptr[t * token + h * head + d] (strides in elements, not
 * negative; q, k, v and their gradients may lie in one buffer, as a joint projection leaves them; a stride of 0 repeats an
 * input).  What is written overlaps neither itself nor anything else of the call.  Any alignment of the dtype is
 * served; bf16 with 16-byte aligned ptr and strides that are multiples of 8 runs on the tensor cores. */
typedef struct {
  void* ptr;
  int64_t token, head;
} vcas_attn_tensor;

int vcas_attn_create(vcas_attn* out, const vcas_attn_desc* desc);
int vcas_attn_destroy(vcas_attn a);
int vcas_attn_workspace_bytes(vcas_attn a, size_t* bytes);      /* host out */

/* o, and lse [heads_q][total] fp32 (needed by the backward). */
int vcas_attn_fwd(vcas_attn a, const vcas_attn_tensor* q, const vcas_attn_tensor* k, const vcas_attn_tensor* v,
                  const int32_t* starts, int32_t N, int32_t total, const vcas_attn_tensor* o, float* lse,
                  vcas_stream stream);
/*
 * The backward from d_o = dL/dO and the forward's o and lse.  alive_in [N] / alive_cnt_in [1] (device, in pairs, may be NULL):
 * ascending list of the sequences whose rows of d_o may be non-zero, as vcas_linear_bwd_chain's kept_out gives it for the
 * layer above (Sec. 4: data dropped by SampleA have a zero gradient in every layer below).  The others are not
 * computed and none of their rows is read; their rows of dq, dk, dv are set to zero, or, with skip_dropped_rows,
 * left unwritten.  A length outside [0, N] (the list then counts as empty), an entry outside [0, N) and one that is not above
 * all others before it are not followed and reported like bad starts.
 */
int vcas_attn_bwd(vcas_attn a, const vcas_attn_tensor* d_o, const vcas_attn_tensor* q, const vcas_attn_tensor* k,
                  const vcas_attn_tensor* v, const vcas_attn_tensor* o, const float* lse, const int32_t* starts, int32_t N,
                  int32_t total, const int32_t* alive_in, const int32_t* alive_cnt_in, int32_t skip_dropped_rows,
                  const vcas_attn_tensor* dq, const vcas_attn_tensor* dk, const vcas_attn_tensor* dv, vcas_stream stream);
/* Synchronises the handle's device, returns its status word (as vcas_last_device_status does) and clears it. */
int vcas_attn_status(vcas_attn a, int32_t* status);
/* Bound of every wait inside the tensor-core kernels, and the test hook of vcas_set_wait_limit: with stall_once the first
 * CTA of every launch leaves out its first loads. */
int vcas_attn_set_wait_limit(vcas_attn a, uint64_t limit_ns, int32_t stall_once);

/* ------------------------------------------------------------------- log probabilities of given tokens ---- */
/*
 * Row r of logits (V values, rows ld elements apart) is a distribution p = softmax(x).  For the given token t_r:
 *   lse = log sum_j exp(x_j),  logp = x_t - lse,  entropy = -sum_j p_j log p_j,
 *   top_ids / top_logp: the `top` largest x_j in descending order, equal ones by ascending index, and x_j - lse.
 * A negative token means none: logp = 0 and no gradient through it.  A token >= V is taken for none and reported as
 * VCAS_ERR_BAD_ARG by vcas_loss_status.  -inf (a token that is not allowed) has p = 0 and adds nothing.  A row that is -inf
 * throughout has no distribution: lse and logp -inf, entropy 0, a zero gradient.  NaN or +inf in a row make its lse, logp,
 * entropy and top_logp NaN, and its top_ids unspecified (within [-1, V)).
 */
typedef struct vcas_loss_s* vcas_loss;

typedef struct {
  int32_t max_rows, vocab;
  int32_t dtype;                      /* vcas_dtype of logits and dlogits */
  int32_t top;                        /* alternatives a row: 0 .. min(32, vocab) */
} vcas_loss_desc;

int vcas_loss_create(vcas_loss* out, const vcas_loss_desc* desc);
int vcas_loss_destroy(vcas_loss l);
/* tokens [rows]: int32 (token_bytes 4) or int64 (8); logp, entropy, lse [rows] fp32, top_logp [rows][top] fp32 and
 * top_ids [rows][top] int32, each may be NULL.  Any ld >= vocab and any alignment of the dtype. */
int vcas_loss_fwd(vcas_loss l, const void* logits, int64_t ld, const void* tokens, int32_t token_bytes, int32_t rows,
                  float* logp, float* entropy, float* lse, float* top_logp, int32_t* top_ids, vcas_stream stream);
/*
 * dlogits_j = g_logp (1[j = t] - p_j) - g_entropy p_j (log p_j + entropy) from the forward's lse and entropy (where lse is 1024 or
 * more away from 0, its fp32 value is too coarse for p, which then comes from the row's logits alone);
 * g_logp, g_entropy [rows]: the loss's derivatives (g_entropy may be NULL, then entropy may be too).  Rows whose factors
 * are both zero (no token and no entropy term, or g_logp = 0) get zeros and are not read.  dlogits may be logits
 * themselves (same ld).  a_out [rows], may be NULL: the square-norm of every row of dlogits as stored, which
 * vcas_linear_bwd_chain takes as a_in with a_in_parts = 1 so that the layer under the loss reads no gradient for its scores.
 */
int vcas_loss_bwd(vcas_loss l, const void* logits, int64_t ld, const void* tokens, int32_t token_bytes, int32_t rows,
                  const float* lse, const float* entropy, const float* g_logp, const float* g_entropy,
                  void* dlogits, int64_t ld_d, float* a_out, vcas_stream stream);
int vcas_loss_status(vcas_loss l, int32_t* status);

/* ------------------------------------------------------------------------------------- optimizer step ---- */
/*
 * AdamW over any number of tensors.  With g' = g * *grad_scale, per element, every operation rounded to fp32 on its own
 * (with 8-bit states, p: the quotient is good to 2^-22 relative, its denominator and p's new value are fused sums; v and eps
 * other than 0 count as no less than 2^-126):
 *   m <- beta1 m + (1 - beta1) g',   v <- beta2 v + (1 - beta2) g' g',
 *   p <- p (1 - lr wd) - (m lr / (1 - beta1^step)) / (sqrt(v) / sqrt(1 - beta2^step) + eps).
 * state_bits 32: m and v are fp32.  state_bits 8: m and r = sqrt(v) are held as e4m3 values, one fp32 scale for each 256
 * consecutive elements (m_scale, v_scale [(n + 255) / 256]); m = value * scale, v = (value * scale)^2.  The step uses the
 * unrounded new m and v; scale = largest of the block / 448, and value / scale goes to one of its two e4m3
 * neighbours, up with the probability of where it lies between them (to 8 random bits), so that a state
 * that moves by less than a rounding step per step still moves; a positive r never becomes 0, and an infinite one (a finite g'
 * whose square is not: p then only decays in this step, by the formula) is held as 2^63.  Random bits:
 * Philox4x32-10 with key = (seed low, seed high), counter = (element / 8, tensor's place in the list, 3, 0); of element e,
 * word e % 8 / 2, halfword e % 2: low byte for m, high byte for r.  Give another seed each step.
 * A NaN or infinite gradient spoils its element, and with 8-bit states the states of its block.
 */
typedef struct {
  void* p;                            /* [n] p_dtype, updated */
  const void* g;                      /* [n] g_dtype */
  void* m;                            /* [n] fp32 or e4m3 */
  void* v;
  float* m_scale;                     /* 8-bit states */
  float* v_scale;
  void* copy;                         /* [n] bf16 copy of the new p for the layers that read it (fp32 p only; may be NULL) */
  int64_t n;                          /* 0 .. 2^34 */
  float weight_decay;
  int32_t p_dtype, g_dtype;           /* vcas_dtype */
  int32_t state_bits;                 /* 8 or 32 */
} vcas_adamw_tensor;

typedef struct {
  double lr, beta1, beta2, eps;
  int64_t step;                       /* 1 for the first */
  uint64_t seed;                      /* 8-bit states */
  const float* grad_scale;            /* device [1], may be NULL (1): a clipping factor, say */
  const float* rates;                 /* device [3], may be NULL: what vcas_adamw_rates gives, read instead of lr and step.  A
                                       * captured step then takes the values that are there when it is replayed */
  const uint64_t* seed_dev;           /* device [1], may be NULL: read instead of seed */
} vcas_adamw_args;

/* tensors: host array, read before the call returns; n_tensors may be 0.  No handle, no allocation.  Runs on the current
 * device, whose stream and tensors they must be.  The tensors of a list must not overlap. */
int vcas_adamw_step(const vcas_adamw_tensor* tensors, int32_t n_tensors, const vcas_adamw_args* args, vcas_stream stream);
/* rates[0..2] (host out) = lr, lr / (1 - beta1^step), 1 / sqrt(1 - beta2^step). */
int vcas_adamw_rates(double lr, double beta1, double beta2, int64_t step, float* rates);

#ifdef __cplusplus
}
#endif
#endif /* VCAS_TRAIN_H_ */
