/* halos_step.h -- operators of a worker's local step, for the B200 (sm_100a).
 *
 * halos.h covers the server side: it takes the result theta_{t,H} of a worker's H local steps (Algorithm 1, lines
 * 22-24) and answers with the model the worker restarts from.  The calls here are what a worker that trains a
 * decoder runs between the two, apart from plain matrix products:
 *
 *   halos_rope               rotary positions on queries and keys, and their way back
 *   halos_attention_fwd/bwd  masked attention; the backward pass recomputes the probabilities
 *   halos_distill_*          cross-entropy mixed with distillation from a teacher's top logits (K pairs per token
 *                            are what a slow link can carry of the global model's opinion), and its gradient
 *   halos_embedding_fwd/bwd  rows of a table by tokens, scaled; the gradient by sorted tokens
 *   halos_rms_norm_fwd/bwd   root-mean-square norm with the residual's addition, in 8 bits with scales if asked for; its gradient
 *   halos_grad_norm, halos_clip_grads, halos_sgd_step      the norm of many gradients at once, clipping by it, and the step
 *
 * Conventions
 *  - No context is needed.  Every call takes one args struct, whose first field is its size (checked), checks it
 *    on the host, makes args->device the calling thread's current device and leaves it so, enqueues its kernels on
 *    args->stream (cudaStream_t, NULL = the legacy default stream) and returns without waiting.  Tensors are
 *    borrowed until those kernels have completed in stream order.
 *  - Pointers are device pointers.  Strides are in elements; the innermost dimension is contiguous.
 *  - Nothing is allocated but 256 bytes of host memory in the first call (and, in calls that write lists of tensors, 24 bytes
 *    for each until the call returns): workspaces are the caller's (halos_*_workspace say how much).
 *  - The same inputs give the same bits, call after call: no result depends on the order of atomics.
 *  - Sums, statistics and everything between load and store are held in 32 bits, and results are rounded once, except that attention rounds p
 *    and ds to the inputs' type where they enter matrix products, and forms D from the o that was returned.
 *  - Status values are those of halos.h; on any other status than HALOS_OK nothing was enqueued (HALOS_ERR_CUDA
 *    excepted).  halos_step_error() is the calling thread's last error as text.
 */
#ifndef HALOS_STEP_H
#define HALOS_STEP_H

#include "halos.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { HALOS_F16 = 2 };  /* beside HALOS_F32 and HALOS_BF16 of halos.h */

const char* halos_step_error(void);

/* Device-side waits of these kernels are bounded.  One that ran out (it never does unless the GPU lost work, or kept a kernel from
 * running for a second) leaves its outputs undefined and a mark, and every later call on that device returns HALOS_ERR_CUDA
 * until the mark has been asked for here: *fault = 0 if there was none, and there is none afterwards.  Waits for the device. */
int halos_step_fault(int32_t device, int32_t* fault);

/* ------------------------------------------------------------------ rotary positions ----------- */

/* Layout of the pairs inside the rotated part [0, rot_dim) of a head. */
enum { HALOS_ROPE_HALF = 0,         /* pair p = elements (p, p + rot_dim/2) */
       HALOS_ROPE_INTERLEAVED = 1   /* pair p = elements (2p, 2p+1) */ };

/* For every token at position t and every pair p of every head of q and k, with a = t * freqs[p]:
 *     y0 = magnitude (x0 cos a - x1 sin a),  y1 = magnitude (x1 cos a + x0 sin a);    elements from rot_dim on are copied.
 * inverse: -a in the place of a, which is the gradient of the forward call.  The angle is reduced in 64-bit fixed
 * point before it is rounded, so that it is as exact at position 10^9 as at 1.  *_out may equal *_in (same strides). */
typedef struct halos_rope_args {
    uint32_t struct_size;
    int32_t device;
    void* stream;
    uint32_t dtype;                 /* HALOS_F32 | HALOS_BF16 | HALOS_F16 */
    uint32_t layout;                /* HALOS_ROPE_* */
    uint32_t inverse;
    uint32_t positions_64;          /* positions are int64, else int32 */
    int64_t batch, seq;
    uint32_t n_q, n_k;              /* heads; n_k = 0: no keys */
    uint32_t head_dim, rot_dim;     /* rot_dim even, <= head_dim <= 256 */
    float magnitude;
    uint32_t reserved;
    const double* freqs;            /* [rot_dim/2] radians per position */
    const void* positions;          /* NULL: token s stands at position_offset + s */
    int64_t position_stride[2];     /* batch, token */
    int64_t position_offset;
    const void *q_in, *k_in;
    void *q_out, *k_out;            /* [batch, seq, heads, head_dim] */
    int64_t q_in_stride[3], k_in_stride[3], q_out_stride[3], k_out_stride[3];  /* batch, token, head */
} halos_rope_args;
int halos_rope(const halos_rope_args* args);

/* ------------------------------------------------------------------ attention ----------- */

/* Query i stands at position t = i + sk - sq and sees the keys lo <= j < hi:
 *     lo = doc_start ? doc_start[b][i] : 0;   n = lens ? lens[b] : sk;   hi = t >= n ? 0 : causal ? min(n, t + 1) : n.
 *     s_ij = scale q_i.k_j;  lse_i = log sum_j exp s_ij;  p_ij = exp(s_ij - lse_i);  o_i = sum_j p_ij v_j.
 * A query that sees nothing has o = 0, lse = -infinity and gives no gradient.  Query head h reads key head
 * h / (n_q / n_kv).  Tokens at or past n, keys before the first or past the last one that any query sees, and queries that
 * see nothing may hold anything, NaN included.  All else has to be finite: a NaN or an infinity in a key or value that
 * some query sees, or that lies between such keys, may also reach queries that do not see it (zero times it is not zero).
 * Backward, with D_i = dout_i.o_i:   ds_ij = p_ij (dout_i.v_j - D_i);  dq_i = scale sum_j ds_ij k_j;
 * dk_j = scale sum ds_ij q_i and dv_j = sum p_ij dout_i over the queries of every head that reads the key head.
 * p and ds enter their matrix products in the inputs' type; all sums are in 32 bits.  Backward with HALOS_F16 they are taken times powers of two,
 * ds by the lengths of dout and v, so that gradients follow dout over its whole range, a loss scale included.
 * scale > 0, and scale log2(e) finite.  Scores are 32-bit sums, and lse one 32-bit number: a p that is formed from it is off by some 2^-23 |lse| of
 * itself, so that gradients of rows with |lse| in the tens of thousands lose what 16-bit types hold.  o is not formed from it.
 * dtype HALOS_BF16 or HALOS_F16 (HALOS_F32: UNSUPPORTED); head_dim a multiple of 8, <= 128; bases and strides of
 * q, k, v, dout multiples of 16 bytes, of the outputs and of o the same (else UNSUPPORTED). */
typedef struct halos_attention_args {
    uint32_t struct_size;
    int32_t device;
    void* stream;
    uint32_t dtype;
    uint32_t causal;
    int64_t batch, sq, sk;
    uint32_t n_q, n_kv, head_dim;
    float scale;
    const int32_t* doc_start;       /* [batch, sq] contiguous, or NULL */
    const int32_t* lens;            /* [batch], or NULL */
    const void *q, *k, *v;          /* [batch, s, heads, head_dim] */
    void* o;                        /* written by fwd, read by bwd */
    float* lse;                     /* [batch, n_q, sq] contiguous; written by fwd, read by bwd */
    const void* dout;               /* bwd only, from here on */
    void *dq, *dk, *dv;
    void* workspace;                /* 16-byte aligned, halos_attention_workspace bytes */
    uint64_t workspace_bytes;
    int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3];                 /* batch, token, head */
    int64_t dout_stride[3], dq_stride[3], dk_stride[3], dv_stride[3];
} halos_attention_args;
int halos_attention_fwd(const halos_attention_args* args);
int halos_attention_bwd(const halos_attention_args* args);
/* Bytes of workspace that halos_attention_bwd needs for these sizes and this dtype (halos_attention_fwd needs none). */
int halos_attention_workspace(const halos_attention_args* args, uint64_t* bytes);

/* ------------------------------------------------------------------ distillation loss ----------- */

/* One row per token: logits z over the vocabulary, label y, and the teacher's k entries (index, logit t); an entry
 * with index -1 is absent.  With T = temperature, m = mix, q1 = softmax(z), qT = softmax(z / T), and p = softmax(t / T)
 * over the entries that are there:
 *     loss = (1 - m) (-log q1[y]) + m T^2 sum_k p_k (log p_k - log qT[idx_k])
 *     dz_j = dloss [ (1 - m) (q1_j - [j = y]) + m T (qT_j - p_j) ]
 * labels NULL: no first term; k = 0 (or no entry there): no second.  A row with label == ignore_index has loss 0 and
 * gradient 0 whatever its logits hold.  Another label, or teacher index, outside the vocabulary makes that row's
 * loss and gradient NaN, and a teacher logit that is NaN or +infinity its loss and, at the teacher's entries, its gradient.  Of two
 * entries with the same index both count.  Logits of -infinity or of the type's lowest value are probability 0 beside others and get the
 * gradient that follows.  The statistics are one 32-bit number each, so a probability is off by some 2^-23 |lse| of itself, and
 * a row of nothing but the lowest value of a type with 8 bits of exponent has probability 1 in every place. */
typedef struct halos_distill_args {
    uint32_t struct_size;
    int32_t device;
    void* stream;
    uint32_t dtype;                 /* of logits and dlogits: HALOS_F32 | HALOS_BF16 | HALOS_F16 */
    uint32_t teacher_dtype;
    uint32_t labels_64, index_64;   /* int64, else int32 */
    int64_t rows, vocab;
    uint32_t k;                     /* <= 1024 */
    float temperature, mix;         /* temperature > 0, 0 <= mix <= 1 */
    uint32_t reserved;
    int64_t ignore_index;
    const void* logits;
    int64_t logits_stride;          /* between rows */
    const void* labels;             /* [rows] or NULL */
    const void* teacher_index;      /* [rows, k], rows teacher_index_stride apart */
    const void* teacher_logits;
    int64_t teacher_index_stride, teacher_logits_stride;
    float* loss;                    /* [rows]; fwd, fwd_bwd */
    float* stats;                   /* [rows, 2] = log sum exp z, log sum exp z/T; written by fwd (by fwd_bwd if not NULL), read by bwd */
    const float* dloss;             /* [rows]; bwd, fwd_bwd */
    void* dlogits;                  /* may equal logits (same stride); bwd, fwd_bwd */
    int64_t dlogits_stride;
} halos_distill_args;
int halos_distill_fwd(const halos_distill_args* args);
int halos_distill_bwd(const halos_distill_args* args);
/* Both in one pass over the logits, for a caller that knows dloss beforehand (1 / tokens, a weight per token). */
int halos_distill_fwd_bwd(const halos_distill_args* args);

/* ------------------------------------------------------------------ embedding ----------- */

/* fwd:  out[t][c] = scale weight[token[t]][c];   bwd:  dweight[v][c] = scale sum of dout[t][c] over the t with token[t] = v, and 0 where there
 * is none; accumulate: that is added to what dweight holds, and rows that no token names are not touched.
 * A token outside [0, vocab) gives a row of NaN and takes no part in the gradient.  dtype is that of out and dout, weight_dtype that of weight
 * and dweight, any pair of the three.  Products and sums are in 32 bits, the sums of a row in a fixed order, and each result is rounded once.
 * What is written may overlap nothing that is read. */
typedef struct halos_embedding_args {
    uint32_t struct_size;
    int32_t device;
    void* stream;
    uint32_t dtype, weight_dtype;
    uint32_t tokens_64;             /* int64, else int32 */
    uint32_t accumulate;
    int64_t tokens, vocab;          /* tokens <= 2^31 - 1, 0 < vocab < 2^31 - 1 */
    uint32_t dim;                   /* > 0 */
    float scale;
    const void* token;              /* [tokens] */
    const void* weight;             /* [vocab, dim]; fwd */
    int64_t weight_stride;          /* between rows, here and below */
    void* out;                      /* [tokens, dim]; fwd */
    int64_t out_stride;
    const void* dout;               /* [tokens, dim]; bwd, from here on */
    int64_t dout_stride;
    void* dweight;                  /* [vocab, dim] */
    int64_t dweight_stride;
    void* workspace;                /* 16-byte aligned, halos_embedding_workspace bytes */
    uint64_t workspace_bytes;
} halos_embedding_args;
int halos_embedding_fwd(const halos_embedding_args* args);
int halos_embedding_bwd(const halos_embedding_args* args);
/* Bytes of workspace that halos_embedding_bwd needs for these sizes (halos_embedding_fwd needs none). */
int halos_embedding_workspace(const halos_embedding_args* args, uint64_t* bytes);

/* ------------------------------------------------------------------ root-mean-square norm ----------- */

/* For every row of dim elements, with s = x + residual (x, without one) in 32 bits:
 *     rstd = 1 / sqrt(mean of s^2 + eps);  y = s rstd weight;  summed = s, rounded to dtype (written if there is a residual).
 * quantized: y is written in 8 bits (4 of exponent, 3 of mantissa, largest 448) as the nearest to the quotient y / scale in 32 bits, of two equally near
 * the even one, and scales has for every `group` neighbouring elements of a row (the last of a row may be fewer; group = 0: the whole row)
 * scale = max(max |y| (1/448), 2^-126), a product in 32 bits.
 * Rows of any size, those whose squares 32 bits do not hold included, give what the formula does: 1 / 0 is infinity, a NaN makes its row NaN, an
 * infinity its own place and the rest 0.  Where rstd is above what 32 bits hold (a root mean square below 2^-128) it is infinity, y is what the formula
 * gives, and bwd, which has rstd alone, gives no finite gradients.
 * bwd, from s as it was rounded (x, without a residual), rstd, dy and dsummed (the gradient of summed, or NULL), with u = s rstd and g = dy weight:
 *     dx = rstd (g - u mean of g u) + dsummed,  which is the gradient of x and of residual;   dweight = sum over rows of dy u.
 * The sums of dweight are in 32 bits and a fixed order, and each result is rounded once.
 * Rows are those of three outer sizes (1 where there are fewer) with strides of their own; the elements of a row lie side by side.  Rows that are
 * written may overlap none that are read or written. */
typedef struct halos_rms_norm_args {
    uint32_t struct_size;
    int32_t device;
    void* stream;
    uint32_t dtype, weight_dtype;   /* of weight and dweight */
    uint32_t quantized;
    uint32_t group;                 /* 0, 32, 64 or 128; quantized */
    int64_t size[3];                /* product <= 2^31 - 1 */
    uint32_t dim;                   /* 0 < dim < 2^30 */
    float eps;                      /* >= 0, finite */
    const void* x;                  /* fwd */
    const void* residual;           /* fwd, or NULL */
    void* summed;                   /* written by fwd if there is a residual, read by bwd */
    void* y;                        /* fwd */
    float* scales;                  /* [rows, groups of a row] contiguous; fwd, quantized */
    float* rstd;                    /* [rows] contiguous; written by fwd, read by bwd */
    const void* weight;             /* [dim] */
    const void* dy;                 /* bwd, from here on */
    const void* dsummed;            /* or NULL */
    void* dx;
    void* dweight;                  /* [dim] */
    void* workspace;                /* 16-byte aligned, halos_rms_norm_workspace bytes */
    uint64_t workspace_bytes;
    int64_t x_stride[3], residual_stride[3], summed_stride[3], y_stride[3], dy_stride[3], dsummed_stride[3], dx_stride[3];
} halos_rms_norm_args;
int halos_rms_norm_fwd(const halos_rms_norm_args* args);
int halos_rms_norm_bwd(const halos_rms_norm_args* args);
/* Bytes of workspace that halos_rms_norm_bwd needs for these sizes (halos_rms_norm_fwd needs none). */
int halos_rms_norm_workspace(const halos_rms_norm_args* args, uint64_t* bytes);

/* ------------------------------------------------------------------ gradients ----------- */

/* n = sqrt(sum of the squares of every element of every gradient), f = n > max_norm ? max_norm / n : 1  (n, f in 64 bits; a NaN n has f = 1;
 * elements are multiplied by f, or rate f, as rounded to 32 bits where those hold it, that is from 2^-126 on, and in 64 bits below)
 *     halos_grad_norm    *norm = n
 *     halos_clip_grads   *norm = n;  out_i = f grad_i;  out_i may be grad_i
 *     halos_sgd_step     out_i = out_i - rate f grad_i;  *norm = n where norm is not NULL.  norm NULL: no norm is formed, f = 1
 * Each element is rounded once, to its type.  Squares are added up in groups of eight in 32 bits where that holds them, else and from there on in
 * 64 bits, in a fixed order.  In place and with f = 1 nothing is written.  Tensors are dense runs of numel elements of any type each; those that
 * are written may overlap neither one another nor another gradient.  The arrays are read before the call returns. */
typedef struct halos_grads_args {
    uint32_t struct_size;
    int32_t device;
    void* stream;
    uint64_t count;
    const void* const* grads;       /* [count] device pointers, in host memory as the other arrays */
    void* const* outs;              /* [count]; clip, step */
    const int64_t* numel;           /* [count] */
    const uint8_t* grad_dtypes;     /* [count] */
    const uint8_t* out_dtypes;      /* [count]; clip, step */
    float max_norm;                 /* >= 0; clip, and step with a norm */
    float rate;                     /* finite; step */
    float* norm;                    /* device */
    void* workspace;                /* 16-byte aligned, halos_grads_workspace bytes; none is needed without a norm */
    uint64_t workspace_bytes;
} halos_grads_args;
int halos_grad_norm(const halos_grads_args* args);
int halos_clip_grads(const halos_grads_args* args);
int halos_sgd_step(const halos_grads_args* args);
/* Bytes of workspace for `count` tensors on this device. */
int halos_grads_workspace(const halos_grads_args* args, uint64_t* bytes);

#ifdef __cplusplus
}
#endif
#endif /* HALOS_STEP_H */
