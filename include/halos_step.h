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
 *
 * Conventions
 *  - No context is needed.  Every call takes one args struct, whose first field is its size (checked), checks it
 *    on the host, makes args->device the calling thread's current device and leaves it so, enqueues its kernels on
 *    args->stream (cudaStream_t, NULL = the legacy default stream) and returns without waiting.  Tensors are
 *    borrowed until those kernels have completed in stream order.
 *  - Pointers are device pointers.  Strides are in elements; the innermost dimension is contiguous.
 *  - Nothing is allocated but 256 bytes of host memory in the first call: workspaces are the caller's
 *    (halos_attention_workspace says how much).
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

#ifdef __cplusplus
}
#endif
#endif /* HALOS_STEP_H */
