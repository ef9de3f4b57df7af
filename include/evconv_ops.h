/* evconv_ops.h - sequence operators of the MI355X (gfx950) library: what mixes the feature vectors
 * of successive time windows behind (or beside) an incremental net.
 *
 *   evconv_delta_rule     the gated delta rule: a matrix per head and stream that every token decays,
 *                         corrects along its key and reads with its query; whole recordings
 *                         (chunked) and single tokens (recurrent) through one call
 *   evconv_block_norm     the norms after and before a block, with the block's gate, residual scale
 *                         and residual sum between them, and the 8-bit rows of the result
 *   evconv_quant_matmul   product of 8-bit integers with one scale per row (token) and per column
 *                         (channel)
 *
 * Plain C, in libevconv.so beside the net's calls, with their statuses (evconv.h).  The text of the
 * last failed call of a host thread is evconv_last_error(NULL).  All pointers are DEVICE memory owned by
 * the caller.  A call checks its arguments, enqueues kernels on `hip_stream` (NULL = the default
 * stream) and returns: it neither allocates nor synchronises nor keeps anything, so it may be captured
 * into a HIP graph, and calls on different streams do not meet as long as their workspaces and
 * outputs are different.  A count of zero tokens (rows) is a valid call that does nothing, except that the
 * delta rule hands the states on.
 *
 * Strides are in elements.  Rows (the last dimension) are contiguous.  Alignment beyond that of an
 * element is not required, but rows of 16-byte multiples at 16-byte addresses are read in wide loads.
 * Outputs may not overlap inputs except where it is said.
 */
#ifndef EVCONV_OPS_H
#define EVCONV_OPS_H

#include "evconv.h"

#ifdef __cplusplus
extern "C" {
#endif

#define EVCONV_OPS_ABI_VERSION 1

/* ---- the gated delta rule -------------------------------------------------------------------------
 * Per sequence and value head, with S a d_k x d_v matrix (rows: key channels) that starts as the given state:
 *   S  = exp(g_t) S
 *   d  = beta_t (v_t - S' k_t)
 *   S += k_t d'
 *   o_t = scale * S' q_t
 * Value head h uses key (query) head h / (heads_v / heads_k).  q, k, v and o are of `dtype`; the state is
 * fp32, and everything that reaches it is computed in fp32 or as sums of bf16 parts that hold an fp32
 * value's 24 bits.  o of a bf16 call is rounded once, token by token from fp32, in chunks from a sum of terms of 16 bits each: where
 * terms cancel, it is off by up to some 2^-16 of the largest instead of itself.
 *
 * EVCONV_DELTA_NORMALIZE: q_t and k_t are first divided by sqrt(sum of squares + 1e-6).
 * EVCONV_DELTA_RAW_GATES: `gate` and `beta` hold what a projection gave, a_t and b_t:
 *   g_t = -a_scale[h] * log(1 + exp(a_t + dt_bias[h])),  beta_t = 1 / (1 + exp(-b_t)).
 * Without it they hold g_t (log of the decay; -inf forgets the state) and beta_t.
 *
 * A value that is not finite makes what depends on it NaN (or infinite): outputs of its sequence and
 * head from its token on, and the state; never an earlier token's output or another sequence's.
 * A finite value of 3.39e38 and more counts as infinite, and so does a query or a key whose sum of squares is beyond
 * fp32 (without EVCONV_DELTA_NORMALIZE: may). */
#define EVCONV_DELTA_NORMALIZE 1u
#define EVCONV_DELTA_RAW_GATES 2u

/* [n_tokens][heads][d] (gate, beta: [n_tokens][heads_v]) */
typedef struct {
  const void* data;
  int64_t token_stride, head_stride;
} evconv_heads;

typedef struct {
  int32_t abi_version;        /* EVCONV_OPS_ABI_VERSION */
  int32_t dtype;              /* of q, k, v, o: EVCONV_F32 or EVCONV_BF16 */
  int32_t gate_dtype;         /* of gate and beta: EVCONV_F32 or EVCONV_BF16 */
  uint32_t flags;             /* EVCONV_DELTA_* */
  int32_t heads_k, heads_v;   /* heads_v a multiple of heads_k; 1..1024 */
  int32_t d_k, d_v;           /* 1..256 */
  int32_t n_seq;              /* sequences, 1..65535 */
  int32_t n_slots;            /* states that state_in and state_out have room for */
  int64_t n_tokens;           /* of all sequences together, below 2^31 - 64 */
  float scale;                /* of the outputs */
  evconv_heads q, k, v, gate, beta;
  void* o;                    /* [n_tokens][heads_v][d_v] */
  int64_t o_token_stride, o_head_stride;
  const float *a_scale, *dt_bias; /* fp32 [heads_v] each; EVCONV_DELTA_RAW_GATES only (then without tokens too) */
  const int32_t* seq_offsets; /* [n_seq + 1] ascending token indices, from 0 to n_tokens; sequence i is tokens
                               * [offsets[i], offsets[i+1]).  NULL: n_seq sequences of n_tokens / n_seq
                               * (a multiple) tokens.  A pair that descends is an empty sequence, what is out of
                               * range is cut off there, and tokens of no sequence have no output.  Sequences
                               * that have tokens must not overlap and stand in the order of their tokens */
  const int32_t* slots;       /* [n_seq]: the state that sequence i continues and leaves; NULL: i.  Outside
                               * [0, n_slots): it starts from zero and leaves none.  No two alike */
  const float* state_in;      /* [n_slots][heads_v][d_k][d_v], or NULL: all start from zero */
  float* state_out;           /* the same, may be state_in; or NULL.  Slots of no sequence stay as they are */
} evconv_delta_args;

/* A call whose largest launch would have 2^32 threads or more (some millions of sequences times heads: a launch has 64 to 1536 to
 * each) is EVCONV_ERR_UNSUPPORTED.
 * Bytes of device workspace the call needs: 0 where nothing passes between launches (a few tokens to a
 * sequence; bf16 keys of up to 128 channels, unless few sequences of some length are split over the chip). */
evconv_status evconv_delta_rule_workspace(const evconv_delta_args* args, size_t* bytes);
/* `workspace`: 256-byte aligned, free to be used again once the call's kernels are done. */
evconv_status evconv_delta_rule(const evconv_delta_args* args, void* workspace, size_t workspace_bytes,
                                void* hip_stream);

/* ---- norms around a block ---------------------------------------------------------------------------
 * Per row of `dim` values, all in fp32, each output rounded once (the sigmoid of bf16 rows by the hardware's exponential and
 * reciprocal, good to about 2^-20 of itself, also where only the 8-bit rows are wanted):
 *   t = norm(branch) * post_weight + post_bias     in groups of `group` values (heads), each with a norm of its own
 *   t = t * act(gate)                              act: 1, sigmoid(z) or z * sigmoid(z)
 *   x' = x + res_scale * t                         (x NULL: x' = res_scale * t;  branch NULL: x' = x)
 *   h = norm(x') * pre_weight + pre_bias           over the whole row, if pre_norm is set (else h = x')
 *   q = rint(h * (127 * (1 / m))), q_scale = m / 127   each operation rounded to fp32; m = max |h| of the row;
 *                                                  a row of zeros has q = 0 and scale 0, one with a value that is
 *                                                  not finite q = 0 and scale NaN; where 1 / m overflows, q = 0
 * norm: EVCONV_NORM_RMS x / sqrt(mean(x^2) + eps), EVCONV_NORM_LAYER (x - mean) / sqrt(variance + eps).
 * Every operand that is NULL is left out of its formula; outputs that are NULL are not written.  x_out may be x. */
typedef enum { EVCONV_NORM_RMS = 0, EVCONV_NORM_LAYER = 1 } evconv_norm;
typedef enum { EVCONV_GATE_NONE = 0, EVCONV_GATE_SIGMOID = 1, EVCONV_GATE_SILU = 2 } evconv_gate;

typedef struct {
  int32_t abi_version;  /* EVCONV_OPS_ABI_VERSION */
  int32_t dtype;        /* of x, branch, gate, x_out, h_out: EVCONV_F32 or EVCONV_BF16 */
  int32_t norm;         /* evconv_norm, of both */
  int32_t gate_act;     /* evconv_gate */
  int32_t pre_norm;     /* 0 or 1 */
  int32_t dim;          /* 1..16384 */
  int32_t group;        /* divides dim; dim itself, or 8..512 with dim / group times the power of two
                         * that holds it at most 16384 */
  float eps;
  int64_t rows;         /* below 2^31 */
  const void *x, *branch, *gate;
  int64_t x_stride, branch_stride, gate_stride; /* elements between rows */
  const float *post_weight, *post_bias;         /* [group] */
  const float* res_scale;                       /* [dim] */
  const float *pre_weight, *pre_bias;           /* [dim] */
  void *x_out, *h_out;
  int64_t x_out_stride, h_out_stride;
  int8_t* q;            /* [rows][q_stride], columns dim .. q_stride become zero */
  int64_t q_stride;     /* bytes, a multiple of 128, at least dim and less than dim + 128 */
  float* q_scale;       /* [rows] */
} evconv_norm_args;

evconv_status evconv_block_norm(const evconv_norm_args* args, void* hip_stream);

/* ---- product in 8-bit integers ------------------------------------------------------------------------
 *   y[m][n] = act(a_scale[m] * b_scale[n] * sum_k a[m][k] b[n][k] + bias[n])
 * The sums are exact (int32), the rest is fp32, rounded once to `dtype`.  a and b are rows of int8 as
 * evconv_block_norm writes them: 16-byte aligned, strides multiples of 128 bytes of at least k, zeros behind
 * column k (of one of the two at least), no value -128.  A weight is quantised by the same call: its rows are
 * the output channels.  act: EVCONV_ACT_NONE, RELU, SIGMOID, TANH. */
typedef struct {
  int32_t abi_version;  /* EVCONV_OPS_ABI_VERSION */
  int32_t dtype;        /* of y: EVCONV_F32 or EVCONV_BF16 */
  int32_t act;          /* evconv_act */
  int32_t n, k;         /* n at most 2^24; k at most 131072: a sum of more products may not fit 32 bits */
  int64_t m;            /* below 2^31, and fewer than 2^23 tiles of 256 x 256 in y */
  const int8_t *a, *b;
  int64_t a_stride, b_stride; /* bytes */
  const float *a_scale, *b_scale, *bias; /* fp32 [m], [n], [n] or NULL */
  void* y;
  int64_t y_stride;     /* elements, at least n */
} evconv_quant_args;

evconv_status evconv_quant_matmul(const evconv_quant_args* args, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* EVCONV_OPS_H */
