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
 *   evconv_cache_append   keys and values of new tokens into a paged cache (bf16 or 4 bits), with the norm
 *                         and the rotation of their heads and their queries' on the way
 *   evconv_cache_read     cached keys and values back as rows
 *   evconv_cache_attend   attention of queries over the cache, whole or over chosen pages
 *   evconv_cache_select   the pages that a bound on their scores makes worth a query's look
 *
 * Plain C, in libevconv.so beside the net's calls, with their statuses (evconv.h).  The text of the
 * last failed call of a host thread is evconv_last_error(NULL).  All pointers are DEVICE memory owned by
 * the caller.  A call checks its arguments, enqueues kernels on `hip_stream` (NULL = the default
 * stream) and returns: it neither allocates nor synchronises nor keeps anything, so it may be captured
 * into a HIP graph, and calls on different streams do not meet as long as their workspaces and
 * outputs are different.  A count of zero tokens (rows) is a valid call that does nothing, except that the
 * delta rule hands the states on.  Arguments that are device memory (tables, positions, offsets) cannot be refused: what of
 * them is out of range is left out, as said at each call, and nothing outside the given buffers is read or written.
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

/* ---- a paged cache of keys and values ----------------------------------------------------------------
 * Tokens of n_seq sequences ("streams") in pages of `page` tokens: table[s * table_stride + i] is the page that holds
 * sequence s's tokens i * page and on.  A sequence has past[s] tokens there; the call's tokens continue it (or look back):
 * token i of sequence s has position past[s] + i.  past is only read: who appends moves it on, once for all layers.
 * A table entry outside [0, n_pages), a negative position and one of width * page and more hold nothing: what is appended
 * there is dropped, what looks there sees nothing.  Pages may be read by several sequences; a page that a call appends to must be
 * one sequence's alone, and stand once among the entries that it appends to (elsewhere in the row as often as one likes: pages may go round).
 *
 * Channels are padded to dp = 32, 64, 96, 128, 192 or 256 with zeros.  All tensors are contiguous, at 16-byte addresses:
 *   EVCONV_CACHE_BF16   k [n_pages][heads][page][dp], v [n_pages][heads][dp][page]  (channels of v in rows: both are
 *                       operands of the matrix instructions as they stand)
 *   EVCONV_CACHE_FP4    the same of 4-bit floating-point values (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign), two to a byte,
 *                       the first in the low bits: neighbouring channels of k, neighbouring tokens of v; times
 *                       k_scale, v_scale fp32 [n_pages][heads][page].  Of a row x with m = max |x|: scale = m / 6, codes
 *                       the nearest of 6 x / m (each operation rounded to fp32), ties to the even code
 *   bounds              bf16 [n_pages][heads][2][dp]: least and largest of bf16(k) per channel over what was appended
 *                       since the page's first token; or NULL (no evconv_cache_select then)
 * A key row with a value that is not finite (in bf16: 3.39e38 and more too) makes what looks at its token NaN; so does a value row.  In
 * 4 bits its scale is NaN; in bf16 the row of the token's key is, also for its value (v itself holds finite values only: one that is not
 * would reach queries that do not see it).  Other tokens and queries are as without it. */
typedef enum { EVCONV_CACHE_BF16 = 0, EVCONV_CACHE_FP4 = 1 } evconv_cache_kind;

typedef struct {
  int32_t kind;    /* evconv_cache_kind */
  int32_t n_pages; /* at least 1 */
  int32_t heads;   /* of keys and values, 1..1024 */
  int32_t page;    /* 32, 64, 128 or 256 */
  int32_t d;       /* channels of a head, 1..256 */
  void *k, *v;
  float *k_scale, *v_scale; /* EVCONV_CACHE_FP4 only */
  void* bounds;
} evconv_cache;

typedef struct {
  int32_t n_seq;               /* sequences, 1..65535 */
  int32_t width;               /* entries of a table row, at least 1; width * page below 2^30 */
  int64_t n_tokens;            /* of all sequences together, below 2^31 - 64 */
  const int32_t* table;        /* [n_seq][width] */
  int64_t table_stride;
  const int32_t* past;         /* [n_seq] */
  const int32_t* seq_offsets;  /* [n_seq + 1] ascending, from 0 to n_tokens: sequence s is tokens [offsets[s], offsets[s+1]).
                                * NULL: n_tokens / n_seq (a multiple) tokens each.  Tokens of no sequence have no output.  Offsets
                                * that do not ascend: which tokens are dealt with is not said */
} evconv_tokens;

/* Per head: norm (q_norm, k_norm: weights, NULL: none): x / sqrt(mean(x^2) + eps) * weight, the sum in 64 bits; then the
 * rotation (freqs): pairs (a, b) of the first `rot` channels become (a cos - b sin, b cos + a sin) of the angle position *
 * freqs[i], taken in 64 bits (one of 2^45 and more turns nothing); all else in fp32.  k and v then go to the cache, q to q_out (rounded once; may be q). */
typedef enum { EVCONV_PAIRS_HALVES = 0, EVCONV_PAIRS_NEIGHBOURS = 1 } evconv_pairs; /* (i, i + rot / 2) or (2 i, 2 i + 1) */

typedef struct {
  int32_t abi_version; /* EVCONV_OPS_ABI_VERSION */
  int32_t dtype;       /* of q, k, v, q_out: EVCONV_F32 or EVCONV_BF16 */
  evconv_cache cache;
  evconv_tokens tokens;
  int32_t heads_q;     /* 0: no queries; else 1..1024 */
  int32_t rot;         /* channels that are rotated, even, at most d; 0: none */
  int32_t pairs;       /* evconv_pairs */
  float eps;
  evconv_heads q, k, v; /* [n_tokens][heads][d] */
  void* q_out;
  int64_t q_out_token_stride, q_out_head_stride;
  const float *q_norm, *k_norm; /* fp32 [d] or NULL */
  const float* freqs;           /* fp32 [rot / 2] */
  const int64_t* positions;     /* [n_tokens]: of the angles; NULL: past[s] + i */
} evconv_append_args;

evconv_status evconv_cache_append(const evconv_append_args* args, void* hip_stream);

/* Keys and values of the tokens past[s] + i as rows [n_tokens][heads][d] of `dtype`; tokens that the cache does not hold are zero. */
typedef struct {
  int32_t abi_version;
  int32_t dtype; /* of k and v: EVCONV_F32 or EVCONV_BF16 */
  evconv_cache cache;
  evconv_tokens tokens;
  void *k, *v;   /* contiguous */
} evconv_read_args;

evconv_status evconv_cache_read(const evconv_read_args* args, void* hip_stream);

/* o = sum over the tokens t that a query sees of softmax_t(scale * q . k_t) v_t, statistics and sums in fp32; a query that
 * sees none gets zeros.  Query head h uses key head h / (heads_q / cache.heads).  Seen are, of the query's sequence, tokens 0 .. its own
 * position (causal: of the last `window` ones of them), or all past[s] (else); of those the ones in chosen pages, if `selected`
 * is given.  Products with bf16 queries are exact; fp32 queries and the weights of fp32 calls enter them as three bf16 parts
 * (24 bits).  The weights of bf16 calls enter as two (16 bits) with chosen pages, and for sequences of up to 16 rows (tokens x query heads
 * of a key head) unless the call has seq_offsets and 64 rows to a sequence or more on average; otherwise rounded to bf16, which is a
 * rounding of the output's own size (sequences of few rows then too: what a row sees is the same, its last bits may hang on the call).
 * Weights go up to 2^8, and are divided by their sum last: values whose 2^8-fold sum is beyond fp32 are too large.  A finite query value of 3.39e38 and more counts as infinite. */
typedef struct {
  int32_t abi_version;
  int32_t dtype;    /* of q and o: EVCONV_F32 or EVCONV_BF16 */
  evconv_cache cache;
  evconv_tokens tokens;
  int32_t heads_q;  /* a multiple of cache.heads, up to 1024 */
  int32_t causal;   /* 0 or 1 */
  int32_t window;   /* 0: no limit; only with causal */
  int32_t count;    /* pages of a query in `selected`, 1..65536 */
  int64_t max_len;  /* no sequence has more tokens than that with the call's; what is behind is not seen.  0: width * page */
  float scale;
  evconv_heads q;   /* [n_tokens][heads_q][d] */
  void* o;
  int64_t o_token_stride, o_head_stride;
  const int32_t* selected; /* [n_tokens][cache.heads][count]: table entries of the query's sequence, what is outside
                            * [0, width) for none; one that is there twice counts twice.  NULL: all.  Not with window */
} evconv_attend_args;

evconv_status evconv_cache_attend_workspace(const evconv_attend_args* args, size_t* bytes);
evconv_status evconv_cache_attend(const evconv_attend_args* args, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Which `count` pages of its sequence each query (and key head) looks at, ascending, then -1.  With c the page of the query's
 * own position: the first `first` pages and the last `last` ones up to c; then, of the others below c, those of the highest
 *   score = max over the query heads of the key head of  sum over channels of max(q lo, q hi)
 * (no query . key product of the page is larger with its keys as bf16, which the bounds are of; with those that a cache in 4 bits holds
 * one may be, by their rounding: of a key's value about a sixth of its row's largest at most), taken in 64 bits and rounded to fp32;
 * ties: the lower page.  A score that is NaN is the highest.  A page that is not there is not chosen. */
typedef struct {
  int32_t abi_version;
  int32_t dtype;   /* of q */
  evconv_cache cache;
  evconv_tokens tokens;
  int32_t heads_q;
  int32_t count;   /* 1..65536 */
  int32_t first;   /* at least 0 */
  int32_t last;    /* at least 1, first + last at most count: the own page's bounds hold tokens that the query does not see */
  int64_t max_len; /* as of evconv_cache_attend */
  evconv_heads q;
  int32_t* selected; /* [n_tokens][cache.heads][count] */
} evconv_select_args;

/* Four bytes for every query, key head and page of max_len. */
evconv_status evconv_cache_select_workspace(const evconv_select_args* args, size_t* bytes);
evconv_status evconv_cache_select(const evconv_select_args* args, void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* EVCONV_OPS_H */
