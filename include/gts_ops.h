/*
 * gts_ops.h — C ABI of the operators of libgts.so: rotary positions, appending
 * keys and values to a paged cache, attention over that cache for a batch that
 * shares a prefix; and the rest of a decoder layer, forward and backward: layer
 * norms, matrix products with their epilogue, attention over whole prompts.
 *
 * They are the kernels of the steps whose tile graphs the package simulates
 * (a decoder layer, its products, flash attention, split-KV decode), run on the
 * card itself: a simulated makespan can stand beside a measured time.
 *
 * Conventions are those of gts.h: int status (GTS_OK or a negative GTS_E_*
 * code, gts_last_error() says which value), no exception crosses the boundary,
 * the caller owns every buffer, streams are void* (a hipStream_t), work is
 * enqueued and not waited for, nothing is allocated, and every call may be
 * captured into a graph.  Pointers are device pointers unless a comment says
 * host.  Strides count elements; the last dimension of every tensor is
 * contiguous.  All sums, softmax statistics and rotations are in 32 bits; a
 * result is rounded once, to the type it is stored in.  One value more is
 * rounded: attention over a 16-bit cache whose rows are aligned to 16 bytes
 * multiplies the values by softmax weights in the cache's type (their sum, and so
 * lse, keeps them in 32 bits).  So do attention over prompts and its gradient with
 * weights and their gradients (in float16 scaled by powers of two that keep them
 * in its range), and gts_linear_backward's dz is in its tensors' type.
 */
#ifndef GTS_OPS_H
#define GTS_OPS_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- element types ------------------------------------------------------- */
#define GTS_F32  0u
#define GTS_BF16 1u
#define GTS_F16  2u

/* ---- rotation flags ------------------------------------------------------ */
#define GTS_ROTARY_INTERLEAVED 1u /* pairs (2i, 2i + 1); else (i, i + rot_dim / 2) */
#define GTS_ROTARY_BACKWARD    2u /* the gradient: the transposed rotation         */
/* ---- append flags (beside GTS_ROTARY_INTERLEAVED) ------------------------ */
#define GTS_APPEND_ZERO_REST   4u /* q_out of tokens without a place: zeros        */

/* ---- limits -------------------------------------------------------------- */
#define GTS_OPS_MAX_DIM  512u     /* head dim of a rotation or an append     */
#define GTS_OPS_MAX_ATTN 256u     /* head dim of attention                   */
#define GTS_OPS_MAX_PAGE 65536u   /* tokens of a page (a power of two)       */
#define GTS_OPS_MAX_WIDTH 16777216u /* columns of a norm or a product        */

/* table[p * rot_dim + i] = scale * cos(p * freq[i]) and
 * table[p * rot_dim + rot_dim / 2 + i] = scale * sin(p * freq[i]) for
 * p < n_positions, i < rot_dim / 2, computed in 64 bits and rounded once.
 * freq: host array [rot_dim / 2], radians per position, read before return. */
int gts_rotary_table(float *table, uint32_t n_positions, uint32_t rot_dim, const double *freq, double scale,
                     void *hip_stream);

/* Rotary positions.  For every (batch, token, head) of x [batch, tokens,
 * heads, dim] with position p, row p of the table giving c_i, s_i, and each
 * pair (a, b) of the leading rot_dim values:
 *   forward   a' = a c - b s,  b' = b c + a s
 *   backward  a' = a c + b s,  b' = b c - a s
 * Values behind rot_dim are copied.  out == x with equal strides rotates in
 * place.  A position outside [0, n_positions) gives NaN in the rotated part. */
typedef struct gts_rotary_args {
  const void *x;
  void *out;
  const void *positions;   /* i32 or i64 (pos_bytes 4 or 8)                   */
  const float *table;      /* [n_positions][rot_dim] as gts_rotary_table      */
  int64_t x_stride[3];     /* batch, token, head                              */
  int64_t out_stride[3];
  int64_t pos_stride[2];   /* batch, token (0 shares a row of positions)      */
  int64_t table_stride;    /* of a position                                   */
  uint32_t batch, tokens, heads, dim, rot_dim, n_positions;
  uint32_t dtype, pos_bytes, flags;
  uint32_t reserved;       /* 0 */
} gts_rotary_args;
int gts_rotary(const gts_rotary_args *a, void *hip_stream);

/* A paged cache: page p holds `page` tokens of every head.  Any order of
 * pages, slots and heads in memory (the strides say which). */
typedef struct gts_kv_cache {
  void *k, *v;
  int64_t k_stride[3], v_stride[3];  /* page, slot, head                      */
  uint32_t n_pages, page, heads, dim;
  uint32_t dtype, reserved;
} gts_kv_cache;

/* A batch of sequences and their new tokens.  Sequence b has the new tokens
 * starts[b] .. starts[b + 1) of the call's tensors (starts = NULL: tokens /
 * batch each) and, with them, lens[b] keys of its own; own key j is in slot
 * j % page of page page_table[b][j / page].  New token i of n is own key
 * lens[b] - n + i, at position prefix_len + that.  A page number outside
 * [0, n_pages) and an own key past max_pages * page name no memory: nothing
 * is written there, and attention has no such key. */
typedef struct gts_kv_batch {
  const int32_t *starts;     /* [batch + 1] ascending, or NULL               */
  const int32_t *lens;       /* [batch]                                      */
  const int32_t *page_table; /* [batch][max_pages]                           */
  int64_t table_stride;
  uint32_t batch, tokens, max_pages, prefix_len;
} gts_kv_batch;

/* Writes the new tokens' keys (rotated, with a table) and values into the
 * cache; with q, also writes q rotated to q_out (which may be q).  A
 * token outside every sequence, or whose own index is negative, has no place:
 * it writes nothing, or with GTS_APPEND_ZERO_REST zeros to its rows of q_out.
 * Two tokens of one call must not name the same slot. */
typedef struct gts_append_args {
  gts_kv_cache cache;
  gts_kv_batch batch;
  const void *k, *v;       /* [tokens][heads][dim]                            */
  const void *q;           /* [tokens][q_heads][dim] or NULL                  */
  void *q_out;
  int64_t k_stride[2], v_stride[2], q_stride[2], q_out_stride[2]; /* token, head */
  const float *table;      /* NULL: nothing is rotated                        */
  int64_t table_stride;
  uint32_t q_heads, rot_dim, n_positions, flags;
} gts_append_args;
int gts_append_kv(const gts_append_args *a, void *hip_stream);

/* Attention of the new tokens over the cache.  Query head h reads key-value
 * head h / (q_heads / heads).  Token i of a sequence sees every key of the
 * prefix (key j in slot j % page of page prefix_pages[j / page], j <
 * prefix_len, the same for all sequences) and its own keys 0 .. lens[b] - n + i:
 *   out = sum_j w_j v_j,  w = softmax_j(scale * q . k_j),
 *   lse = log sum_j exp(scale * q . k_j).
 * A token without a key, or outside every sequence, has out = 0 and
 * lse = -inf.  One that has keys, but none whose score is above -inf, is 0 / 0:
 * out = NaN and lse = -inf.  A score of +inf or NaN makes both NaN.  lse may be
 * NULL.  The scratch needs no initialisation.
 * 16-bit caches whose rows of q, k and v are aligned to 16 bytes, with a dim of
 * whole 16 bytes and an even out, read the prefix once for all sequences; any
 * other call reads each key for every query head that sees it. */
typedef struct gts_attention_args {
  gts_kv_cache cache;
  gts_kv_batch batch;
  const void *q;             /* [tokens][q_heads][dim]                        */
  void *out;                 /* the same shape                                */
  float *lse;                /* [tokens][q_heads] contiguous, or NULL         */
  int64_t q_stride[2], out_stride[2]; /* token, head                          */
  const int32_t *prefix_pages;        /* [n_prefix_pages]                     */
  uint32_t n_prefix_pages, q_heads;
  float scale;
  uint32_t reserved;         /* 0 */
  void *scratch;
  uint64_t scratch_bytes;
} gts_attention_args;
int gts_shared_prefix_attention(const gts_attention_args *a, void *hip_stream);

/* Bytes of scratch for a batch of these sizes (whatever its lengths). */
int gts_shared_prefix_attention_scratch(uint32_t batch, uint32_t tokens, uint32_t q_heads, uint32_t kv_heads,
                                        uint32_t dim, uint64_t *bytes);

/* ---- layer norm ------------------------------------------------------------ */
#define GTS_NORM_CENTER 1u /* the mean is taken off; else it is 0 (RMS norm)    */

/* For every row x of dim values:
 *   mu = mean(x) (with GTS_NORM_CENTER, else 0), r = 1 / sqrt(mean((x - mu)^2) + eps),
 *   out = (x - mu) r weight + bias.
 * weight, bias [dim] may be NULL (1 and 0).  mean and rstd (float [rows], may be
 * NULL) receive mu and r for the backward pass.  out may be x with the same stride. */
typedef struct gts_norm_args {
  const void *x;
  void *out;
  const void *weight, *bias;
  float *mean, *rstd;
  int64_t x_stride, out_stride;   /* of a row */
  uint32_t rows, dim;
  float eps;
  uint32_t dtype, flags;
  uint32_t reserved;              /* 0 */
} gts_norm_args;
int gts_layer_norm(const gts_norm_args *a, void *hip_stream);

/* Its gradient.  With h = (x - mean) rstd and g = dy weight:
 *   dx = rstd (g - mean(g) - h mean(g h)) (without GTS_NORM_CENTER no mean(g)),
 *   dweight = sum over rows of dy h,  dbias = sum over rows of dy.
 * dx, dweight and dbias may each be NULL; dx may be dy or x with the same stride.
 * The order of the sums is fixed: the same bits on every run. */
typedef struct gts_norm_grad_args {
  const void *dy, *x, *weight;
  const float *mean, *rstd;       /* mean: NULL without GTS_NORM_CENTER         */
  void *dx, *dweight, *dbias;
  int64_t dy_stride, x_stride, dx_stride;
  uint32_t rows, dim, dtype, flags;
  void *scratch;                  /* needs no initialisation                    */
  uint64_t scratch_bytes;
} gts_norm_grad_args;
int gts_layer_norm_backward(const gts_norm_grad_args *a, void *hip_stream);
int gts_layer_norm_backward_scratch(uint32_t rows, uint32_t dim, uint64_t *bytes);

/* ---- matrix product with its epilogue ---------------------------------------- */
#define GTS_ACT_NONE      0u
#define GTS_ACT_RELU      1u
#define GTS_ACT_GELU      2u /* z times the normal distribution below z          */
#define GTS_ACT_GELU_TANH 3u /* z / (1 + exp(-2 sqrt(2/pi) (z + 0.044715 z^3)))  */
#define GTS_ACT_SILU      4u /* z / (1 + exp(-z))                                */

#define GTS_MATMUL_A_COLUMNS 1u /* a is stored [k][m], else [m][k]               */
#define GTS_MATMUL_B_COLUMNS 2u /* b is stored [k][n], else [n][k]               */

/*   z[i][j] = sum over l < k of a[i][l] b[j][l] + bias[j],
 *   out = act(z) gate + residual.
 * bias [n], gate and residual [m][n] may be NULL.  preact (NULL or [m][n])
 * receives z for the backward pass.  Everything up to out is in 32 bits.  out may be
 * gate or residual with the same stride; out and preact share no other memory. */
typedef struct gts_matmul_args {
  const void *a, *b;
  void *out, *preact;
  const void *bias, *gate, *residual;
  int64_t a_stride, b_stride, out_stride, preact_stride, gate_stride, residual_stride; /* of a row as stored */
  uint32_t m, n, k;
  uint32_t dtype, activation, flags;
  void *scratch;                  /* needs no initialisation                    */
  uint64_t scratch_bytes;
} gts_matmul_args;
int gts_matmul(const gts_matmul_args *a, void *hip_stream);
int gts_matmul_scratch(uint32_t m, uint32_t n, uint32_t k, uint64_t *bytes);

/* The elementwise part of its gradient: with d = dy gate act'(preact),
 *   dz = d, dgate = dy act(preact), dbias[j] = sum over i of d[i][j].
 * dz, dgate and dbias may each be NULL; preact may be NULL without an activation
 * and without dgate.  dz may be dy with the same stride.  The gradients of the operands
 * are products with dz. */
typedef struct gts_linear_grad_args {
  const void *dy, *preact, *gate;
  void *dz, *dgate, *dbias;
  int64_t dy_stride, preact_stride, gate_stride, dz_stride, dgate_stride;
  uint32_t m, n, dtype, activation;
  void *scratch;                  /* needs no initialisation                    */
  uint64_t scratch_bytes;
} gts_linear_grad_args;
int gts_linear_backward(const gts_linear_grad_args *a, void *hip_stream);
int gts_linear_backward_scratch(uint32_t m, uint32_t n, uint64_t *bytes);

/* ---- attention over whole prompts -------------------------------------------- */
#define GTS_PROMPT_CAUSAL 1u /* a token sees its sequence up to itself; else all of it */

/* The tokens of sequence b are starts[b] .. starts[b + 1) (starts = NULL: one
 * sequence of all tokens, batch 1).  Query head h reads key-value head
 * h / (q_heads / kv_heads).
 *   s_ij = scale q_i . k_j,  lse_i = log sum_j exp(s_ij),  out_i = sum_j exp(s_ij - lse_i) v_j.
 * A token outside every sequence has out = 0 and lse = -inf.  One whose scores are all
 * -inf is 0 / 0: NaN, lse = -inf.  lse may be NULL. */
typedef struct gts_prompt_args {
  const void *q, *k, *v;      /* [tokens][heads][dim]                           */
  void *out;
  float *lse;                 /* [tokens][q_heads] contiguous, or NULL          */
  const int32_t *starts;      /* [batch + 1] ascending, or NULL                 */
  int64_t q_stride[2], k_stride[2], v_stride[2], out_stride[2]; /* token, head  */
  uint32_t batch, tokens, q_heads, kv_heads, dim, dtype;
  float scale;
  uint32_t flags;
} gts_prompt_args;
int gts_prompt_attention(const gts_prompt_args *a, void *hip_stream);

/* Its gradient, from out and lse of the forward pass.  dk and dv are summed over
 * the query heads of a key-value head.  Tokens outside every sequence get zeros.  The
 * same bits on every run. */
typedef struct gts_prompt_grad_args {
  const void *dout, *q, *k, *v, *out;
  const float *lse;
  const int32_t *starts;
  void *dq, *dk, *dv;
  int64_t dout_stride[2], q_stride[2], k_stride[2], v_stride[2], out_stride[2], dq_stride[2], dk_stride[2],
      dv_stride[2];           /* token, head                                    */
  uint32_t batch, tokens, q_heads, kv_heads, dim, dtype;
  float scale;
  uint32_t flags;
  void *scratch;              /* needs no initialisation                        */
  uint64_t scratch_bytes;
} gts_prompt_grad_args;
int gts_prompt_attention_backward(const gts_prompt_grad_args *a, void *hip_stream);
int gts_prompt_attention_backward_scratch(uint32_t batch, uint32_t tokens, uint32_t q_heads, uint32_t kv_heads,
                                          uint32_t dim, uint64_t *bytes);

#ifdef __cplusplus
}
#endif
#endif /* GTS_OPS_H */
