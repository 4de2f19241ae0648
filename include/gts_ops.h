/*
 * gts_ops.h — C ABI of the serving-step operators of libgts.so: rotary
 * positions, appending keys and values to a paged cache, and attention over
 * that cache for a batch that shares a prefix.
 *
 * They are the kernels of the step whose tile graphs the package simulates
 * (the rotation inside a decoder layer, split-KV decode attention), run on the
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
 * lse, keeps them in 32 bits).
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

#ifdef __cplusplus
}
#endif
#endif /* GTS_OPS_H */
