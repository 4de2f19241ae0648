// gts_ops_host.cpp — argument checks and entry points of the operators
// (include/gts_ops.h).  Nothing here touches the device; the launch functions are
// those of gts_rotary.hip, gts_attention.hip, gts_norm.hip, gts_linear.hip and
// gts_prompt.hip.
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "gts_ops.h"

namespace gts {
int report(int code, const char* message);
void clear_error();
int report_hip(hipError_t e, const char* what);
}  // namespace gts

namespace {

constexpr uint32_t kMaxCount = 0x7FFFFFFFu;  // tokens and sequences: the kernels' 32-bit indices
constexpr uint32_t kMaxHeads = 65535u;

int refuse(int code, const char* fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return gts::report(code, buf);
}

int check_type(uint32_t dtype) {
  return dtype <= GTS_F16 ? GTS_OK : refuse(GTS_E_ARG, "unknown element type %u", dtype);
}

int check_rotation(uint32_t rot_dim, uint32_t dim, uint32_t n_positions, uint32_t flags, uint32_t known) {
  if (flags & ~known) return refuse(GTS_E_ARG, "unknown flag bits 0x%x", flags & ~known);
  if (rot_dim == 0 || rot_dim % 2 || rot_dim > dim)
    return refuse(GTS_E_RANGE, "rotated part of %u values in a head of %u: it must be even, at least 2 and inside", rot_dim,
                  dim);
  if (n_positions == 0 || n_positions > kMaxCount) return refuse(GTS_E_RANGE, "table of %u positions", n_positions);
  return GTS_OK;
}

int check_dim(uint32_t dim) {
  if (dim == 0 || dim % 2 || dim > GTS_OPS_MAX_DIM)
    return refuse(GTS_E_RANGE, "head dim %u: it must be even and at most %u", dim, GTS_OPS_MAX_DIM);
  return GTS_OK;
}

int check_cache(const gts_kv_cache& c) {
  if (int rc = check_type(c.dtype)) return rc;
  if (c.reserved) return refuse(GTS_E_ARG, "reserved word of the cache is not zero");
  if (c.heads == 0 || c.heads > kMaxHeads) return refuse(GTS_E_RANGE, "%u key-value heads", c.heads);
  if (c.page == 0 || c.page > GTS_OPS_MAX_PAGE || (c.page & (c.page - 1)))
    return refuse(GTS_E_RANGE, "pages of %u tokens: a power of two up to %u", c.page, GTS_OPS_MAX_PAGE);
  if (c.n_pages > kMaxCount) return refuse(GTS_E_RANGE, "%u pages", c.n_pages);
  if (c.n_pages && (!c.k || !c.v)) return refuse(GTS_E_ARG, "the cache is NULL");
  return GTS_OK;
}

int check_batch(const gts_kv_batch& b) {
  if (b.batch == 0 || b.batch > kMaxCount || b.tokens > kMaxCount)
    return refuse(GTS_E_RANGE, "%u sequences with %u new tokens", b.batch, b.tokens);
  if (b.prefix_len > kMaxCount) return refuse(GTS_E_RANGE, "prefix of %u keys", b.prefix_len);
  if (!b.lens) return refuse(GTS_E_ARG, "lens is NULL");
  if (b.max_pages && !b.page_table) return refuse(GTS_E_ARG, "page_table is NULL");
  if (!b.starts && b.tokens % b.batch)
    return refuse(GTS_E_ARG, "%u new tokens are not the same number for each of %u sequences: pass starts", b.tokens,
                  b.batch);
  return GTS_OK;
}

}  // namespace

extern "C" {

int gts_rotary_table(float* table, uint32_t n_positions, uint32_t rot_dim, const double* freq, double scale,
                     void* hip_stream) {
  gts::clear_error();
  if (!table || !freq) return refuse(GTS_E_ARG, "table or freq is NULL");
  if (int rc = check_dim(rot_dim)) return rc;
  if (int rc = check_rotation(rot_dim, rot_dim, n_positions, 0, 0)) return rc;
  if (!std::isfinite(scale)) return refuse(GTS_E_ARG, "scale is not finite");
  gts::TableFreqs f{};
  for (uint32_t i = 0; i < rot_dim / 2; ++i) {
    if (!std::isfinite(freq[i])) return refuse(GTS_E_ARG, "freq[%u] is not finite", i);
    f.f[i] = freq[i];
  }
  const hipError_t e = gts::launch_rotary_table(table, n_positions, rot_dim, f, scale, (hipStream_t)hip_stream);
  return e == hipSuccess ? GTS_OK : gts::report_hip(e, "launch of the rotary table");
}

int gts_rotary(const gts_rotary_args* a, void* hip_stream) {
  gts::clear_error();
  if (!a) return refuse(GTS_E_ARG, "args is NULL");
  if (int rc = check_type(a->dtype)) return rc;
  if (int rc = check_dim(a->dim)) return rc;
  if (int rc = check_rotation(a->rot_dim, a->dim, a->n_positions, a->flags,
                              GTS_ROTARY_INTERLEAVED | GTS_ROTARY_BACKWARD))
    return rc;
  if (a->reserved) return refuse(GTS_E_ARG, "reserved word is not zero");
  if (a->pos_bytes != 4 && a->pos_bytes != 8) return refuse(GTS_E_ARG, "positions of %u bytes", a->pos_bytes);
  if (a->heads > kMaxHeads || (uint64_t)a->batch * a->tokens > kMaxCount)
    return refuse(GTS_E_RANGE, "%u x %u tokens with %u heads", a->batch, a->tokens, a->heads);
  if (a->batch == 0 || a->tokens == 0 || a->heads == 0) return GTS_OK;
  if (!a->x || !a->out || !a->positions || !a->table) return refuse(GTS_E_ARG, "x, out, positions or table is NULL");
  const hipError_t e = gts::launch_rotary(*a, (hipStream_t)hip_stream);
  return e == hipSuccess ? GTS_OK : gts::report_hip(e, "launch of the rotation");
}

int gts_append_kv(const gts_append_args* a, void* hip_stream) {
  gts::clear_error();
  if (!a) return refuse(GTS_E_ARG, "args is NULL");
  if (int rc = check_cache(a->cache)) return rc;
  if (int rc = check_dim(a->cache.dim)) return rc;
  if (int rc = check_batch(a->batch)) return rc;
  constexpr uint32_t known = GTS_ROTARY_INTERLEAVED | GTS_APPEND_ZERO_REST;
  if (a->flags & ~known) return refuse(GTS_E_ARG, "unknown flag bits 0x%x", a->flags & ~known);
  if (a->table)
    if (int rc = check_rotation(a->rot_dim, a->cache.dim, a->n_positions, a->flags, known)) return rc;
  if (a->q && (a->q_heads == 0 || a->q_heads > kMaxHeads)) return refuse(GTS_E_RANGE, "%u query heads", a->q_heads);
  if (a->batch.tokens == 0) return GTS_OK;
  if (!a->k || !a->v) return refuse(GTS_E_ARG, "k or v is NULL");
  if (a->q && !a->q_out) return refuse(GTS_E_ARG, "q_out is NULL");
  const hipError_t e = gts::launch_append(*a, (hipStream_t)hip_stream);
  return e == hipSuccess ? GTS_OK : gts::report_hip(e, "launch of the append");
}

static int check_attention_sizes(uint32_t batch, uint32_t tokens, uint32_t q_heads, uint32_t kv_heads, uint32_t dim) {
  if (dim == 0 || dim > GTS_OPS_MAX_ATTN) return refuse(GTS_E_RANGE, "head dim %u: at most %u", dim, GTS_OPS_MAX_ATTN);
  if (kv_heads == 0 || q_heads == 0 || q_heads > kMaxHeads || q_heads % kv_heads)
    return refuse(GTS_E_RANGE, "%u query heads over %u key-value heads", q_heads, kv_heads);
  if (batch == 0 || batch > kMaxCount || (uint64_t)tokens * q_heads > kMaxCount)
    return refuse(GTS_E_RANGE, "%u sequences, %u tokens of %u heads", batch, tokens, q_heads);
  return GTS_OK;
}

int gts_shared_prefix_attention_scratch(uint32_t batch, uint32_t tokens, uint32_t q_heads, uint32_t kv_heads,
                                        uint32_t dim, uint64_t* bytes) {
  gts::clear_error();
  if (!bytes) return refuse(GTS_E_ARG, "bytes is NULL");
  if (int rc = check_attention_sizes(batch, tokens, q_heads, kv_heads, dim)) return rc;
  *bytes = gts::attention_scratch(batch, tokens, q_heads, kv_heads, dim);
  return GTS_OK;
}

int gts_shared_prefix_attention(const gts_attention_args* a, void* hip_stream) {
  gts::clear_error();
  if (!a) return refuse(GTS_E_ARG, "args is NULL");
  if (int rc = check_cache(a->cache)) return rc;
  if (int rc = check_batch(a->batch)) return rc;
  if (int rc = check_attention_sizes(a->batch.batch, a->batch.tokens, a->q_heads, a->cache.heads, a->cache.dim))
    return rc;
  if (a->reserved) return refuse(GTS_E_ARG, "reserved word is not zero");
  if (!std::isfinite(a->scale)) return refuse(GTS_E_ARG, "scale is not finite");
  if (a->batch.prefix_len && !a->prefix_pages) return refuse(GTS_E_ARG, "prefix_pages is NULL");
  if ((uint64_t)a->n_prefix_pages * a->cache.page < a->batch.prefix_len)
    return refuse(GTS_E_RANGE, "%u prefix pages of %u tokens do not hold %u keys", a->n_prefix_pages, a->cache.page,
                  a->batch.prefix_len);
  if (a->batch.tokens == 0) return GTS_OK;
  if (!a->q || !a->out) return refuse(GTS_E_ARG, "q or out is NULL");
  const uint64_t need =
      gts::attention_scratch(a->batch.batch, a->batch.tokens, a->q_heads, a->cache.heads, a->cache.dim);
  if (a->scratch_bytes < need || (need && !a->scratch))
    return refuse(GTS_E_SCRATCH, "scratch needs %llu bytes, got %llu", (unsigned long long)need,
                  (unsigned long long)a->scratch_bytes);
  const hipError_t e = gts::launch_attention(*a, (hipStream_t)hip_stream);
  return e == hipSuccess ? GTS_OK : gts::report_hip(e, "launch of the attention");
}

static int check_scratch(uint64_t need, const void* scratch, uint64_t bytes) {
  if (bytes < need || (need && !scratch))
    return refuse(GTS_E_SCRATCH, "scratch needs %llu bytes, got %llu", (unsigned long long)need,
                  (unsigned long long)(scratch ? bytes : 0));
  return (uintptr_t)scratch % 16 ? refuse(GTS_E_ARG, "scratch is not aligned to 16 bytes") : GTS_OK;
}

// ---- layer norm ------------------------------------------------------------------

static int check_rows(uint32_t rows, uint32_t dim) {
  if (dim == 0 || dim > GTS_OPS_MAX_WIDTH || rows > kMaxCount) return refuse(GTS_E_RANGE, "%u rows of %u values", rows, dim);
  return GTS_OK;
}

int gts_layer_norm(const gts_norm_args* a, void* hip_stream) {
  gts::clear_error();
  if (!a) return refuse(GTS_E_ARG, "args is NULL");
  if (int rc = check_type(a->dtype)) return rc;
  if (int rc = check_rows(a->rows, a->dim)) return rc;
  if (a->flags & ~GTS_NORM_CENTER) return refuse(GTS_E_ARG, "unknown flag bits 0x%x", a->flags & ~GTS_NORM_CENTER);
  if (a->reserved) return refuse(GTS_E_ARG, "reserved word is not zero");
  if (!std::isfinite(a->eps) || a->eps < 0) return refuse(GTS_E_ARG, "eps is not a finite number from 0 on");
  if (a->rows == 0) return GTS_OK;
  if (!a->x || !a->out) return refuse(GTS_E_ARG, "x or out is NULL");
  const hipError_t e = gts::launch_norm(*a, (hipStream_t)hip_stream);
  return e == hipSuccess ? GTS_OK : gts::report_hip(e, "launch of the norm");
}

int gts_layer_norm_backward_scratch(uint32_t rows, uint32_t dim, uint64_t* bytes) {
  gts::clear_error();
  if (!bytes) return refuse(GTS_E_ARG, "bytes is NULL");
  if (int rc = check_rows(rows, dim)) return rc;
  *bytes = gts::norm_grad_scratch(rows, dim);
  return GTS_OK;
}

int gts_layer_norm_backward(const gts_norm_grad_args* a, void* hip_stream) {
  gts::clear_error();
  if (!a) return refuse(GTS_E_ARG, "args is NULL");
  if (int rc = check_type(a->dtype)) return rc;
  if (int rc = check_rows(a->rows, a->dim)) return rc;
  if (a->flags & ~GTS_NORM_CENTER) return refuse(GTS_E_ARG, "unknown flag bits 0x%x", a->flags & ~GTS_NORM_CENTER);
  if (a->rows && (!a->dy || !a->x || !a->rstd || ((a->flags & GTS_NORM_CENTER) && !a->mean)))
    return refuse(GTS_E_ARG, "dy, x, rstd or mean is NULL");
  if (int rc = check_scratch(a->dweight || a->dbias ? gts::norm_grad_scratch(a->rows, a->dim) : 0, a->scratch,
                             a->scratch_bytes))
    return rc;
  if (!a->dweight && !a->dbias && (!a->dx || a->rows == 0)) return GTS_OK;
  const hipError_t e = gts::launch_norm_grad(*a, (hipStream_t)hip_stream);
  return e == hipSuccess ? GTS_OK : gts::report_hip(e, "launch of the norm's gradient");
}

// ---- matrix product ----------------------------------------------------------------

static int check_activation(uint32_t act) {
  return act <= GTS_ACT_SILU ? GTS_OK : refuse(GTS_E_ARG, "unknown activation %u", act);
}
static int check_product(uint32_t m, uint32_t n, uint32_t k) {
  if (m > kMaxCount || k > kMaxCount || n > GTS_OPS_MAX_WIDTH) return refuse(GTS_E_RANGE, "product of %u x %u x %u", m, n, k);
  // tiles of a launch: where smaller ones or splits of the sum would be too many, these are taken
  if ((((uint64_t)m + 127) / 128) * (((uint64_t)n + 127) / 128) > gts::kMostGroups)
    return refuse(GTS_E_RANGE, "a result of %u x %u is too large", m, n);
  return GTS_OK;
}

int gts_matmul_scratch(uint32_t m, uint32_t n, uint32_t k, uint64_t* bytes) {
  gts::clear_error();
  if (!bytes) return refuse(GTS_E_ARG, "bytes is NULL");
  if (int rc = check_product(m, n, k)) return rc;
  *bytes = gts::matmul_scratch(m, n, k);
  return GTS_OK;
}

int gts_matmul(const gts_matmul_args* a, void* hip_stream) {
  gts::clear_error();
  if (!a) return refuse(GTS_E_ARG, "args is NULL");
  if (int rc = check_type(a->dtype)) return rc;
  if (int rc = check_activation(a->activation)) return rc;
  constexpr uint32_t known = GTS_MATMUL_A_COLUMNS | GTS_MATMUL_B_COLUMNS;
  if (a->flags & ~known) return refuse(GTS_E_ARG, "unknown flag bits 0x%x", a->flags & ~known);
  if (int rc = check_product(a->m, a->n, a->k)) return rc;
  if (a->m == 0 || a->n == 0) return GTS_OK;
  if (!a->out || (a->k && (!a->a || !a->b))) return refuse(GTS_E_ARG, "a, b or out is NULL");
  if (int rc = check_scratch(gts::matmul_scratch(a->m, a->n, a->k), a->scratch, a->scratch_bytes)) return rc;
  const hipError_t e = gts::launch_matmul(*a, (hipStream_t)hip_stream);
  return e == hipSuccess ? GTS_OK : gts::report_hip(e, "launch of the product");
}

int gts_linear_backward_scratch(uint32_t m, uint32_t n, uint64_t* bytes) {
  gts::clear_error();
  if (!bytes) return refuse(GTS_E_ARG, "bytes is NULL");
  if (int rc = check_product(m, n, 0)) return rc;
  *bytes = gts::linear_grad_scratch(m, n);
  return GTS_OK;
}

int gts_linear_backward(const gts_linear_grad_args* a, void* hip_stream) {
  gts::clear_error();
  if (!a) return refuse(GTS_E_ARG, "args is NULL");
  if (int rc = check_type(a->dtype)) return rc;
  if (int rc = check_activation(a->activation)) return rc;
  if (int rc = check_product(a->m, a->n, 0)) return rc;
  if (a->n == 0 || (a->m == 0 && !a->dbias) || (!a->dz && !a->dgate && !a->dbias)) return GTS_OK;
  if (a->m && !a->dy) return refuse(GTS_E_ARG, "dy is NULL");
  if (a->m && !a->preact && (a->activation != GTS_ACT_NONE || a->dgate)) return refuse(GTS_E_ARG, "preact is NULL");
  if (int rc = check_scratch(a->dbias ? gts::linear_grad_scratch(a->m, a->n) : 0, a->scratch, a->scratch_bytes)) return rc;
  const hipError_t e = gts::launch_linear_grad(*a, (hipStream_t)hip_stream);
  return e == hipSuccess ? GTS_OK : gts::report_hip(e, "launch of the product's gradient");
}

// ---- attention over prompts -----------------------------------------------------------

static int check_prompt(uint32_t batch, uint32_t tokens, uint32_t q_heads, uint32_t kv_heads, uint32_t dim) {
  if (int rc = check_attention_sizes(batch, tokens, q_heads, kv_heads, dim)) return rc;
  if (tokens > kMaxCount || gts::prompt_groups(batch, tokens, q_heads) > gts::kMostGroups)
    return refuse(GTS_E_RANGE, "%u sequences with %u tokens of %u heads", batch, tokens, q_heads);
  return GTS_OK;
}
}  // extern "C"

template <typename A>
static int check_prompt_args(const A& a) {
  if (int rc = check_type(a.dtype)) return rc;
  if (int rc = check_prompt(a.batch, a.tokens, a.q_heads, a.kv_heads, a.dim)) return rc;
  if (a.flags & ~GTS_PROMPT_CAUSAL) return refuse(GTS_E_ARG, "unknown flag bits 0x%x", a.flags & ~GTS_PROMPT_CAUSAL);
  if (!std::isfinite(a.scale)) return refuse(GTS_E_ARG, "scale is not finite");
  if (!a.starts && a.batch != 1) return refuse(GTS_E_ARG, "starts is NULL for %u sequences", a.batch);
  return GTS_OK;
}

extern "C" {

int gts_prompt_attention(const gts_prompt_args* a, void* hip_stream) {
  gts::clear_error();
  if (!a) return refuse(GTS_E_ARG, "args is NULL");
  if (int rc = check_prompt_args(*a)) return rc;
  if (a->tokens == 0) return GTS_OK;
  if (!a->q || !a->k || !a->v || !a->out) return refuse(GTS_E_ARG, "q, k, v or out is NULL");
  const hipError_t e = gts::launch_prompt(*a, (hipStream_t)hip_stream);
  return e == hipSuccess ? GTS_OK : gts::report_hip(e, "launch of the attention over prompts");
}

int gts_prompt_attention_backward_scratch(uint32_t batch, uint32_t tokens, uint32_t q_heads, uint32_t kv_heads,
                                          uint32_t dim, uint64_t* bytes) {
  gts::clear_error();
  if (!bytes) return refuse(GTS_E_ARG, "bytes is NULL");
  if (int rc = check_prompt(batch, tokens, q_heads, kv_heads, dim)) return rc;
  *bytes = gts::prompt_grad_scratch(batch, tokens, q_heads, kv_heads, dim);
  return GTS_OK;
}

int gts_prompt_attention_backward(const gts_prompt_grad_args* a, void* hip_stream) {
  gts::clear_error();
  if (!a) return refuse(GTS_E_ARG, "args is NULL");
  if (int rc = check_prompt_args(*a)) return rc;
  if (a->tokens == 0) return GTS_OK;
  if (!a->dout || !a->q || !a->k || !a->v || !a->out || !a->lse || !a->dq || !a->dk || !a->dv)
    return refuse(GTS_E_ARG, "dout, q, k, v, out, lse, dq, dk or dv is NULL");
  const uint64_t need = gts::prompt_grad_scratch(a->batch, a->tokens, a->q_heads, a->kv_heads, a->dim);
  if (int rc = check_scratch(need, a->scratch, a->scratch_bytes)) return rc;
  const hipError_t e = gts::launch_prompt_grad(*a, (hipStream_t)hip_stream);
  return e == hipSuccess ? GTS_OK : gts::report_hip(e, "launch of the prompts' gradient");
}

}  // extern "C"
