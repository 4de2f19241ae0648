// gts_attention.hip — attention of new tokens over a paged cache and the
// prefix that all sequences share.
//
// The row kernel: one wavefront per (token, query head) walks the row's keys 64
// at a time, one key a lane, with the running maximum and sum of the softmax;
// the weighted values are summed with a lane per group of dims.  Takes every
// type, head dim, stride and alignment.
#include "gts_ops.h"

namespace gts {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// What the kernels need beside the arguments.
struct AttnParams {
  gts_attention_args a;
  uint32_t page_shift;
  uint32_t group;  // query heads of a key-value head
};

// Element offset of own or prefix key j in the cache (before the head), -1
// when no page holds it.
__device__ __forceinline__ int64_t key_page(const gts_attention_args& a, const int32_t* pages, uint32_t n, uint32_t shift,
                                            uint32_t j) {
  const uint32_t at = j >> shift;
  if (at >= n) return -1;
  const int32_t p = pages[at];
  return p >= 0 && (uint32_t)p < a.cache.n_pages ? p : -1;
}

template <typename T>
__global__ __launch_bounds__(256) void row_kernel(AttnParams p) {
  const gts_attention_args& a = p.a;
  __shared__ float s_q[4][GTS_OPS_MAX_ATTN];
  const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63u;
  const uint64_t row = (uint64_t)blockIdx.x * 4 + wave;
  if (row >= (uint64_t)a.batch.tokens * a.q_heads) return;
  const uint32_t t = (uint32_t)(row / a.q_heads), hq = (uint32_t)(row % a.q_heads), h = hq / p.group;
  const uint32_t D = a.cache.dim;
  uint32_t seq = 0, index = 0, count = 0;
  const bool has = find_sequence(a.batch, t, &seq, &index, &count);
  int64_t own = has ? (int64_t)a.batch.lens[seq] - count + index + 1 : 0;
  if (own < 0) own = 0;
  const uint32_t n_prefix = has ? a.batch.prefix_len : 0;
  const T* q = (const T*)a.q + (int64_t)t * a.q_stride[0] + (int64_t)hq * a.q_stride[1];
  for (uint32_t d = lane; d < D; d += 64) s_q[wave][d] = (float)q[d];
  float m = -INFINITY, l = 0.f, o[GTS_OPS_MAX_ATTN / 64] = {};
  const float scale = a.scale * kLog2e;
  for (int part = 0; part < 2; ++part) {
    const uint32_t n = part ? (uint32_t)own : n_prefix;
    const int32_t* pages = part ? a.batch.page_table + (int64_t)seq * a.batch.table_stride : a.prefix_pages;
    const uint32_t n_pages = part ? a.batch.max_pages : a.n_prefix_pages;
    for (uint32_t j0 = 0; j0 < n; j0 += 64) {
      const uint32_t j = j0 + lane;
      const int64_t page = j < n ? key_page(a, pages, n_pages, p.page_shift, j) : -1;
      const uint32_t slot = j & (a.cache.page - 1);
      float s = -INFINITY;
      if (page >= 0) {
        const T* k = (const T*)a.cache.k + page * a.cache.k_stride[0] + (int64_t)slot * a.cache.k_stride[1] +
                     (int64_t)h * a.cache.k_stride[2];
        float acc = 0.f;
        for (uint32_t d = 0; d < D; ++d) acc += s_q[wave][d] * (float)k[d];
        s = acc * scale;
      }
      float mx = s;
      for (int i = 32; i; i >>= 1) mx = fmaxf(mx, __shfl_xor(mx, i));
      const float m1 = fmaxf(m, mx);
      const float base = m1 == -INFINITY ? 0.f : m1;
      const float w = page >= 0 ? exp2f(s - base) : 0.f;
      const float alpha = exp2f(m - base);
      l = l * alpha + w;
      for (uint32_t i = 0; i * 64 < D; ++i) o[i] *= alpha;
      m = m1;
      const uint64_t there = __ballot(page >= 0);
      for (uint64_t todo = there; todo; todo &= todo - 1) {
        const int src = __builtin_ctzll(todo);
        const float wj = __shfl(w, src);
        const int64_t pj = __shfl((int)page, src);
        const T* v = (const T*)a.cache.v + pj * a.cache.v_stride[0] +
                     (int64_t)((j0 + src) & (a.cache.page - 1)) * a.cache.v_stride[1] + (int64_t)h * a.cache.v_stride[2];
#pragma unroll
        for (uint32_t i = 0; i < GTS_OPS_MAX_ATTN / 64; ++i) {
          const uint32_t d = i * 64 + lane;
          if (d < D) o[i] += wj * (float)v[d];
        }
      }
    }
  }
  for (int i = 32; i; i >>= 1) l += __shfl_xor(l, i);
  const float inv = l == 0.f ? 0.f : 1.f / l;  // no key: zeros
  T* out = (T*)a.out + (int64_t)t * a.out_stride[0] + (int64_t)hq * a.out_stride[1];
#pragma unroll
  for (uint32_t i = 0; i < GTS_OPS_MAX_ATTN / 64; ++i) {
    const uint32_t d = i * 64 + lane;
    if (d < D) out[d] = (T)(o[i] * inv);
  }
  if (a.lse && lane == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

}  // namespace

uint64_t attention_scratch(uint32_t, uint32_t, uint32_t, uint32_t, uint32_t) { return 0; }

hipError_t launch_attention(const gts_attention_args& a, hipStream_t stream) {
  AttnParams p{};
  p.a = a;
  p.page_shift = (uint32_t)__builtin_ctz(a.cache.page);
  p.group = a.q_heads / a.cache.heads;
  const uint64_t rows = (uint64_t)a.batch.tokens * a.q_heads;
  const dim3 grid((uint32_t)((rows + 3) / 4)), block(256);
  if (a.cache.dtype == GTS_F32)
    row_kernel<float><<<grid, block, 0, stream>>>(p);
  else if (a.cache.dtype == GTS_BF16)
    row_kernel<__bf16><<<grid, block, 0, stream>>>(p);
  else
    row_kernel<_Float16><<<grid, block, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace gts
