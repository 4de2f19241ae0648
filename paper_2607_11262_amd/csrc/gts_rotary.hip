// gts_rotary.hip — rotary positions and the paged append.
//
// Both kernels move every value once: a unit is V pairs (a, b) of one head,
// 2 V values, loaded with one or two accesses, turned with V cosines and sines
// in 32 bits, rounded and stored.  Rows of the table are read from L1 after the
// first head of a token.  Neither has anything to wait for but memory, so
// they are bound by HBM when large and by the launch when small.
#include "gts_ops.h"

namespace gts {
namespace {

// One unit of a row: values [at(u, 0), +V) and [at(u, 1), +V).  Rotated pairs
// stand rot / 2 apart (half) or side by side (interleaved); the units behind
// the rotated part are copied.
template <typename T, int V, bool INTER>
__device__ __forceinline__ void unit_addresses(uint32_t u, uint32_t rot_units, uint32_t rot, uint32_t* p0, uint32_t* p1) {
  if (INTER || u >= rot_units) {
    *p0 = u * 2 * V;
    *p1 = u * 2 * V + V;
  } else {
    *p0 = u * V;
    *p1 = rot / 2 + u * V;
  }
}

template <typename T, int V, bool INTER>
__device__ __forceinline__ void rotate_unit(Pack<T, V>& x0, Pack<T, V>& x1, const float* cs, uint32_t u, uint32_t rot,
                                            float sign) {
  constexpr int W = V < 4 ? V : 4;
  float c[V], s[V];
#pragma unroll
  for (int i = 0; i < V; i += W) {
    const Pack<float, W> pc = *reinterpret_cast<const Pack<float, W>*>(cs + u * V + i);
    const Pack<float, W> ps = *reinterpret_cast<const Pack<float, W>*>(cs + rot / 2 + u * V + i);
#pragma unroll
    for (int j = 0; j < W; ++j) {
      c[i + j] = pc.v[j];
      s[i + j] = sign * ps.v[j];
    }
  }
  T* x[2] = {x0.v, x1.v};
#pragma unroll
  for (int i = 0; i < V; ++i) {
    T& ra = INTER ? x[2 * i / V][2 * i % V] : x0.v[i];
    T& rb = INTER ? x[(2 * i + 1) / V][(2 * i + 1) % V] : x1.v[i];
    const float a = (float)ra, b = (float)rb;
    ra = (T)(a * c[i] - b * s[i]);
    rb = (T)(b * c[i] + a * s[i]);
  }
}

// Position outside the table: its rotated values are NaN.
template <typename T, int V>
__device__ __forceinline__ void spoil(Pack<T, V>& x0, Pack<T, V>& x1) {
#pragma unroll
  for (int i = 0; i < V; ++i) x0.v[i] = x1.v[i] = (T)__builtin_nanf("");
}

struct RotaryParams {
  gts_rotary_args a;
  FastDiv per_token, per_head, tokens;  // units of a token, of a head; tokens of a batch entry
  uint32_t token_block;                 // tokens of a workgroup
  uint32_t n_tokens;
};

template <typename T, int V, bool INTER>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryParams p) {
  const gts_rotary_args& a = p.a;
  const uint32_t t0 = blockIdx.x * p.token_block;
  const uint32_t nt = p.n_tokens - t0 < p.token_block ? p.n_tokens - t0 : p.token_block;
  const uint32_t units = nt * p.per_token.d;
  const uint32_t rot_units = a.rot_dim / (2 * V);
  const float sign = a.flags & GTS_ROTARY_BACKWARD ? -1.f : 1.f;
  for (uint32_t i = threadIdx.x; i < units; i += 256) {
    const uint32_t tl = p.per_token.div(i), r = i - tl * p.per_token.d;
    const uint32_t h = p.per_head.div(r), u = r - h * p.per_head.d;
    const uint32_t t = t0 + tl;
    const uint32_t b = p.tokens.div(t), s = t - b * a.tokens;
    const T* x = (const T*)a.x + (int64_t)b * a.x_stride[0] + (int64_t)s * a.x_stride[1] + (int64_t)h * a.x_stride[2];
    T* o = (T*)a.out + (int64_t)b * a.out_stride[0] + (int64_t)s * a.out_stride[1] + (int64_t)h * a.out_stride[2];
    uint32_t p0, p1;
    unit_addresses<T, V, INTER>(u, rot_units, a.rot_dim, &p0, &p1);
    Pack<T, V> x0 = *reinterpret_cast<const Pack<T, V>*>(x + p0);
    Pack<T, V> x1 = *reinterpret_cast<const Pack<T, V>*>(x + p1);
    if (u < rot_units) {
      const int64_t at = (int64_t)b * a.pos_stride[0] + (int64_t)s * a.pos_stride[1];
      const int64_t pos = a.pos_bytes == 8 ? ((const int64_t*)a.positions)[at] : (int64_t)((const int32_t*)a.positions)[at];
      if (pos >= 0 && pos < (int64_t)a.n_positions)
        rotate_unit<T, V, INTER>(x0, x1, a.table + pos * a.table_stride, u, a.rot_dim, sign);
      else
        spoil<T, V>(x0, x1);
    }
    *reinterpret_cast<Pack<T, V>*>(o + p0) = x0;
    *reinterpret_cast<Pack<T, V>*>(o + p1) = x1;
  }
}

struct AppendParams {
  gts_append_args a;
  FastDiv per_token, per_head;
  uint32_t token_block, page_shift;
};

constexpr uint32_t kAppendTokens = 16;  // most tokens of a workgroup

template <typename T, int V, bool INTER>
__global__ __launch_bounds__(256) void append_kernel(AppendParams p) {
  const gts_append_args& a = p.a;
  __shared__ int64_t s_pos[kAppendTokens];   // position; -1: the token is in no sequence
  __shared__ int64_t s_page[kAppendTokens];  // page; -1: none
  __shared__ uint32_t s_slot[kAppendTokens];
  const uint32_t t0 = blockIdx.x * p.token_block;
  const uint32_t nt = a.batch.tokens - t0 < p.token_block ? a.batch.tokens - t0 : p.token_block;
  for (uint32_t i = threadIdx.x >> 6; i < nt; i += 4) {
    uint32_t seq, index, count;
    int64_t pos = -1, page = -1;
    uint32_t slot = 0;
    if (find_sequence(a.batch, t0 + i, &seq, &index, &count)) {
      const int64_t j = (int64_t)a.batch.lens[seq] - count + index;
      if (j >= 0) {
        pos = (int64_t)a.batch.prefix_len + j;
        const uint64_t at = (uint64_t)j >> p.page_shift;
        slot = (uint32_t)j & (a.cache.page - 1);
        if (at < a.batch.max_pages) {
          page = a.batch.page_table[(int64_t)seq * a.batch.table_stride + (int64_t)at];
          if (page >= (int64_t)a.cache.n_pages) page = -1;
        }
      }
    }
    if ((threadIdx.x & 63u) == 0) {
      s_pos[i] = pos;
      s_page[i] = page;
      s_slot[i] = slot;
    }
  }
  __syncthreads();
  const uint32_t units = nt * p.per_token.d;
  const uint32_t rot_units = a.table ? a.rot_dim / (2 * V) : 0;
  const uint32_t hkv = a.cache.heads;
  for (uint32_t i = threadIdx.x; i < units; i += 256) {
    const uint32_t tl = p.per_token.div(i), r = i - tl * p.per_token.d;
    uint32_t h = p.per_head.div(r);
    const uint32_t u = r - h * p.per_head.d;
    const uint32_t t = t0 + tl;
    const int64_t pos = s_pos[tl], page = s_page[tl];
    const T* x;
    T* o;
    bool rotated = u < rot_units;
    if (h < 2 * hkv) {
      if (page < 0) continue;
      const bool isv = h >= hkv;
      h -= isv ? hkv : 0;
      const int64_t* xs = isv ? a.v_stride : a.k_stride;
      const int64_t* os = isv ? a.cache.v_stride : a.cache.k_stride;
      x = (const T*)(isv ? a.v : a.k) + (int64_t)t * xs[0] + (int64_t)h * xs[1];
      o = (T*)(isv ? a.cache.v : a.cache.k) + page * os[0] + (int64_t)s_slot[tl] * os[1] + (int64_t)h * os[2];
      rotated = rotated && !isv;
    } else {
      if (pos < 0) continue;
      h -= 2 * hkv;
      x = (const T*)a.q + (int64_t)t * a.q_stride[0] + (int64_t)h * a.q_stride[1];
      o = (T*)a.q_out + (int64_t)t * a.q_out_stride[0] + (int64_t)h * a.q_out_stride[1];
    }
    uint32_t p0, p1;
    unit_addresses<T, V, INTER>(u, rot_units, a.rot_dim, &p0, &p1);
    if (!rotated) {  // a value row, or behind the rotated part: a plain copy
      p0 = u * 2 * V;
      p1 = p0 + V;
    }
    Pack<T, V> x0 = *reinterpret_cast<const Pack<T, V>*>(x + p0);
    Pack<T, V> x1 = *reinterpret_cast<const Pack<T, V>*>(x + p1);
    if (rotated) {
      if (pos < (int64_t)a.n_positions)
        rotate_unit<T, V, INTER>(x0, x1, a.table + pos * a.table_stride, u, a.rot_dim, 1.f);
      else
        spoil<T, V>(x0, x1);
    }
    *reinterpret_cast<Pack<T, V>*>(o + p0) = x0;
    *reinterpret_cast<Pack<T, V>*>(o + p1) = x1;
  }
}

// One thread a table entry pair; cos and sin in 64 bits.
__global__ __launch_bounds__(256) void table_kernel(float* table, uint32_t n_positions, uint32_t half, TableFreqs f,
                                                    double scale) {
  const uint64_t n = (uint64_t)n_positions * half;
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) {
    const uint64_t p = i / half;
    const uint32_t j = (uint32_t)(i - p * half);
    double s, c;
    sincos((double)p * f.f[j], &s, &c);
    table[p * 2 * half + j] = (float)(scale * c);
    table[p * 2 * half + half + j] = (float)(scale * s);
  }
}

// ---- which V: the widest access that every row, stride and part allows ------
// (16 bytes of 16-bit values at best; measured beside the kernels' rule below)
struct Width {
  uint32_t e;       // bytes of an element
  uint64_t bits;    // or of everything that must divide by V elements
  uint64_t bytes;   // or of everything that must divide by V * e bytes
  uint64_t pairs;   // or of everything that must divide by 2 V elements
  uint64_t table;   // or of everything in the table that must divide by 4 floats (or by V < 4)
  uint64_t table_bytes;
  bool fits(uint32_t v) const {
    const uint32_t w = v < 4 ? v : 4;
    return bits % v == 0 && bytes % (v * e) == 0 && pairs % (2 * v) == 0 && table % w == 0 && table_bytes % (4 * w) == 0;
  }
  uint32_t widest() const {
    for (uint32_t v = e == 4 ? 4 : 8; v > 1; v /= 2)
      if (fits(v)) return v;
    return 1;
  }
};

template <typename T, int V, template <typename, int, bool> class K, typename P>
void launch_v(uint32_t flags, uint32_t blocks, const P& p, hipStream_t s) {
  if (flags & GTS_ROTARY_INTERLEAVED)
    K<T, V, true>::go(blocks, p, s);
  else
    K<T, V, false>::go(blocks, p, s);
}

template <typename T, template <typename, int, bool> class K, typename P>
void launch_t(uint32_t v, uint32_t flags, uint32_t blocks, const P& p, hipStream_t s) {
  if (sizeof(T) == 2 && v == 8)
    launch_v<T, sizeof(T) == 2 ? 8 : 4, K>(flags, blocks, p, s);
  else if (v == 4)
    launch_v<T, 4, K>(flags, blocks, p, s);
  else if (v == 2)
    launch_v<T, 2, K>(flags, blocks, p, s);
  else
    launch_v<T, 1, K>(flags, blocks, p, s);
}

template <template <typename, int, bool> class K, typename P>
hipError_t launch_dtype(uint32_t dtype, uint32_t v, uint32_t flags, uint32_t blocks, const P& p, hipStream_t s) {
  if (dtype == GTS_F32)
    launch_t<float, K>(v, flags, blocks, p, s);
  else if (dtype == GTS_BF16)
    launch_t<__bf16, K>(v, flags, blocks, p, s);
  else
    launch_t<_Float16, K>(v, flags, blocks, p, s);
  return hipGetLastError();
}

template <typename T, int V, bool INTER>
struct RotaryKernel {
  static void go(uint32_t blocks, const RotaryParams& p, hipStream_t s) {
    rotary_kernel<T, V, INTER><<<dim3(blocks), dim3(256), 0, s>>>(p);
  }
};
template <typename T, int V, bool INTER>
struct AppendKernel {
  static void go(uint32_t blocks, const AppendParams& p, hipStream_t s) {
    append_kernel<T, V, INTER><<<dim3(blocks), dim3(256), 0, s>>>(p);
  }
};

// Tokens of a workgroup: one pass of its 256 threads while that leaves fewer
// than four workgroups a CU, up to four passes (the table's row is read once
// a token and workgroup) for larger calls.
uint32_t tokens_per_block(uint64_t tokens, uint32_t units_per_token) {
  const uint64_t passes = tokens * units_per_token / (256ull * 1024ull);
  const uint64_t want = 256ull * (passes < 1 ? 1 : passes > 4 ? 4 : passes);
  const uint64_t n = want / units_per_token;
  return n < 1 ? 1 : (uint32_t)n;
}

uint64_t or_strides(const int64_t* s, int n) {
  uint64_t r = 0;
  for (int i = 0; i < n; ++i) r |= (uint64_t)(s[i] < 0 ? -s[i] : s[i]);
  return r;
}

}  // namespace

hipError_t launch_rotary(const gts_rotary_args& a, hipStream_t stream) {
  const bool inter = a.flags & GTS_ROTARY_INTERLEAVED;
  Width w{};
  w.e = a.dtype == GTS_F32 ? 4 : 2;
  w.bits = or_strides(a.x_stride, 3) | or_strides(a.out_stride, 3) | (inter ? 0 : a.rot_dim / 2);
  w.bytes = (uint64_t)(uintptr_t)a.x | (uint64_t)(uintptr_t)a.out;
  w.pairs = a.rot_dim | (a.dim - a.rot_dim);
  w.table = (uint64_t)a.table_stride | (a.rot_dim / 2);
  w.table_bytes = (uint64_t)(uintptr_t)a.table;
  const uint32_t v = w.widest();
  RotaryParams p{};
  p.a = a;
  const uint32_t per_head = a.dim / (2 * v);
  p.per_head = FastDiv(per_head);
  p.per_token = FastDiv(per_head * a.heads);
  p.tokens = FastDiv(a.tokens);
  p.n_tokens = a.batch * a.tokens;
  p.token_block = tokens_per_block(p.n_tokens, per_head * a.heads);
  const uint32_t blocks = (p.n_tokens + p.token_block - 1) / p.token_block;
  return launch_dtype<RotaryKernel>(a.dtype, v, a.flags, blocks, p, stream);
}

hipError_t launch_append(const gts_append_args& a, hipStream_t stream) {
  const bool inter = a.flags & GTS_ROTARY_INTERLEAVED;
  const uint32_t rot = a.table ? a.rot_dim : 0;
  Width w{};
  w.e = a.cache.dtype == GTS_F32 ? 4 : 2;
  w.bits = or_strides(a.k_stride, 2) | or_strides(a.v_stride, 2) | or_strides(a.cache.k_stride, 3) |
           or_strides(a.cache.v_stride, 3) | (inter ? 0 : rot / 2);
  w.bytes = (uint64_t)(uintptr_t)a.k | (uint64_t)(uintptr_t)a.v | (uint64_t)(uintptr_t)a.cache.k |
            (uint64_t)(uintptr_t)a.cache.v;
  if (a.q) {
    w.bits |= or_strides(a.q_stride, 2) | or_strides(a.q_out_stride, 2);
    w.bytes |= (uint64_t)(uintptr_t)a.q | (uint64_t)(uintptr_t)a.q_out;
  }
  w.pairs = rot | (a.cache.dim - rot);
  w.table = a.table ? (uint64_t)a.table_stride | (rot / 2) : 0;
  w.table_bytes = (uint64_t)(uintptr_t)a.table;
  const uint32_t v = w.widest();
  AppendParams p{};
  p.a = a;
  if (!a.table) p.a.rot_dim = 0;
  const uint32_t per_head = a.cache.dim / (2 * v);
  const uint32_t per_token = per_head * (2 * a.cache.heads + (a.q ? a.q_heads : 0));
  p.per_head = FastDiv(per_head);
  p.per_token = FastDiv(per_token);
  p.page_shift = (uint32_t)__builtin_ctz(a.cache.page);
  p.token_block = tokens_per_block(a.batch.tokens, per_token);
  if (p.token_block > kAppendTokens) p.token_block = kAppendTokens;
  const uint32_t blocks = (a.batch.tokens + p.token_block - 1) / p.token_block;
  return launch_dtype<AppendKernel>(a.cache.dtype, v, a.flags, blocks, p, stream);
}

hipError_t launch_rotary_table(float* table, uint32_t n_positions, uint32_t rot_dim, const TableFreqs& f, double scale,
                               hipStream_t stream) {
  const uint64_t n = (uint64_t)n_positions * (rot_dim / 2);
  const uint64_t blocks = (n + 255) / 256;
  table_kernel<<<dim3((uint32_t)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, stream>>>(table, n_positions,
                                                                                         rot_dim / 2, f, scale);
  return hipGetLastError();
}

}  // namespace gts
