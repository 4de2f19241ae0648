// gts_rotary.hip — rotary positions and the paged append.
//
// Both kernels move every value once: a unit is V pairs (a, b) of one head,
// 2 V values, loaded with one or two accesses, turned with V cosines and sines
// in 32 bits, rounded and stored.  Rows of the table are read from L1 after the
// first head of a token.  Neither has anything to wait for but memory, so
// they are bound by HBM when large and by the launch when small.  A workgroup
// takes 256 or 512 units in a row, wherever a token ends; a thread one of them, or
// with 2^19 units and more two, both loaded before either is turned.  The
// gradient of 8 x 4096 tokens of 32 heads of 128 (550 MB): 103 us with one, 94
// (5.9 TB/s) with two, 96 with four; one decode step of 64 tokens: 2.1, 2.7, 4.1.
#include "gts_ops.h"

namespace gts {
namespace {

// One unit of a row: 2 V values in N accesses of W.  Rotated pairs stand rot / 2
// apart (half: two accesses) or side by side (interleaved: one); the units
// behind the rotated part are copied.
template <typename T, int V, bool INTER>
struct Unit {
  static constexpr int N = INTER ? 1 : 2, W = INTER ? 2 * V : V;
  Pack<T, W> x[N];
  // Where access i of unit u begins in its row.
  static __device__ __forceinline__ uint32_t at(int i, uint32_t u, bool rotated, uint32_t rot) {
    return INTER ? u * 2 * V : rotated ? i * (rot / 2) + u * V : u * 2 * V + i * V;
  }
  // cs: the row of the table.
  __device__ __forceinline__ void rotate(const float* cs, uint32_t u, uint32_t rot, float sign) {
    constexpr int F = V < 4 ? V : 4;
    float c[V], s[V];
#pragma unroll
    for (int i = 0; i < V; i += F) {
      const Pack<float, F> pc = *reinterpret_cast<const Pack<float, F>*>(cs + u * V + i);
      const Pack<float, F> ps = *reinterpret_cast<const Pack<float, F>*>(cs + rot / 2 + u * V + i);
#pragma unroll
      for (int j = 0; j < F; ++j) {
        c[i + j] = pc.v[j];
        s[i + j] = sign * ps.v[j];
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      T& ra = INTER ? x[0].v[2 * i] : x[0].v[i];
      T& rb = INTER ? x[0].v[2 * i + 1] : x[N - 1].v[i];
      const float a = (float)ra, b = (float)rb;
      // one product rounded, the other not: said here, so that every variant of a
      // kernel gives the same bits
      ra = (T)__builtin_fmaf(a, c[i], -(b * s[i]));
      rb = (T)__builtin_fmaf(b, c[i], a * s[i]);
    }
  }
  // Position outside the table: its rotated values are NaN.
  __device__ __forceinline__ void spoil() {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < W; ++j) x[i].v[j] = (T)__builtin_nanf("");
  }
};

// The widest access, with the hint that the value is not needed again.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <bool ONCE, typename T, int V>
__device__ __forceinline__ Pack<T, V> load(const T* p) {
  if constexpr (ONCE && sizeof(Pack<T, V>) == 16)
    return __builtin_bit_cast(Pack<T, V>, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)));
  else
    return *reinterpret_cast<const Pack<T, V>*>(p);
}
template <bool ONCE, typename T, int V>
__device__ __forceinline__ void store(T* p, const Pack<T, V>& x) {
  if constexpr (ONCE && sizeof(Pack<T, V>) == 16)
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, x), reinterpret_cast<u32x4*>(p));
  else
    *reinterpret_cast<Pack<T, V>*>(p) = x;
}

// Units of a call: per token and head, and the token and unit of unit `first`.
struct Units {
  FastDiv per_token, per_head;
  uint64_t all;
  __device__ __forceinline__ void begin(uint64_t first, uint32_t* token, uint32_t* unit) const {
    *token = all < (1ull << 31) ? per_token.div((uint32_t)first) : (uint32_t)(first / per_token.d);
    *unit = (uint32_t)(first - (uint64_t)*token * per_token.d);
  }
};

struct RotaryParams {
  gts_rotary_args a;
  Units units;
  FastDiv tokens;  // tokens of a batch entry
};

template <typename T, int V, bool INTER, int R>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryParams p) {
  typedef Unit<T, V, INTER> U;
  const gts_rotary_args& a = p.a;
  const uint64_t first = block_number() * (256 * R);
  if (first >= p.units.all) return;
  const uint64_t left = p.units.all - first;
  uint32_t t0, i0;
  p.units.begin(first, &t0, &i0);
  U v[R];
  T* o[R] = {};  // NULL: nothing to write
  int64_t pos[R];
  uint32_t unit[R];
  bool rotated[R];
#pragma unroll
  for (int k = 0; k < R; ++k) {
    if (threadIdx.x + 256 * k >= left) break;
    const uint32_t i = i0 + threadIdx.x + 256 * k, tl = p.units.per_token.div(i), r = i - tl * p.units.per_token.d;
    const uint32_t h = p.units.per_head.div(r), u = r - h * p.units.per_head.d, t = t0 + tl;
    const uint32_t b = p.tokens.div(t), s = t - b * a.tokens;
    const T* x = (const T*)a.x + (int64_t)b * a.x_stride[0] + (int64_t)s * a.x_stride[1] + (int64_t)h * a.x_stride[2];
    o[k] = (T*)a.out + (int64_t)b * a.out_stride[0] + (int64_t)s * a.out_stride[1] + (int64_t)h * a.out_stride[2];
    unit[k] = u;
    rotated[k] = u < a.rot_dim / (2 * V);
#pragma unroll
    for (int y = 0; y < U::N; ++y) v[k].x[y] = load<false, T, U::W>(x + U::at(y, u, rotated[k], a.rot_dim));
    const int64_t at = (int64_t)b * a.pos_stride[0] + (int64_t)s * a.pos_stride[1];
    pos[k] = a.pos_bytes == 8 ? ((const int64_t*)a.positions)[at] : (int64_t)((const int32_t*)a.positions)[at];
  }
#pragma unroll
  for (int k = 0; k < R; ++k) {
    if (!o[k]) continue;
    if (rotated[k]) {
      if (pos[k] >= 0 && pos[k] < (int64_t)a.n_positions)
        v[k].rotate(a.table + pos[k] * a.table_stride, unit[k], a.rot_dim, a.flags & GTS_ROTARY_BACKWARD ? -1.f : 1.f);
      else
        v[k].spoil();
    }
    // without the hint 9.4 instead of 8.3 us for 43 MB, 106 instead of 103 for 550 MB
#pragma unroll
    for (int y = 0; y < U::N; ++y) store<true, T, U::W>(o[k] + U::at(y, unit[k], rotated[k], a.rot_dim), v[k].x[y]);
  }
}

struct AppendParams {
  gts_append_args a;
  Units units;
  uint32_t page_shift;
};

// BIG: calls from 64 MB on, which no cache holds, take two units a thread and load
// with the hint that the values are not needed again (the cache's lines are wanted
// soon, by the attention, and stored without it).
template <typename T, int V, bool INTER, bool BIG>
__global__ __launch_bounds__(256) void append_kernel(AppendParams p) {
  typedef Unit<T, V, INTER> U;
  constexpr int R = BIG ? 2 : 1;
  constexpr uint32_t kTokens = 128 * R + 2;  // most tokens that 256 R units touch (two units a token at least)
  const gts_append_args& a = p.a;
  __shared__ int64_t s_pos[kTokens];   // position; -1: the token is in no sequence
  __shared__ int32_t s_page[kTokens];  // page; -1: none
  __shared__ uint32_t s_slot[kTokens];
  const uint64_t first = block_number() * (256 * R);
  if (first >= p.units.all) return;
  const uint64_t left = p.units.all - first;
  uint32_t t0, i0;
  p.units.begin(first, &t0, &i0);
  const uint32_t nt = p.units.per_token.div(i0 + (left < 256 * R ? (uint32_t)left : 256 * R) - 1) + 1;
  for (uint32_t k = threadIdx.x >> 6; k < nt; k += 4) {
    uint32_t seq, index, count;
    int64_t pos = -1;
    int32_t page = -1;
    uint32_t slot = 0;
    if (find_sequence(a.batch, t0 + k, &seq, &index, &count)) {
      const int64_t j = (int64_t)a.batch.lens[seq] - count + index;
      if (j >= 0) {
        pos = (int64_t)a.batch.prefix_len + j;
        const uint64_t at = (uint64_t)j >> p.page_shift;
        slot = (uint32_t)j & (a.cache.page - 1);
        if (at < a.batch.max_pages) {
          page = a.batch.page_table[(int64_t)seq * a.batch.table_stride + (int64_t)at];
          if (page < 0 || (uint32_t)page >= a.cache.n_pages) page = -1;
        }
      }
    }
    if ((threadIdx.x & 63u) == 0) {
      s_pos[k] = pos;
      s_page[k] = page;
      s_slot[k] = slot;
    }
  }
  __syncthreads();
  const uint32_t rot_units = a.table ? a.rot_dim / (2 * V) : 0, hkv = a.cache.heads;
  U v[R];
  T* o[R] = {};  // NULL: nothing to write
  int64_t pos[R];
  uint32_t unit[R];
  bool rotated[R];
#pragma unroll
  for (int k = 0; k < R; ++k) {
    if (threadIdx.x + 256 * k >= left) break;
    const uint32_t i = i0 + threadIdx.x + 256 * k, tl = p.units.per_token.div(i), r = i - tl * p.units.per_token.d;
    const uint32_t head = p.units.per_head.div(r), u = r - head * p.units.per_head.d, t = t0 + tl;
    const int64_t page = s_page[tl];
    pos[k] = s_pos[tl];
    unit[k] = u;
    rotated[k] = u < rot_units && (head < hkv || head >= 2 * hkv);
    const T* x;
    if (head < 2 * hkv) {
      if (page < 0) continue;
      const bool isv = head >= hkv;
      const uint32_t h = head - (isv ? hkv : 0);
      const int64_t* xs = isv ? a.v_stride : a.k_stride;
      const int64_t* os = isv ? a.cache.v_stride : a.cache.k_stride;
      x = (const T*)(isv ? a.v : a.k) + (int64_t)t * xs[0] + (int64_t)h * xs[1];
      o[k] = (T*)(isv ? a.cache.v : a.cache.k) + page * os[0] + (int64_t)s_slot[tl] * os[1] + (int64_t)h * os[2];
    } else {
      if (pos[k] < 0 && !(a.flags & GTS_APPEND_ZERO_REST)) continue;
      const uint32_t h = head - 2 * hkv;
      x = (const T*)a.q + (int64_t)t * a.q_stride[0] + (int64_t)h * a.q_stride[1];
      o[k] = (T*)a.q_out + (int64_t)t * a.q_out_stride[0] + (int64_t)h * a.q_out_stride[1];
      if (pos[k] < 0) {
        rotated[k] = false;
        v[k] = U{};
        continue;
      }
    }
#pragma unroll
    for (int y = 0; y < U::N; ++y) v[k].x[y] = load<BIG, T, U::W>(x + U::at(y, u, rotated[k], a.rot_dim));
  }
#pragma unroll
  for (int k = 0; k < R; ++k) {
    if (!o[k]) continue;
    if (rotated[k]) {
      if (pos[k] < (int64_t)a.n_positions)
        v[k].rotate(a.table + pos[k] * a.table_stride, unit[k], a.rot_dim, 1.f);
      else
        v[k].spoil();
    }
#pragma unroll
    for (int y = 0; y < U::N; ++y) store<false, T, U::W>(o[k] + U::at(y, unit[k], rotated[k], a.rot_dim), v[k].x[y]);
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
// 16 bytes at best (8 x 4 x 128 x 64 of 16-bit values unaligned, so V = 1: 6 times
// the time of V = 8).
struct Width {
  uint32_t e;            // bytes of an element
  uint32_t w;            // values of an access for V = 1: 2 interleaved, else 1
  uint64_t strides = 0;  // or of everything that must be a multiple of V w elements
  uint64_t bytes = 0;    // or of everything that must be a multiple of V w e bytes
  uint64_t pairs = 0;    // or of everything that must be a multiple of 2 V elements
  uint64_t table = 0;    // or of everything in the table that must be a multiple of 4 floats (or of V < 4)
  uint64_t table_bytes = 0;
  bool fits(uint32_t v) const {
    const uint32_t f = v < 4 ? v : 4;
    return strides % (v * w) == 0 && bytes % (v * w * e) == 0 && pairs % (2 * v) == 0 && table % f == 0 &&
           table_bytes % (4 * f) == 0;
  }
  uint32_t widest() const {
    for (uint32_t v = 16 / (e * w); v > 1; v /= 2)
      if (fits(v)) return v;
    return 1;
  }
};

template <typename T, int V, template <typename, int, bool> class K, typename P>
hipError_t launch_v(uint32_t flags, const P& p, hipStream_t s) {
  return flags & GTS_ROTARY_INTERLEAVED ? K<T, V, true>::go(p, s) : K<T, V, false>::go(p, s);
}

template <typename T, template <typename, int, bool> class K, typename P>
hipError_t launch_t(uint32_t v, uint32_t flags, const P& p, hipStream_t s) {
  constexpr bool wide = sizeof(T) == 4;
  if (v == 8) return K<T, wide ? 4 : 8, false>::go(p, s);  // 16-bit, half
  if (v == 4 && wide) return K<T, 4, false>::go(p, s);
  if (v == 4) return launch_v<T, wide ? 2 : 4, K>(flags, p, s);
  if (v == 2) return launch_v<T, 2, K>(flags, p, s);
  return launch_v<T, 1, K>(flags, p, s);
}

template <template <typename, int, bool> class K, typename P>
hipError_t launch_dtype(uint32_t dtype, uint32_t v, uint32_t flags, const P& p, hipStream_t s) {
  if (dtype == GTS_F32) return launch_t<float, K>(v, flags, p, s);
  if (dtype == GTS_BF16) return launch_t<__bf16, K>(v, flags, p, s);
  return launch_t<_Float16, K>(v, flags, p, s);
}

// 0: more workgroups than a launch can have.
uint64_t blocks_of(const Units& u, int r) {
  const uint64_t n = (u.all + 256 * r - 1) / (256 * r);
  return n <= kMostBlocks ? n : 0;
}

template <typename T, int V, bool INTER>
struct RotaryKernel {
  static hipError_t go(const RotaryParams& p, hipStream_t s) {
    const bool two = p.units.all >= (1u << 19);
    const uint64_t blocks = blocks_of(p.units, two ? 2 : 1);
    if (!blocks) return hipErrorInvalidValue;
    if (two)
      rotary_kernel<T, V, INTER, 2><<<grid_of(blocks), dim3(256), 0, s>>>(p);
    else
      rotary_kernel<T, V, INTER, 1><<<grid_of(blocks), dim3(256), 0, s>>>(p);
    return hipGetLastError();
  }
};
template <typename T, int V, bool INTER>
struct AppendKernel {
  static hipError_t go(const AppendParams& p, hipStream_t s) {
    const bool big = p.units.all * (2 * V * sizeof(T)) >= (64ull << 20);
    const uint64_t blocks = blocks_of(p.units, big ? 2 : 1);
    if (!blocks) return hipErrorInvalidValue;
    if (big)
      append_kernel<T, V, INTER, true><<<grid_of(blocks), dim3(256), 0, s>>>(p);
    else
      append_kernel<T, V, INTER, false><<<grid_of(blocks), dim3(256), 0, s>>>(p);
    return hipGetLastError();
  }
};

Units units_of(uint64_t tokens, uint32_t per_head, uint32_t heads) {
  Units u;
  u.per_head = FastDiv(per_head);
  u.per_token = FastDiv(per_head * heads);
  u.all = tokens * per_head * heads;
  return u;
}
uint64_t or_strides(const int64_t* s, int n) {
  uint64_t r = 0;
  for (int i = 0; i < n; ++i) r |= (uint64_t)(s[i] < 0 ? -s[i] : s[i]);
  return r;
}

}  // namespace

hipError_t launch_rotary(const gts_rotary_args& a, hipStream_t stream) {
  const bool inter = a.flags & GTS_ROTARY_INTERLEAVED;
  Width w{a.dtype == GTS_F32 ? 4u : 2u, inter ? 2u : 1u};
  w.strides = or_strides(a.x_stride, 3) | or_strides(a.out_stride, 3) | (inter ? 0 : a.rot_dim / 2);
  w.bytes = (uint64_t)(uintptr_t)a.x | (uint64_t)(uintptr_t)a.out;
  w.pairs = a.rot_dim | (a.dim - a.rot_dim);
  w.table = (uint64_t)a.table_stride | (a.rot_dim / 2);
  w.table_bytes = (uint64_t)(uintptr_t)a.table;
  const uint32_t v = w.widest();
  RotaryParams p{};
  p.a = a;
  p.units = units_of((uint64_t)a.batch * a.tokens, a.dim / (2 * v), a.heads);
  p.tokens = FastDiv(a.tokens);
  return launch_dtype<RotaryKernel>(a.dtype, v, a.flags, p, stream);
}

hipError_t launch_append(const gts_append_args& a, hipStream_t stream) {
  const bool inter = a.flags & GTS_ROTARY_INTERLEAVED;
  const uint32_t rot = a.table ? a.rot_dim : 0;
  Width w{a.cache.dtype == GTS_F32 ? 4u : 2u, inter ? 2u : 1u};
  w.strides = or_strides(a.k_stride, 2) | or_strides(a.v_stride, 2) | or_strides(a.cache.k_stride, 3) |
           or_strides(a.cache.v_stride, 3) | (inter ? 0 : rot / 2);
  w.bytes = (uint64_t)(uintptr_t)a.k | (uint64_t)(uintptr_t)a.v | (uint64_t)(uintptr_t)a.cache.k |
            (uint64_t)(uintptr_t)a.cache.v;
  if (a.q) {
    w.strides |= or_strides(a.q_stride, 2) | or_strides(a.q_out_stride, 2);
    w.bytes |= (uint64_t)(uintptr_t)a.q | (uint64_t)(uintptr_t)a.q_out;
  }
  w.pairs = rot | (a.cache.dim - rot);
  w.table = a.table ? (uint64_t)a.table_stride | (rot / 2) : 0;
  w.table_bytes = (uint64_t)(uintptr_t)a.table;
  const uint32_t v = w.widest();
  AppendParams p{};
  p.a = a;
  if (!a.table) p.a.rot_dim = 0;
  p.units = units_of(a.batch.tokens, a.cache.dim / (2 * v), 2 * a.cache.heads + (a.q ? a.q_heads : 0));
  p.page_shift = (uint32_t)__builtin_ctz(a.cache.page);
  return launch_dtype<AppendKernel>(a.cache.dtype, v, a.flags, p, stream);
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
