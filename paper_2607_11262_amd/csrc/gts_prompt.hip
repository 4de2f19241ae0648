// gts_prompt.hip — attention over whole prompts packed one behind the other, and its
// gradient.
//
//   forward   s_ij = scale q_i . k_j over the keys of i's sequence (up to its own: causal),
//             lse_i = log sum_j exp(s_ij),  out_i = sum_j exp(s_ij - lse_i) v_j
//   backward  p_ij = exp(s_ij - lse_i),  delta_i = dout_i . out_i,  dp_ij = dout_i . v_j,
//             ds_ij = p_ij (dp_ij - delta_i),
//             dv_j = sum_i p_ij dout_i,  dk_j = scale sum_i ds_ij q_i,  dq_i = scale sum_j ds_ij k_j
//
// Scores are computed so that a lane has one row (forward and dq: keys x rows) or one key
// (dk, dv: rows x keys): what leaves the first product is an operand of the second as it
// stands.  The gradient takes two kernels, one by rows for dq and one by keys for dk and
// dv, which compute scores again (seven products instead of five; eight in the tile kernels): sums stay in registers,
// without atomics, the same bits on every run; the query heads that share a key-value head
// are summed there too.
//
// Bound by matrix and vector issue (the exponentials, conversions and maxima of a tile take about as
// long as its products): 8 x 4096 tokens of 32 heads of 128 in bfloat16 2423 us forward (908 TFLOP/s;
// a large library product reached 1369 on the same card), 8 causal texts of 512 to 8192 tokens, 32 / 8 heads,
// 2211 us backward (483 TFLOP/s of the five products).
#include "gts_ops.h"
#include "gts_tile.h"

namespace gts {
namespace {

// ---- which rows a workgroup takes -------------------------------------------------------
// The tokens before the first sequence, the sequences, and the tokens behind the last are
// batch + 2 spans.  Span e has the places floor(first(e) / tile) + e on: as many as its
// tiles or one more, because ceil(n / tile) is at most floor(end / tile) - floor(first / tile) + 1.
// So a place's span is found without a plan of the lengths.
struct Span {
  uint32_t first, n;  // of the span
  uint32_t tile;      // its tile
  bool in;            // a sequence
};
__device__ __forceinline__ uint32_t bound_of(const int32_t* starts, uint32_t batch, uint32_t tokens, uint32_t e) {
  if (e == 0) return 0;
  if (e == batch + 2) return tokens;
  if (!starts) return e == 1 ? 0 : tokens;
  const int32_t s = starts[e - 1];
  return s < 0 ? 0 : (uint32_t)s < tokens ? (uint32_t)s : tokens;
}
__host__ __device__ inline uint32_t places_of(uint32_t batch, uint32_t tokens, uint32_t tile) {
  return tokens / tile + batch + 2;
}
// All 64 lanes with the same place; false: nothing is there.
__device__ __forceinline__ bool find_span(const int32_t* starts, uint32_t batch, uint32_t tokens, uint32_t tile,
                                          uint32_t place, Span* s) {
  const uint32_t lane = threadIdx.x & 63u;
  uint32_t lo = 0, n = batch + 2;  // the span is one of lo .. lo + n - 1
  while (n > 1) {
    const uint32_t step = (n + 63u) / 64u, e = lane * step;
    const bool le = e < n && (lane == 0 || bound_of(starts, batch, tokens, lo + e) / tile + lo + e <= place);
    const uint32_t last = 63u - (uint32_t)__builtin_clzll(__ballot(le));
    lo += last * step;
    n = n - last * step < step ? n - last * step : step;
  }
  const uint32_t b0 = uni(bound_of(starts, batch, tokens, lo)), b1 = uni(bound_of(starts, batch, tokens, lo + 1));
  s->first = b0;
  s->n = b1 > b0 ? b1 - b0 : 0;
  s->tile = place - (b0 / tile + lo);
  s->in = lo > 0 && lo <= batch;
  return (uint64_t)s->tile * tile < s->n;
}

// ---- the general kernels ----------------------------------------------------------------
// Any type, head, stride and alignment.  128 rows (or keys) a workgroup, 32 a wave, which
// holds their operands in registers; 32 keys (or rows) at a time go through registers to
// LDS.  In 32 bits the matrix rate is a sixteenth; what is left is bound by the way to LDS and its
// barriers (one causal prompt, 32 bits: 4096 tokens, 16 / 4 heads of 64 541 us forward, 2872 backward;
// 3807 with all query heads of a key-value head in one workgroup).
constexpr uint32_t kRows = 128, kStep = 32;
constexpr uint32_t kKeys = 64;  // keys of a workgroup of dkv_tile_kernel

template <typename T, int DP>
struct Held {  // 32 rows of a wave
  Vec8<T> x[DP / 16];
  __device__ __forceinline__ void load(const T* p, bool valid, uint32_t dim, uint32_t half) {
#pragma unroll
    for (int i = 0; i < DP / 16; ++i)
      x[i] = load8(p + i * 16 + 8 * half, valid ? (int64_t)dim - (i * 16 + 8 * half) : 0);
  }
};
template <typename T, int DP>
constexpr uint32_t kRowPitch = DP + 8;

// Rows j0 .. j0 + 31 of n to LDS, zeros where there is none.  Returns whether a value was
// not finite; with `clear`, those are zeros in LDS.
template <typename T, int DP>
__device__ __forceinline__ bool stage_rows(const T* p, int64_t stride, uint32_t j0, uint32_t n, uint32_t dim, bool clear,
                                           T* s) {
  bool found = false;
#pragma unroll 4
  for (uint32_t id = threadIdx.x; id < kStep * (DP / 8); id += 256) {
    const uint32_t r = id / (DP / 8), c = id % (DP / 8) * 8;
    Vec8<T> x = load8(p + (int64_t)(j0 + r) * stride + c, j0 + r < n ? (int64_t)dim - c : 0);
    if (clear) found |= clear_not_finite(x);
    write8(s + r * kRowPitch<T, DP> + c, x);
  }
  return found;
}
// Clears them in LDS afterwards (where the product before wanted them).
template <typename T, int DP>
__device__ __forceinline__ void clear_rows(T* s) {
  for (uint32_t id = threadIdx.x; id < kStep * (DP / 8); id += 256) {
    T* at = s + id / (DP / 8) * kRowPitch<T, DP> + id % (DP / 8) * 8;
    Vec8<T> x = read8(at);
    if (clear_not_finite(x)) write8(at, x);
  }
}

// sum += rows of LDS x held rows: a 32 x 32 product over the head.
template <typename T, int DP>
__device__ __forceinline__ f32x16 times_held(const T* s, const Held<T, DP>& h, uint32_t lane) {
  f32x16 r;
#pragma unroll
  for (int i = 0; i < 16; ++i) r[i] = 0.f;
#pragma unroll
  for (int i = 0; i < DP / 16; ++i) r = mfma(frag_rows(s, kRowPitch<T, DP>, 0, i * 16, lane), h.x[i], r);
  return r;
}
// o (dims x the lane's row or key) += turned rows of LDS x weights w of 32 rows, rounded to T.
template <typename T, int DP>
__device__ __forceinline__ void add_weighted(f32x16* o, const T* s, const f32x16& w, uint32_t lane) {
  Vec8<T> u[2];
#pragma unroll
  for (int i = 0; i < 16; ++i) u[i / 8][i % 8] = (T)w[i];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int k = 0; k < 2; ++k) o[d] = mfma(frag_columns<true>(s, kRowPitch<T, DP>, k * 16, d * 32, lane), u[k], o[d]);
}
template <int N>
__device__ __forceinline__ void clear(f32x16 (&o)[N]) {
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
}
// Values that are not finite in a block whose rows some lanes do not see to its end: 0
// times one of them would reach lanes that must not see it.  They are cleared in the copy
// that is multiplied, and added here, from memory, where `sees(j)`: themselves, or NaN, as
// which they reach a gradient's sum whatever their weight.
// N blocks of 32 columns from `column` on.
template <typename T, int N, typename F>
__device__ __forceinline__ void add_odd(f32x16* o, const T* p, int64_t stride, uint32_t j0, uint32_t n, uint32_t column,
                                        uint32_t dim, uint32_t half, bool as_nan, F sees) {
#pragma unroll 1
  for (uint32_t j = j0; j < n && j < j0 + kStep; ++j) {
    const T* row = p + (int64_t)j * stride;
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t c = column + d * 32 + frag_row(i, half);
        if (c >= dim) continue;
        const float x = (float)row[c];
        if (not_finite(x) && sees(j)) o[d][i] += as_nan ? __builtin_nanf("") : x;
      }
  }
}
// The lane's row of a result.
template <typename T, int DP>
__device__ __forceinline__ void write_row(T* out, const f32x16* o, float f, uint32_t dim, uint32_t half) {
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t c = d * 32 + frag_row(i, half);
      if (c < dim) out[c] = (T)(o[d][i] * f);
    }
}

struct PromptParams {
  gts_prompt_args a;
  uint32_t group;
  uint32_t places;
  bool vec;  // rows of q, k and v are aligned to 16 bytes: loads of that
};

template <typename T, int DP>
__global__ __launch_bounds__(256) void prompt_kernel(PromptParams p) {
  const gts_prompt_args& a = p.a;
  __shared__ __align__(16) T s_k[kStep * kRowPitch<T, DP>], s_v[kStep * kRowPitch<T, DP>];
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, half = lane / 32;
  const uint32_t hq = blockIdx.x % a.q_heads, h = hq / p.group;
  Span sp;
  if (!find_span(a.starts, a.batch, a.tokens, kRows, blockIdx.x / a.q_heads, &sp)) return;
  const uint32_t r0 = sp.tile * kRows, row = r0 + wave * 32 + lane % 32, token = sp.first + row;
  const bool valid = row < sp.n, causal = a.flags & GTS_PROMPT_CAUSAL;
  T* out = (T*)a.out + (int64_t)token * a.out_stride[0] + (int64_t)hq * a.out_stride[1];
  f32x16 o[DP / 32];
  clear(o);
  if (!sp.in) {
    if (valid) {
      write_row<T, DP>(out, o, 0.f, a.dim, half);
      if (a.lse && half == 0) a.lse[(uint64_t)token * a.q_heads + hq] = -INFINITY;
    }
    return;
  }
  Held<T, DP> q;
  q.load((const T*)a.q + (int64_t)token * a.q_stride[0] + (int64_t)hq * a.q_stride[1], valid, a.dim, half);
  const T* k = (const T*)a.k + (int64_t)sp.first * a.k_stride[0] + (int64_t)h * a.k_stride[1];
  const T* v = (const T*)a.v + (int64_t)sp.first * a.v_stride[0] + (int64_t)h * a.v_stride[1];
  const uint32_t keys = causal && r0 + kRows < sp.n ? r0 + kRows : sp.n;
  const uint32_t sees = causal ? row + 1 : sp.n;
  const float c = a.scale * kLog2e;
  float m = -INFINITY, l = 0.f;
  for (uint32_t j0 = 0; j0 < keys; j0 += kStep) {
    const bool edge = causal && j0 + kStep > r0 + 1;  // some row does not see all of the block
    __syncthreads();
    stage_rows<T, DP>(k, a.k_stride[0], j0, sp.n, a.dim, false, s_k);
    const bool found = stage_rows<T, DP>(v, a.v_stride[0], j0, sp.n, a.dim, edge, s_v);
    const bool odd = __syncthreads_or(found);
    f32x16 s = times_held<T, DP>(s_k, q, lane);
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t j = j0 + frag_row(i, half);
      s[i] = j < sees && j < sp.n ? s[i] * c : -INFINITY;
      mx = fmaxf(mx, s[i]);
    }
    const float m1 = fmaxf(m, max_halves(mx));
    const float base = m1 == -INFINITY ? 0.f : m1, alpha = exp2_(m - base);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = exp2_(s[i] - base);
      sum += s[i];
    }
    l = l * alpha + add_halves(sum);
    m = m1;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) o[d] *= alpha;
    add_weighted<T, DP>(o, s_v, s, lane);
    if (odd) add_odd<T, DP / 32>(o, v, a.v_stride[0], j0, sp.n, 0, a.dim, half, false, [&](uint32_t j) { return j < sees; });
  }
  if (!valid) return;
  write_row<T, DP>(out, o, 1.f / l, a.dim, half);
  if (a.lse && half == 0) a.lse[(uint64_t)token * a.q_heads + hq] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// ---- the tile kernels ---------------------------------------------------------------------
// 16-bit values whose rows are aligned to 16 bytes, heads of whole 16 bytes.  As the general
// kernels (8 x 4096 tokens, 32 heads of 128: 6758 us there, 2305 here when both were timed), with tiles
// of 64 rows of two matrices (keys and values, or queries and dout) that
// go straight to LDS while the tile before is worked on: one barrier a tile.
constexpr uint32_t kTile = 64;

__device__ __align__(16) const uint32_t g_zeros[GTS_OPS_MAX_ATTN / 2] = {};  // a row that is not there

template <typename T, int DP>
struct Tiles {
  static constexpr int C = DP / 8;      // 16-byte chunks of a row
  static constexpr int RPI = 64 / C;    // rows of one load of a wave
  static constexpr int N = kTile * DP;  // values of a tile
  // Chunk c of row r stands at c ^ swizzle(r): reads of 16 rows at one chunk, and reads of 4
  // rows x 64 bytes that are turned on the way, each touch all 64 banks once.
  static __device__ __forceinline__ uint32_t swizzle(uint32_t r) {
    return C >= 16 ? ((r & 3) << 2) | ((r >> 2) & 3) : ((r & 2) << 1) | ((r >> 2) & 3);
  }
};

// Loads tiles of two matrices to LDS: each of W waves 64 / W rows of both.
template <typename T, int DP, int W = 4>
struct Loader {
  using L = Tiles<T, DP>;
  static constexpr uint32_t R = kTile / W;  // rows of a wave
  static constexpr int NL = R / L::RPI;     // its loads
  static_assert(NL * L::RPI == R, "whole loads");
  const T *a, *b;  // of the first row
  int64_t a_stride, b_stride;
  uint32_t n, dim;                      // rows that are there, values of a row
  // Bytes from a load's first row to this lane's, and from a row to the lane's chunk in the first load:
  // swizzle joins bits of a row's number, so that load i's chunk is that ^ swizzle of i's first row.  Three
  // registers; one for each load spills in the gradient (float16 heads of 256: 2965 us so, 2736 now).
  uint32_t a_row, b_row, chunk;

  __device__ __forceinline__ void start() {
    static_assert(R % 16 == 0, "no wave's first row has a bit that swizzle takes");
    const uint32_t lane = fresh_lane(), r0 = lane / L::C;
    a_row = 2 * r0 * (uint32_t)a_stride;
    b_row = 2 * r0 * (uint32_t)b_stride;
    chunk = 16 * (lane % L::C ^ L::swizzle(r0));
  }
  __device__ __forceinline__ void load(uint32_t j0, uint32_t wave, T* sa, T* sb) const {
    const uint32_t j = j0 + wave * R;
    const char* pa = (const char*)(a + (int64_t)j * a_stride);
    const char* pb = (const char*)(b + (int64_t)j * b_stride);
    uint32_t c0 = chunk;
    asm volatile("" : "+v"(c0));  // places are computed here, not kept across the loops around
    if (j + R <= n && dim == DP) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const uint32_t c = c0 ^ 16 * L::swizzle(i * L::RPI);
        load_to_lds(pa + i * (2 * L::RPI * a_stride), a_row + c, sa + (wave * R + i * L::RPI) * DP);
        load_to_lds(pb + i * (2 * L::RPI * b_stride), b_row + c, sb + (wave * R + i * L::RPI) * DP);
      }
      return;
    }
    const uint32_t r0 = fresh_lane() / L::C;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const uint32_t c = c0 ^ 16 * L::swizzle(i * L::RPI);
      const bool there = j + i * L::RPI + r0 < n && c < 2 * dim;
      load_to_lds(there ? pa + i * (2 * L::RPI * a_stride) + (a_row + c) : (const char*)g_zeros, sa + (wave * R + i * L::RPI) * DP);
      load_to_lds(there ? pb + i * (2 * L::RPI * b_stride) + (b_row + c) : (const char*)g_zeros, sb + (wave * R + i * L::RPI) * DP);
    }
  }
};
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Where a lane's parts of a tile's fragments stand, in bytes from the row that the fragment begins
// with (a whole number of 16): kept for all tiles, because computing them took a quarter of the vector
// instructions (8 x 4096 tokens, 32 heads of 128: 2673 us, 2465 so).
template <typename T, int DP>
struct Parts {
  uint32_t row[DP / 16], column[2][DP / 32];
  __device__ __forceinline__ void start(uint32_t lane) {
    using L = Tiles<T, DP>;
    const uint32_t c = lane / 32 ^ L::swizzle(lane % 32);
#pragma unroll
    for (int kk = 0; kk < DP / 16; ++kk) row[kk] = 2 * (lane % 32 * DP + (c ^ (2 * kk)) * 8);
    const uint32_t g = lane / 16, r = 4 * (g / 2) + lane % 16 / 4, cc = g % 2 * 2 + lane % 4 / 2;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
        column[x][d] = 2 * ((r + 8 * x) * DP + lane % 2 * 4 + ((cc ^ L::swizzle(r + 8 * x)) ^ (d * 4)) * 8);
  }
  // Rows at + lane % 32 of s, places 16 kk + 8 half ..
  __device__ __forceinline__ Vec8<T> rows(const T* s, uint32_t at, int kk) const {
    return *(const Vec8<T>*)((const char*)s + row[kk] + at * DP * 2);
  }
  // Columns 32 d + lane % 32, rows at + 4 half .. + 3 and 8 further.
  __device__ __forceinline__ Vec8<T> columns(const T* s, uint32_t at, int d) const {
    typedef __attribute__((address_space(3))) i16x4* lds_t;
    union {
      i16x4 h[2];
      Vec8<T> v;
    } u;
#pragma unroll
    for (int x = 0; x < 2; ++x)
      u.h[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)((const char*)s + column[x][d] + at * DP * 2));
    return u.v;
  }
};
// The same columns for a block d that is not known when this is compiled.
template <typename T, int DP>
__device__ __forceinline__ Vec8<T> column_frag(const T* s, uint32_t row, int d, uint32_t lane) {
  using L = Tiles<T, DP>;
  const uint32_t g = lane / 16, r = 4 * (g / 2) + lane % 16 / 4, c = g % 2 * 2 + lane % 4 / 2;  // row: whole 16s
  typedef __attribute__((address_space(3))) i16x4* lds_t;
  union {
    i16x4 h[2];
    Vec8<T> v;
  } u;
  const T* at = s + (row + r) * DP + lane % 2 * 4;
  u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(at + ((c ^ L::swizzle(r)) ^ (d * 4)) * 8));
  u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(at + 8 * DP + ((c ^ L::swizzle(r + 8)) ^ (d * 4)) * 8));
  return u.v;
}
template <typename T, int N>
__device__ __forceinline__ void clear_tile(T* s) {
  for (uint32_t x = threadIdx.x; x < N / 8; x += 256) *(u32x4*)(s + x * 8) = finite_only<T>(*(const u32x4*)(s + x * 8));
}
// The wave's 32 rows of a result (N blocks of 32 columns x rows, a lane its row) to memory, through
// LDS that the wave has for itself, so that whole rows are written.
template <typename T, int N>
__device__ __forceinline__ void write_rows(T* s, const f32x16* o, float f, T* out, int64_t stride, uint32_t rows,
                                           uint32_t column, uint32_t dim, uint32_t lane) {
  constexpr uint32_t P = N * 32 + 8;
  const uint32_t half = lane / 32;
  asm volatile("" ::: "memory");  // a wave's accesses to LDS keep their order
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      Pack<T, 4> x;
#pragma unroll
      for (int j = 0; j < 4; ++j) x.v[j] = (T)(o[d][i + j] * f);
      *(Pack<T, 4>*)(s + lane % 32 * P + d * 32 + frag_row(i, half)) = x;
    }
  asm volatile("" ::: "memory");
#pragma unroll
  for (uint32_t i = 0; i < N * 2; ++i) {
    const uint32_t id = i * 64 + lane, r = id / (N * 4), c = id % (N * 4) * 8;
    if (r < rows && column + c < dim) *(u32x4*)(out + (int64_t)r * stride + column + c) = *(const u32x4*)(s + r * P + c);
  }
}

// Position of a workgroup among the heads of a place: those of a key-value head, and as many
// key-value heads as divide 8, stand 8 / that many apart, so that they meet in the L2 of one XCD.
__device__ __forceinline__ uint32_t head_at(uint32_t at, uint32_t kv_heads, uint32_t group, uint32_t* kv) {
  const uint32_t s = kv_heads % 8 == 0 ? 8 : kv_heads % 4 == 0 ? 4 : kv_heads % 2 == 0 ? 2 : 1;
  *kv = at % s + at / (s * group) * s;
  return *kv * group + at / s % group;
}

// Which (place, head) pair a workgroup takes, the last places first: with a causal mask they see
// the most keys.  Of one sequence whose workgroups are all at work at once, two a CU, the second of
// a CU should be short if its first is long: the second 256 come in the other order.  Places without
// tokens are then the last.
__device__ __forceinline__ uint32_t place_at(uint32_t batch, uint32_t tokens, uint32_t places, uint32_t heads, bool causal,
                                             uint32_t* at) {
  uint32_t i = blockIdx.x;
  const uint32_t n = (tokens + kRows - 1) / kRows;
  if (batch == 1 && causal && n * heads <= 512 && i >= 256 && i < n * heads) i = 256 + n * heads - 1 - i;
  *at = i % heads;
  i /= heads;
  return batch > 1 ? places - 1 - i : i < n ? n - i : i == n ? 0 : i;
}

// What a wave of the forward kernel holds: 32 rows, and N blocks of 32 columns of their results.
template <typename T, int DP, int N>
struct Rows {
  Vec8<T> q[DP / 16];
  f32x16 o[N];
  Parts<T, DP> at;
  int d0;  // the first of the blocks; 0 where they are all
  float m, l;  // reference maximum of q.k (unscaled), sum of this half's weights

  // 32 NS keys from LDS row `key` on; the lane's row sees those before `sees` (from there).
  template <int NS>
  __device__ __forceinline__ void step(uint32_t lane, const T* sk, const T* sv, uint32_t key, float c, bool mask, int32_t sees) {
    f32x16 s[NS];
#pragma unroll
    for (int b = 0; b < NS; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
    // The fragments of two matrix steps are read while the two before are multiplied; the
    // fences keep that order.
    Vec8<T> kf[2][2][NS];
    const auto read = [&](int to, int kk) {
#pragma unroll
      for (int b = 0; b < NS; ++b)
#pragma unroll
        for (int x = 0; x < 2; ++x) kf[to][x][b] = at.rows(sk, key + b * 32, kk + x);
    };
    read(0, 0);
#pragma unroll
    for (int kk = 0; kk < DP / 16; kk += 2) {
      if (kk + 2 < DP / 16) read(kk / 2 + 1 & 1, kk + 2);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int b = 0; b < NS; ++b) s[b] = mfma(kf[kk / 2 & 1][x][b], q[kk + x], s[b]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (mask) {
#pragma unroll
      for (int b = 0; b < NS; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[b][i] = (int32_t)(b * 32 + frag_row(i, lane / 32)) < sees ? s[b][i] : -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int b = 0; b < NS; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[b][i]);
    mx = max_halves(mx);
    // The reference follows the maximum only when that is 2^8 ahead: weights up to 256 are as
    // exact, and sums and output are rescaled rarely.
    if (__any((mx - m) * c > 8.f || (m == -INFINITY && mx > m))) {
      const float m1 = fmaxf(m, mx);
      const float alpha = m == -INFINITY ? 0.f : exp2_((m - m1) * c);
      l *= alpha;
#pragma unroll
      for (int b = 0; b < N; ++b) o[b] *= alpha;
      m = m1;
    }
    const float base = m == -INFINITY ? 0.f : -m * c;
    // Weights are multiplied in the tensors' type, as the matrix instruction takes them,
    // and summed in 32 bits, which lse keeps.
    float sum[2] = {0.f, 0.f};
    Vec8<T> pw[2 * NS];
    const auto weigh = [&](int kb, int i) {
      const float e = exp2_(__builtin_fmaf(s[kb / 2][kb % 2 * 8 + i], c, base));
      sum[i & 1] += e;
      pw[kb][i] = (T)e;
    };
    // The weights of 16 keys are computed, and the values of 16 keys read, between the
    // products of the 16 keys before.
    Vec8<T> vf[2][N];
    const auto values = [&](uint32_t from, int d) {
      if constexpr (N == DP / 32)
        return at.columns(sv, from, d);
      else
        return column_frag<T, DP>(sv, from, d0 + d, lane);
    };
#pragma unroll
    for (int d = 0; d < N; ++d) vf[0][d] = values(key, d);
#pragma unroll
    for (int i = 0; i < 8; ++i) weigh(0, i);
#pragma unroll
    for (int kb = 0; kb < 2 * NS; ++kb) {
      if (kb + 1 < 2 * NS) {
#pragma unroll
        for (int d = 0; d < N; ++d) vf[kb + 1 & 1][d] = values(key + kb * 16 + 16, d);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int d = 0; d < N; ++d) {
        o[d] = mfma(vf[kb & 1][d], pw[kb], o[d]);
        if (kb + 1 < 2 * NS) {
#pragma unroll
          for (int i = d * 8 / N; i < (d + 1) * 8 / N; ++i) weigh(kb + 1, i);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    l += sum[0] + sum[1];
  }
};

// 128 rows, 32 a wave.  First without a look at values that are not finite; a workgroup that
// then finds one among its results computes them again with it (`odd`): 0 times one of them
// would reach rows that must not see it.  That takes 32 columns at a time (block d0), so that
// it does not need more registers than the usual way.
template <typename T, int DP, bool ODD>
__device__ __forceinline__ bool prompt_rows(const PromptParams& p, const Span& sp, uint32_t hq, uint32_t h, T* s_kv,
                                            int d0 = 0) {
  constexpr int N = ODD ? 1 : DP / 32;
  using L = Tiles<T, DP>;
  const gts_prompt_args& a = p.a;
  const uint32_t lane = fresh_lane(), wave = uni(threadIdx.x >> 6), half = lane / 32;
  const uint32_t r0 = sp.tile * kRows, w0 = r0 + wave * 32, row = w0 + lane % 32;
  const bool valid = row < sp.n, causal = a.flags & GTS_PROMPT_CAUSAL;
  const float c = a.scale == 0.f ? 1.f : __builtin_fabsf(a.scale) * kLog2e;
  Loader<T, DP> ld;
  ld.a = (const T*)a.k + (int64_t)sp.first * a.k_stride[0] + (int64_t)h * a.k_stride[1];
  ld.b = (const T*)a.v + (int64_t)sp.first * a.v_stride[0] + (int64_t)h * a.v_stride[1];
  ld.a_stride = a.k_stride[0];
  ld.b_stride = a.v_stride[0];
  ld.n = sp.n;
  ld.dim = a.dim;
  ld.start();
  const uint32_t keys = causal && r0 + kRows < sp.n ? r0 + kRows : sp.n, tiles = (keys + kTile - 1) / kTile;
  __syncthreads();
  ld.load(0, wave, s_kv, s_kv + L::N);
  Rows<T, DP, N> r;
  clear(r.o);
  r.d0 = d0;
  r.at.start(lane);
  r.m = -INFINITY;
  r.l = 0.f;
  {
    // scale's sign (and 0) go into the queries: the maximum of q.k is then that of the scores
    const T sign = (T)(a.scale == 0.f ? 0.f : a.scale < 0.f ? -1.f : 1.f);
    const T* q = (const T*)a.q + (int64_t)(sp.first + (valid ? row : 0)) * a.q_stride[0] + (int64_t)hq * a.q_stride[1];
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
      const uint32_t at = i * 16 + 8 * half;
      r.q[i] = *(const Vec8<T>*)(at < a.dim ? q + at : (const T*)g_zeros);
      if (a.scale <= 0.f) r.q[i] *= sign;
    }
  }
  for (uint32_t t = 0; t < tiles; ++t) {
    const uint32_t j0 = t * kTile;
    T *sk = s_kv + (t & 1) * 2 * L::N, *sv = sk + L::N;
    wait_loads();
    __syncthreads();
    if (t + 1 < tiles) {
      T* next = s_kv + ((t + 1) & 1) * 2 * L::N;
      ld.load(j0 + kTile, wave, next, next + L::N);
    }
    const uint32_t seen = causal && row + 1 < sp.n ? row + 1 : sp.n;  // keys of the lane's row
    bool odd = false;
    if constexpr (ODD) {
      if (causal && j0 + kTile > r0 + 1) {
        bool found = false;
        for (uint32_t x = threadIdx.x; x < L::N / 8; x += 256) found |= any_not_finite<T>(*(const u32x4*)(sv + x * 8));
        odd = __syncthreads_or(found);
        if (odd) {
          clear_tile<T, L::N>(sv);
          __syncthreads();
        }
      }
    }
    // some row of the wave does not see all of the tile; it sees none of it
    const uint32_t low = causal ? w0 + 1 : sp.n;
    if (causal && j0 > w0 + 31) continue;
    const bool mask = j0 + kTile > low || j0 + kTile > sp.n;
    if constexpr (DP <= 64) {
      r.template step<2>(lane, sk, sv, 0, c, mask, (int32_t)(seen - j0));
    } else {
#pragma unroll 1
      for (uint32_t x = 0; x < kTile; x += 32) r.template step<1>(lane, sk, sv, x, c, mask, (int32_t)(seen - j0 - x));
    }
    if constexpr (ODD) {
      if (odd)
        for (uint32_t x = 0; x < kTile; x += 32)
          add_odd<T, N>(r.o, ld.b, ld.b_stride, j0 + x, sp.n, d0 * 32, a.dim, half, false,
                        [&](uint32_t j) { return j < seen; });
    }
  }
  const float l = add_halves(r.l), inv = 1.f / l;
  bool found = false;
  if constexpr (!ODD) {
    if (causal && valid) {
      float x = 0.f;  // NaN or infinite if one of them is
#pragma unroll
      for (int d = 0; d < N; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) x = fmaxf(x, not_finite(r.o[d][i]) ? 1.f : 0.f);
      found = x > 0.f;
    }
    found = __syncthreads_or(found);
    if (found) return true;
  } else {
    __syncthreads();
  }
  T* out = (T*)a.out + (int64_t)(sp.first + w0) * a.out_stride[0] + (int64_t)hq * a.out_stride[1];
  write_rows<T, N>(s_kv + wave * 32 * (DP + 8), r.o, inv, out, a.out_stride[0], sp.n > w0 ? sp.n - w0 : 0, d0 * 32, a.dim, lane);
  if (a.lse && valid && half == 0 && d0 == 0)
    a.lse[(uint64_t)(sp.first + row) * a.q_heads + hq] = l == 0.f ? -INFINITY : (r.m * c + log2f(l)) * kLn2;
  return false;
}

// Zeros to the rows of a tile that is in no sequence.
template <uint32_t ROWS, typename T>
__device__ __forceinline__ void zero_rows(T* out, const int64_t* stride, const Span& sp, uint32_t head, uint32_t dim) {
  const uint32_t rows = sp.n - sp.tile * ROWS < ROWS ? sp.n - sp.tile * ROWS : ROWS, first = sp.first + sp.tile * ROWS;
  for (uint32_t i = threadIdx.x; i < rows * (dim / 8); i += blockDim.x)
    *(u32x4*)(out + (int64_t)(first + i / (dim / 8)) * stride[0] + (int64_t)head * stride[1] + i % (dim / 8) * 8) =
        u32x4{0, 0, 0, 0};
}

template <typename T, int DP>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void prompt_tile_kernel(PromptParams p) {
  const gts_prompt_args& a = p.a;
  __shared__ __align__(16) T s_kv[4 * Tiles<T, DP>::N];
  uint32_t h;
  uint32_t at;
  const uint32_t place = place_at(a.batch, a.tokens, p.places, a.q_heads, a.flags & GTS_PROMPT_CAUSAL, &at);
  const uint32_t hq = head_at(at, a.kv_heads, p.group, &h);
  Span sp;
  if (!find_span(a.starts, a.batch, a.tokens, kRows, place, &sp)) return;
  if (!sp.in) {
    zero_rows<kRows>((T*)a.out, a.out_stride, sp, hq, a.dim);
    const uint32_t first = sp.tile * kRows;
    if (a.lse)
      for (uint32_t i = first + threadIdx.x; i < sp.n && i < first + kRows; i += 256)
        a.lse[(uint64_t)(sp.first + i) * a.q_heads + hq] = -INFINITY;
    return;
  }
  if (prompt_rows<T, DP, false>(p, sp, hq, h, s_kv))
    for (int d = 0; d < DP / 32; ++d) prompt_rows<T, DP, true>(p, sp, hq, h, s_kv, d);
}

// ---- float16 in the gradient ------------------------------------------------------------------
// Weights p and their gradients ds are rounded to the tensors' type for the products.  float16 has all
// its bits from 2^-14 to 65504 only: p of n equal keys is 1 / n, and ds goes with dout and v, whose
// size nothing bounds.  So p is lifted by 2^10 (lse is 10 less in base 2), and ds scaled by a power of
// two of the lane's, whose row (dq) or key (dk) the sums are: the first that is not 0 to 2^8, and less
// when one has grown past 2^15.  The sums take both back in 32 bits.  bfloat16 has the range of
// 32 bits.  Largest, scaling and their registers cost 4 % of the gradient (4 x 2048 tokens, 16 heads of
// 128: 706 us without, 736 with), 11 % with heads of 256 (2 x 4096 causal, 16 / 4 heads: 2498, 2779).
template <typename T>
constexpr float kLift = __is_same(T, _Float16) ? 10.f : 0.f;

template <typename T>
struct Scaled {
  template <int N>
  __device__ __forceinline__ void fit(f32x16*, f32x16&) {}
  template <int N>
  __device__ __forceinline__ void back(f32x16*) const {}
};
template <>
struct Scaled<_Float16> {
  float f = 0x1p100f;  // 2^-120 at least
  __device__ __forceinline__ static float inverse(float power) { return __uint_as_float((254u << 23) - __float_as_uint(power)); }
  // w becomes f w; the sums o follow when f changes.
  template <int N>
  __device__ __forceinline__ void fit(f32x16* o, f32x16& w) {
    float mx = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, __builtin_fabsf(w[i]));
    mx = max_halves(mx);
    const bool large = mx * f > 0x1p15f;
    if (__any(large)) {
      const float f1 = large ? __uint_as_float((262u - (__float_as_uint(mx) >> 23)) << 23) : f, r = f1 * inverse(f);
#pragma unroll
      for (int d = 0; d < N; ++d) o[d] *= r;
      f = f1;
    }
    w *= f;
  }
  template <int N>
  __device__ __forceinline__ void back(f32x16* o) const {
    const float r = 0x1p-10f * inverse(f);
#pragma unroll
    for (int d = 0; d < N; ++d) o[d] *= r;
  }
};
// The same for sums of weights.
template <typename T, int N>
__device__ __forceinline__ void lower(f32x16* o) {
  if constexpr (kLift<T> != 0.f) {
#pragma unroll
    for (int d = 0; d < N; ++d) o[d] *= 0x1p-10f;
  }
}

struct PromptGradParams {
  gts_prompt_grad_args a;
  uint32_t group;
  uint32_t places;
  bool vec;      // rows of dout, q, k and v are aligned to 16 bytes
  // [q_heads][tokens]: a head's values side by side; lse in base 2, less kLift
  float *lse, *delta;
  uint32_t key_places;
  // The query heads of a key-value head are summed in this many parts; with more than one, the
  // parts are [splits][tokens][kv_heads][dim] in 32 bits.
  uint32_t splits;
  float* parts;
  uint32_t* order;  // [key_places] those with the most rows to a key first
  __device__ __forceinline__ uint64_t stat(uint32_t head, uint32_t token) const { return (uint64_t)head * a.tokens + token; }
};

// The order in which places of keys are taken: a workgroup's work goes with the rows that see its
// keys, and the longest must not begin last (8 packed texts in the order of their tokens: a fifth
// more time).  Places are counted by the logarithm of their work; a thread a place.
__device__ __forceinline__ void sort_places(const PromptGradParams& p) {
  const gts_prompt_grad_args& a = p.a;
  __shared__ uint32_t s_count[256];
  const auto bucket = [&](uint32_t place) {
    uint32_t lo = 0, n = a.batch + 2;  // as find_span, by one thread
    while (n > 1) {
      const uint32_t e = lo + n / 2;
      if (bound_of(a.starts, a.batch, a.tokens, e) / kKeys + e <= place) {
        lo = e;
        n -= n / 2;
      } else {
        n /= 2;
      }
    }
    const uint32_t b0 = bound_of(a.starts, a.batch, a.tokens, lo), b1 = bound_of(a.starts, a.batch, a.tokens, lo + 1);
    const uint64_t n_rows = b1 > b0 ? b1 - b0 : 0, k0 = (uint64_t)(place - (b0 / kKeys + lo)) * kKeys;
    const uint64_t work = k0 >= n_rows ? 0 : a.flags & GTS_PROMPT_CAUSAL ? n_rows - k0 : n_rows;
    return 255u - (uint32_t)(log2f((float)(work / kTile + 1)) * 9.f);  // 2^31 rows: 225
  };
  s_count[threadIdx.x] = 0;
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < p.key_places; i += 256) atomicAdd(&s_count[bucket(i)], 1u);
  __syncthreads();
  if (threadIdx.x == 0) {
    uint32_t sum = 0;
    for (int i = 0; i < 256; ++i) {
      const uint32_t c = s_count[i];
      s_count[i] = sum;
      sum += c;
    }
  }
  __syncthreads();
  // places of one bucket in any order: it says when they are taken, not what they give
  for (uint32_t i = threadIdx.x; i < p.key_places; i += 256) p.order[atomicAdd(&s_count[bucket(i)], 1u)] = i;
}

// delta, and lse in base 2: 64 tokens of a head a workgroup, 16 lanes a row.  The first workgroup
// sorts the places.
template <typename T>
__global__ __launch_bounds__(256) void stats_kernel(PromptGradParams p) {
  const gts_prompt_grad_args& a = p.a;
  if (blockIdx.x == 0) {
    sort_places(p);
    return;
  }
  const uint32_t h = (blockIdx.x - 1) % a.q_heads, t0 = (blockIdx.x - 1) / a.q_heads * 64, lane = threadIdx.x & 63u;
  const uint32_t sub = lane / 16, li = lane % 16;
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    const uint32_t t = t0 + (threadIdx.x >> 6) * 16 + i * 4 + sub;
    float sum = 0.f;
    if (t < a.tokens) {
      const T* x = (const T*)a.dout + (int64_t)t * a.dout_stride[0] + (int64_t)h * a.dout_stride[1];
      const T* y = (const T*)a.out + (int64_t)t * a.out_stride[0] + (int64_t)h * a.out_stride[1];
      for (uint32_t d = li * 8; d < a.dim; d += 128) {
        const Vec8<T> u = load8(x + d, (int64_t)a.dim - d), v = load8(y + d, (int64_t)a.dim - d);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += (float)u[j] * (float)v[j];
      }
    }
#pragma unroll
    for (int k = 8; k; k >>= 1) sum += __shfl_xor(sum, k);
    if (li == 0 && t < a.tokens) {
      p.delta[p.stat(h, t)] = sum;
      p.lse[p.stat(h, t)] = a.lse[(uint64_t)t * a.q_heads + h] * kLog2e - kLift<T>;
    }
  }
}

template <typename T, int DP>
__global__ __launch_bounds__(256) void dq_kernel(PromptGradParams p) {
  const gts_prompt_grad_args& a = p.a;
  __shared__ __align__(16) T s_k[kStep * kRowPitch<T, DP>], s_v[kStep * kRowPitch<T, DP>];
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, half = lane / 32;
  const uint32_t hq = blockIdx.x % a.q_heads, h = hq / p.group;
  Span sp;
  if (!find_span(a.starts, a.batch, a.tokens, kRows, blockIdx.x / a.q_heads, &sp)) return;
  const uint32_t r0 = sp.tile * kRows, row = r0 + wave * 32 + lane % 32, token = sp.first + row;
  const bool valid = row < sp.n, causal = a.flags & GTS_PROMPT_CAUSAL;
  T* dq = (T*)a.dq + (int64_t)token * a.dq_stride[0] + (int64_t)hq * a.dq_stride[1];
  f32x16 o[DP / 32];
  clear(o);
  if (!sp.in) {
    if (valid) write_row<T, DP>(dq, o, 0.f, a.dim, half);
    return;
  }
  Held<T, DP> q, dout;
  q.load((const T*)a.q + (int64_t)token * a.q_stride[0] + (int64_t)hq * a.q_stride[1], valid, a.dim, half);
  dout.load((const T*)a.dout + (int64_t)token * a.dout_stride[0] + (int64_t)hq * a.dout_stride[1], valid, a.dim, half);
  const T* k = (const T*)a.k + (int64_t)sp.first * a.k_stride[0] + (int64_t)h * a.k_stride[1];
  const T* v = (const T*)a.v + (int64_t)sp.first * a.v_stride[0] + (int64_t)h * a.v_stride[1];
  const uint32_t keys = causal && r0 + kRows < sp.n ? r0 + kRows : sp.n;
  const uint32_t sees = !valid ? 0 : causal ? row + 1 : sp.n;
  const float c = a.scale * kLog2e;
  const float lse = valid ? p.lse[p.stat(hq, token)] : 0.f;
  const float delta = valid ? p.delta[p.stat(hq, token)] : 0.f;
  Scaled<T> scaled;
  for (uint32_t j0 = 0; j0 < keys; j0 += kStep) {
    const bool edge = causal && j0 + kStep > r0 + 1;
    __syncthreads();
    stage_rows<T, DP>(k, a.k_stride[0], j0, sp.n, a.dim, false, s_k);
    stage_rows<T, DP>(v, a.v_stride[0], j0, sp.n, a.dim, false, s_v);
    __syncthreads();
    f32x16 s = times_held<T, DP>(s_k, q, lane);
    const f32x16 dp = times_held<T, DP>(s_v, dout, lane);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t j = j0 + frag_row(i, half);
      s[i] = j < sees && j < sp.n ? exp2_(s[i] * c - lse) * (dp[i] - delta) : 0.f;
    }
    bool odd = false;
    if (edge) {
      bool found = false;
      for (uint32_t id = threadIdx.x; id < kStep * (DP / 8); id += 256) {
        Vec8<T> x = read8(s_k + id / (DP / 8) * kRowPitch<T, DP> + id % (DP / 8) * 8);
        found |= clear_not_finite(x);
      }
      odd = __syncthreads_or(found);
      if (odd) {
        clear_rows<T, DP>(s_k);
        __syncthreads();
      }
    }
    scaled.template fit<DP / 32>(o, s);
    add_weighted<T, DP>(o, s_k, s, lane);
    if (odd) add_odd<T, DP / 32>(o, k, a.k_stride[0], j0, sp.n, 0, a.dim, half, true, [&](uint32_t j) { return j < sees; });
  }
  scaled.template back<DP / 32>(o);
  if (valid) write_row<T, DP>(dq, o, a.scale, a.dim, half);
}

// WHAT: 1 dv, 2 dk, 3 both (with one part only: the parts' memory is for one of them).
template <typename T, int DP, int WHAT>
__global__ __launch_bounds__(256) void dkv_kernel(PromptGradParams p) {
  const gts_prompt_grad_args& a = p.a;
  constexpr bool kV = WHAT & 1, kK = WHAT & 2;
  __shared__ __align__(16) T s_q[kStep * kRowPitch<T, DP>], s_o[kStep * kRowPitch<T, DP>];
  __shared__ float s_lse[kStep], s_delta[kStep];
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, half = lane / 32;
  const uint32_t h = blockIdx.x % a.kv_heads, at = blockIdx.x / a.kv_heads, place = at / p.splits, split = at - place * p.splits;
  Span sp;
  if (!find_span(a.starts, a.batch, a.tokens, kRows, place, &sp)) return;
  const uint32_t g0 = split * (p.group / p.splits), g1 = g0 + p.group / p.splits;  // its query heads
  const uint32_t k0 = sp.tile * kRows, key = k0 + wave * 32 + lane % 32, token = sp.first + key;
  const bool valid = key < sp.n, causal = a.flags & GTS_PROMPT_CAUSAL;
  T* dk = (T*)a.dk + (int64_t)token * a.dk_stride[0] + (int64_t)h * a.dk_stride[1];
  T* dv = (T*)a.dv + (int64_t)token * a.dv_stride[0] + (int64_t)h * a.dv_stride[1];
  f32x16 ok[kK ? DP / 32 : 1], ov[kV ? DP / 32 : 1];
  clear(ok);
  clear(ov);
  if (sp.in) {
    Held<T, DP> k, v;
    k.load((const T*)a.k + (int64_t)token * a.k_stride[0] + (int64_t)h * a.k_stride[1], valid, a.dim, half);
    if constexpr (kK)
      v.load((const T*)a.v + (int64_t)token * a.v_stride[0] + (int64_t)h * a.v_stride[1], valid, a.dim, half);
    const float c = a.scale * kLog2e;
    Scaled<T> scaled;
    const uint32_t first = causal ? k0 : 0;
    for (uint32_t g = g0; g < g1; ++g) {
      const uint32_t hq = h * p.group + g;
      const T* q = (const T*)a.q + (int64_t)sp.first * a.q_stride[0] + (int64_t)hq * a.q_stride[1];
      const T* dout = (const T*)a.dout + (int64_t)sp.first * a.dout_stride[0] + (int64_t)hq * a.dout_stride[1];
      for (uint32_t i0 = first; i0 < sp.n; i0 += kStep) {
        const bool edge = causal && i0 + 1 < k0 + kRows;  // some key is not seen by all of the rows
        __syncthreads();
        stage_rows<T, DP>(q, a.q_stride[0], i0, sp.n, a.dim, false, s_q);
        stage_rows<T, DP>(dout, a.dout_stride[0], i0, sp.n, a.dim, false, s_o);
        if (threadIdx.x < kStep) {
          const bool in = i0 + threadIdx.x < sp.n;
          const uint64_t at = p.stat(hq, sp.first + i0 + threadIdx.x);
          s_lse[threadIdx.x] = in ? p.lse[at] : 0.f;
          s_delta[threadIdx.x] = in ? p.delta[at] : 0.f;
        }
        __syncthreads();
        f32x16 s = times_held<T, DP>(s_q, k, lane), ds;
        if constexpr (kK) ds = times_held<T, DP>(s_o, v, lane);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t r = frag_row(i, half), row = i0 + r;
          const bool seen = row < sp.n && (!causal || key <= row);
          s[i] = seen ? exp2_(s[i] * c - s_lse[r]) : 0.f;
          if constexpr (kK) ds[i] = seen ? s[i] * (ds[i] - s_delta[r]) : 0.f;
        }
        bool odd = false;
        if (edge) {
          bool found = false;
          for (uint32_t id = threadIdx.x; id < kStep * (DP / 8); id += 256) {
            const uint32_t at = id / (DP / 8) * kRowPitch<T, DP> + id % (DP / 8) * 8;
            Vec8<T> x = read8(s_q + at), y = read8(s_o + at);
            found |= clear_not_finite(x);
            found |= clear_not_finite(y);
          }
          odd = __syncthreads_or(found);
          if (odd) {
            clear_rows<T, DP>(s_q);
            clear_rows<T, DP>(s_o);
            __syncthreads();
          }
        }
        if constexpr (kV) add_weighted<T, DP>(ov, s_o, s, lane);
        if constexpr (kK) {
          scaled.template fit<DP / 32>(ok, ds);
          add_weighted<T, DP>(ok, s_q, ds, lane);
        }
        if (odd) {
          const auto sees = [&](uint32_t row) { return key <= row; };
          if constexpr (kV) add_odd<T, DP / 32>(ov, dout, a.dout_stride[0], i0, sp.n, 0, a.dim, half, false, sees);
          if constexpr (kK) add_odd<T, DP / 32>(ok, q, a.q_stride[0], i0, sp.n, 0, a.dim, half, true, sees);
        }
      }
    }
    if constexpr (kV) lower<T, DP / 32>(ov);
    if constexpr (kK) scaled.template back<DP / 32>(ok);
  }
  if (!valid || (!sp.in && split)) return;
  if (WHAT != 3 && p.splits > 1 && sp.in) {
    float* out = p.parts + (((uint64_t)split * a.tokens + token) * a.kv_heads + h) * a.dim;
    if constexpr (kV)
      write_row<float, DP>(out, ov, 1.f, a.dim, half);
    else
      write_row<float, DP>(out, ok, a.scale, a.dim, half);
    return;
  }
  if constexpr (kV) write_row<T, DP>(dv, ov, 1.f, a.dim, half);
  if constexpr (kK) write_row<T, DP>(dk, ok, a.scale, a.dim, half);
}

// ---- the gradient's tile kernels -------------------------------------------------------------
// As prompt_tile_kernel: values that are not finite are looked for only where a result has one.
// Masked exponents are -inf then, whatever scale's sign and the row's log-sum are; with `odd` masked
// weights and their gradients are 0 whatever else the row has.
template <int N>
__device__ __forceinline__ bool any_odd(const f32x16 (&o)[N]) {
  bool found = false;
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) found |= not_finite(o[d][i]);
  return found;
}

// 32 rows of one or two tiles times held rows (B): the fragments of AHEAD steps are read while those
// before are multiplied.
template <typename T, int DP, bool BOTH, int AHEAD>
__device__ __forceinline__ void two_products(const Parts<T, DP>& at, const T* sa, const T* sb, uint32_t row, const Vec8<T>* a,
                                             const Vec8<T>* b, f32x16& ra, f32x16& rb) {
#pragma unroll
  for (int i = 0; i < 16; ++i) ra[i] = rb[i] = 0.f;
  Vec8<T> f[2][AHEAD][2];
  const auto read = [&](int kk) {
#pragma unroll
    for (int x = 0; x < AHEAD; ++x) {
      f[kk / AHEAD & 1][x][0] = at.rows(sa, row, kk + x);
      if constexpr (BOTH) f[kk / AHEAD & 1][x][1] = at.rows(sb, row, kk + x);
    }
  };
  read(0);
#pragma unroll
  for (int kk = 0; kk < DP / 16; kk += AHEAD) {
    if (kk + AHEAD < DP / 16) read(kk + AHEAD);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int x = 0; x < AHEAD; ++x) {
      ra = mfma(f[kk / AHEAD & 1][x][0], a[kk + x], ra);
      if constexpr (BOTH) rb = mfma(f[kk / AHEAD & 1][x][1], b[kk + x], rb);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}
// N blocks of columns, from block d0 on, of 32 rows of a tile times the lane's weights, rounded to T.
template <typename T, int DP, int N>
__device__ __forceinline__ void add_columns(const Parts<T, DP>& at, f32x16* o, const T* s, uint32_t row, int d0, const f32x16& w,
                                            uint32_t lane) {
  Vec8<T> u[2], f[2][N];
  const auto columns = [&](uint32_t from, int d) {
    if constexpr (N == DP / 32)
      return at.columns(s, from, d);
    else
      return column_frag<T, DP>(s, from, d0 + d, lane);
  };
#pragma unroll
  for (int d = 0; d < N; ++d) f[0][d] = columns(row, d);
#pragma unroll
  for (int i = 0; i < 16; ++i) u[i / 8][i % 8] = (T)w[i];
#pragma unroll
  for (int d = 0; d < N; ++d) f[1][d] = columns(row + 16, d);
#pragma unroll
  for (int y = 0; y < 2; ++y)
#pragma unroll
    for (int d = 0; d < N; ++d) o[d] = mfma(f[y][d], u[y], o[d]);
}
// At an edge, once every wave has its scores: whether the tile has a value that is not finite; those
// are zeros afterwards.
template <typename T, int N>
__device__ __forceinline__ bool clear_if_odd(T* s, bool edge, uint32_t threads) {
  if (!edge) return false;
  bool found = false;
  for (uint32_t x = threadIdx.x; x < N / 8; x += threads) found |= any_not_finite<T>(*(const u32x4*)(s + x * 8));
  if (!__syncthreads_or(found)) return false;
  for (uint32_t x = threadIdx.x; x < N / 8; x += threads) *(u32x4*)(s + x * 8) = finite_only<T>(*(const u32x4*)(s + x * 8));
  __syncthreads();
  return true;
}

template <typename T, int DP, bool ODD>
__device__ __forceinline__ bool dq_rows(const PromptGradParams& p, const Span& sp, uint32_t hq, uint32_t h, T* s_kv,
                                        int d0 = 0) {
  constexpr int N = ODD ? 1 : DP / 32;
  using L = Tiles<T, DP>;
  const gts_prompt_grad_args& a = p.a;
  const uint32_t lane = fresh_lane(), wave = uni(threadIdx.x >> 6), half = lane / 32;
  const uint32_t r0 = sp.tile * kRows, w0 = r0 + wave * 32, row = w0 + lane % 32, there = row < sp.n ? row : 0;
  const bool valid = row < sp.n, causal = a.flags & GTS_PROMPT_CAUSAL;
  const float c = a.scale * kLog2e;
  Loader<T, DP> ld;
  ld.a = (const T*)a.k + (int64_t)sp.first * a.k_stride[0] + (int64_t)h * a.k_stride[1];
  ld.b = (const T*)a.v + (int64_t)sp.first * a.v_stride[0] + (int64_t)h * a.v_stride[1];
  ld.a_stride = a.k_stride[0];
  ld.b_stride = a.v_stride[0];
  ld.n = sp.n;
  ld.dim = a.dim;
  ld.start();
  const uint32_t keys = causal && r0 + kRows < sp.n ? r0 + kRows : sp.n, tiles = (keys + kTile - 1) / kTile;
  __syncthreads();
  ld.load(0, wave, s_kv, s_kv + L::N);
  Vec8<T> q[DP / 16], dout[DP / 16];
  const T* qp = (const T*)a.q + (int64_t)(sp.first + there) * a.q_stride[0] + (int64_t)hq * a.q_stride[1];
  const T* op = (const T*)a.dout + (int64_t)(sp.first + there) * a.dout_stride[0] + (int64_t)hq * a.dout_stride[1];
#pragma unroll
  for (int i = 0; i < DP / 16; ++i) {
    const uint32_t c0 = i * 16 + 8 * half;
    q[i] = *(const Vec8<T>*)(c0 < a.dim ? qp + c0 : (const T*)g_zeros);
    dout[i] = *(const Vec8<T>*)(c0 < a.dim ? op + c0 : (const T*)g_zeros);
  }
  const float lse = p.lse[p.stat(hq, sp.first + there)], delta = p.delta[p.stat(hq, sp.first + there)];
  f32x16 o[N];
  clear(o);
  Parts<T, DP> at;
  at.start(lane);
  Scaled<T> scaled;
  for (uint32_t t = 0; t < tiles; ++t) {
    const uint32_t j0 = t * kTile;
    T *sk = s_kv + (t & 1) * 2 * L::N, *sv = sk + L::N;
    wait_loads();
    __syncthreads();
    if (t + 1 < tiles) {
      T* next = s_kv + ((t + 1) & 1) * 2 * L::N;
      ld.load(j0 + kTile, wave, next, next + L::N);
    }
    const uint32_t seen = causal && row + 1 < sp.n ? row + 1 : sp.n;
    if (!ODD && causal && j0 > w0 + 31) continue;  // the wave sees none of it
    const bool mask = j0 + kTile > (causal ? w0 + 1 : sp.n) || j0 + kTile > sp.n;
    const auto weigh = [&](uint32_t x, f32x16& s, const f32x16& dp, bool masked) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const bool hidden = masked && j0 + x + frag_row(i, half) >= seen;
        float y = __builtin_fmaf(s[i], c, -lse);  // hidden behind the product: c has scale's sign
        if (!ODD && hidden) y = -INFINITY;
        y = exp2_(y) * (dp[i] - delta);
        s[i] = ODD && hidden ? 0.f : y;
      }
    };
    if constexpr (!ODD) {
#pragma unroll 1
      for (uint32_t x = 0; x < kTile; x += 32) {
        f32x16 s, dp;
        two_products<T, DP, true, 1>(at, sk, sv, x, q, dout, s, dp);
        if (mask)
          weigh(x, s, dp, true);
        else
          weigh(x, s, dp, false);
        scaled.template fit<N>(o, s);
        add_columns<T, DP, N>(at, o, sk, x, 0, s, lane);
      }
    } else {
      f32x16 s[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        f32x16 dp;
        two_products<T, DP, true, 1>(at, sk, sv, x * 32, q, dout, s[x], dp);
        weigh(x * 32, s[x], dp, true);
      }
      const bool odd = clear_if_odd<T, L::N>(sk, causal && j0 + kTile > r0 + 1, 256);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        scaled.template fit<N>(o, s[x]);
        add_columns<T, DP, N>(at, o, sk, x * 32, d0, s[x], lane);
        if (odd)
          add_odd<T, N>(o, ld.a, ld.a_stride, j0 + x * 32, sp.n, d0 * 32, a.dim, half, true,
                        [&](uint32_t j) { return j < seen; });
      }
    }
  }
  scaled.template back<N>(o);
  if constexpr (!ODD) {
    if (__syncthreads_or(causal && valid && any_odd(o))) return true;
  } else {
    __syncthreads();
  }
  T* out = (T*)a.dq + (int64_t)(sp.first + w0) * a.dq_stride[0] + (int64_t)hq * a.dq_stride[1];
  write_rows<T, N>(s_kv + wave * 32 * (DP + 8), o, a.scale, out, a.dq_stride[0], sp.n > w0 ? sp.n - w0 : 0, d0 * 32, a.dim, lane);
  return false;
}

template <typename T, int DP>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void dq_tile_kernel(PromptGradParams p) {
  const gts_prompt_grad_args& a = p.a;
  __shared__ __align__(16) T s_kv[4 * Tiles<T, DP>::N];
  uint32_t h;
  uint32_t at;
  const uint32_t place = place_at(a.batch, a.tokens, p.places, a.q_heads, a.flags & GTS_PROMPT_CAUSAL, &at);
  const uint32_t hq = head_at(at, a.kv_heads, p.group, &h);
  Span sp;
  if (!find_span(a.starts, a.batch, a.tokens, kRows, place, &sp)) return;
  if (!sp.in) {
    zero_rows<kRows>((T*)a.dq, a.dq_stride, sp, hq, a.dim);
    return;
  }
  if (dq_rows<T, DP, false>(p, sp, hq, h, s_kv))
    for (int d = 0; d < DP / 32; ++d) dq_rows<T, DP, true>(p, sp, hq, h, s_kv, d);
}

// 4 bytes a lane from memory to LDS, as load_to_lds.
__device__ __forceinline__ void load_to_lds4(const void* from, void* to) {
  const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)to;
  uint32_t m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %2, off\n\ts_mov_b32 m0, %0"
               : "=&s"(m0)
               : "s"(at), "v"(from)
               : "memory");
}

// 64 keys, two groups of 32; all rows that see them, of all query heads of the key-value head,
// 64 at a time: four waves, one for each group of keys and half of the rows, whose sums are joined
// at the end.  dv and dk take a kernel each (`DV`), which computes the scores once more but leaves
// registers for two waves a SIMD, one of which computes weights while the other multiplies.
// Heads of 256 take two passes of 128 columns each, for which there are registers.  8 packed texts of
// 512 to 8192 tokens, 32 / 8 heads of 128: dq 729, dk 819 and dv 654 us under the profiler (the whole gradient took
// 2604 with one kernel for both, one wave a SIMD; 2360 with two).
template <int DP>
constexpr int kBlocks = DP / 32 < 4 ? DP / 32 : 4;

template <typename T, int DP, bool DV, bool ODD>
__device__ __forceinline__ bool dkv_keys(const PromptGradParams& p, const Span& sp, uint32_t h, uint32_t split, T* s_qo,
                                         float (*s_stat)[2][kTile], int d0 = 0) {
  using L = Tiles<T, DP>;
  constexpr int KK = DP / 16, N = ODD ? 1 : kBlocks<DP>;
  const gts_prompt_grad_args& a = p.a;
  const uint32_t lane = fresh_lane(), wave = uni(threadIdx.x >> 6), half = lane / 32, x0 = wave / 2 * 32;
  const uint32_t k0 = sp.tile * kKeys, w0 = k0 + wave % 2 * 32, key = w0 + lane % 32, there = key < sp.n ? key : 0;
  const bool valid = key < sp.n, causal = a.flags & GTS_PROMPT_CAUSAL;
  const float c = a.scale * kLog2e;
  Loader<T, DP> ld;
  ld.a_stride = a.q_stride[0];
  ld.b_stride = a.dout_stride[0];
  ld.n = sp.n;
  ld.dim = a.dim;
  ld.start();
  const uint32_t first = causal ? k0 / kTile : 0, tiles = (sp.n + kTile - 1) / kTile;
  const auto load = [&](uint32_t g, uint32_t t, uint32_t buffer) {
    const uint32_t hq = h * p.group + g;
    ld.a = (const T*)a.q + (int64_t)sp.first * a.q_stride[0] + (int64_t)hq * a.q_stride[1];
    ld.b = (const T*)a.dout + (int64_t)sp.first * a.dout_stride[0] + (int64_t)hq * a.dout_stride[1];
    T* to = s_qo + buffer * 2 * L::N;
    ld.load(t * kTile, wave, to, to + L::N);
    if (wave < 2) {  // statistics: a wave each
      const uint32_t i = t * kTile + fresh_lane();
      const float* from = (wave ? p.delta : p.lse) + p.stat(hq, sp.first + i);
      load_to_lds4(i < sp.n ? from : (const float*)g_zeros, s_stat[buffer][wave]);
    }
  };
  const uint32_t g0 = split * (p.group / p.splits), g1 = g0 + p.group / p.splits;  // its query heads
  __syncthreads();
  load(g0, first, 0);
  Vec8<T> k[KK], v[DV ? 1 : KK];
  const T* kp = (const T*)a.k + (int64_t)(sp.first + there) * a.k_stride[0] + (int64_t)h * a.k_stride[1];
  const T* vp = (const T*)a.v + (int64_t)(sp.first + there) * a.v_stride[0] + (int64_t)h * a.v_stride[1];
#pragma unroll
  for (int i = 0; i < KK; ++i) {
    const uint32_t at = i * 16 + 8 * half;
    k[i] = *(const Vec8<T>*)(at < a.dim ? kp + at : (const T*)g_zeros);
    if constexpr (!DV) v[i] = *(const Vec8<T>*)(at < a.dim ? vp + at : (const T*)g_zeros);
  }
  f32x16 o[N];
  clear(o);
  Parts<T, DP> at;
  at.start(lane);
  Scaled<T> scaled;
  uint32_t buffer = 0;
  for (uint32_t g = g0; g < g1; ++g)
    for (uint32_t t = first; t < tiles; ++t, buffer ^= 1) {
      const uint32_t i0 = t * kTile + x0;  // the wave's first row
      T *sq = s_qo + buffer * 2 * L::N, *so = sq + L::N, *added = DV ? so : sq;
      wait_loads();
      __syncthreads();
      if (t + 1 < tiles)
        load(g, t + 1, buffer ^ 1);
      else if (g + 1 < g1)
        load(g + 1, first, buffer ^ 1);
      if (!ODD && ((causal && i0 + 32 <= w0) || i0 >= sp.n)) continue;  // no row of the wave's sees a key of its
      const bool mask = (causal && i0 < w0 + 31) || i0 + 32 > sp.n;
      f32x16 s, dp;
      two_products<T, DP, !DV, 2>(at, sq, so, x0, k, v, s, dp);
      const auto weigh = [&](bool masked) {
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const uint32_t r = frag_row(e, half);  // four rows side by side
          const f32x4 lse = *(const f32x4*)&s_stat[buffer][0][x0 + r];
          f32x4 delta = {};
          if constexpr (!DV) delta = *(const f32x4*)&s_stat[buffer][1][x0 + r];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool hidden = masked && ((causal && i0 + r + i < key) || i0 + r + i >= sp.n);
            float y = __builtin_fmaf(s[e + i], c, -lse[i]);  // hidden behind the product: c has scale's sign
            if (!ODD && hidden) y = -INFINITY;
            y = exp2_(y);
            if constexpr (!DV) y *= dp[e + i] - delta[i];
            s[e + i] = ODD && hidden ? 0.f : y;
          }
        }
      };
      if (ODD || mask)
        weigh(true);
      else
        weigh(false);
      bool odd = false;
      if constexpr (ODD) odd = clear_if_odd<T, L::N>(added, causal && t * kTile + 1 < k0 + kKeys, 256);
      if constexpr (!DV) scaled.template fit<N>(o, s);
      add_columns<T, DP, N>(at, o, added, x0, d0, s, lane);
      if constexpr (ODD) {
        if (odd) {
          const uint32_t hq = h * p.group + g;
          const T* from = DV ? (const T*)a.dout + (int64_t)sp.first * a.dout_stride[0] + (int64_t)hq * a.dout_stride[1]
                             : (const T*)a.q + (int64_t)sp.first * a.q_stride[0] + (int64_t)hq * a.q_stride[1];
          add_odd<T, N>(o, from, DV ? a.dout_stride[0] : a.q_stride[0], i0, sp.n, d0 * 32, a.dim, half, !DV,
                        [&](uint32_t row) { return key <= row; });
        }
      }
    }
  if constexpr (DV)
    lower<T, N>(o);
  else
    scaled.template back<N>(o);
  // the second half's sums, a block of columns at a time, to the first half's waves
  __syncthreads();
  float* s_sum = (float*)s_qo + wave % 2 * (N * 1024) + lane * 4;
  static_assert(2 * N * 1024 * 4 <= 4 * L::N * sizeof(T), "the sums fit the tiles' LDS");
  if (wave >= 2) {
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = o[d][i * 4 + e];
        *(f32x4*)(s_sum + d * 1024 + i * 256) = y;
      }
  }
  __syncthreads();
  if (wave < 2) {
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 y = *(const f32x4*)(s_sum + d * 1024 + i * 256);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[d][i * 4 + e] += y[e];
      }
  }
  if constexpr (!ODD) {
    if (__syncthreads_or(causal && wave < 2 && valid && any_odd(o))) return true;
  } else {
    __syncthreads();
  }
  if (wave >= 2) return false;
  const uint32_t rows = sp.n > w0 ? sp.n - w0 : 0;
  if (p.splits == 1) {
    const int64_t* stride = DV ? a.dv_stride : a.dk_stride;
    T* out = (T*)(DV ? a.dv : a.dk) + (int64_t)(sp.first + w0) * stride[0] + (int64_t)h * stride[1];
    write_rows<T, N>(s_qo + wave * 32 * (DP + 8), o, DV ? 1.f : a.scale, out, stride[0], rows, d0 * 32, a.dim, lane);
  } else if (valid) {
    float* out = p.parts + (((uint64_t)split * a.tokens + sp.first + key) * a.kv_heads + h) * a.dim;
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const uint32_t c = (d0 + d) * 32 + frag_row(i, half);
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = o[d][i + e] * (DV ? 1.f : a.scale);
        if (c < a.dim) *(f32x4*)(out + c) = y;
      }
  }
  return false;
}

template <typename T, int DP, bool DV>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void dkv_tile_kernel(PromptGradParams p) {
  const gts_prompt_grad_args& a = p.a;
  __shared__ __align__(16) T s_qo[4 * Tiles<T, DP>::N];
  __shared__ __align__(16) float s_stat[2][2][kTile];
  const uint32_t h = blockIdx.x % a.kv_heads, at = blockIdx.x / a.kv_heads, place = at / p.splits, split = at - place * p.splits;
  Span sp;
  if (!find_span(a.starts, a.batch, a.tokens, kKeys, uni(p.order[place]), &sp)) return;
  if (!sp.in) {
    if (split) return;
    if (DV)
      zero_rows<kKeys>((T*)a.dv, a.dv_stride, sp, h, a.dim);
    else
      zero_rows<kKeys>((T*)a.dk, a.dk_stride, sp, h, a.dim);
    return;
  }
  bool odd = false;
  for (int d = 0; d < DP / 32; d += kBlocks<DP>) odd |= dkv_keys<T, DP, DV, false>(p, sp, h, split, s_qo, s_stat, d);
  if (odd)
    for (int d = 0; d < DP / 32; ++d) dkv_keys<T, DP, DV, true>(p, sp, h, split, s_qo, s_stat, d);
}

// The parts' sum, in order, for the tokens of the sequences; V values a thread.
template <typename T, int V>
__global__ __launch_bounds__(256) void join_parts_kernel(PromptGradParams p, T* out, int64_t stride0, int64_t stride1) {
  const gts_prompt_grad_args& a = p.a;
  const uint64_t i = (block_number() * 256 + threadIdx.x) * V, all = (uint64_t)a.tokens * a.kv_heads * a.dim;
  if (i >= all) return;
  const uint64_t row = i / a.dim;
  const uint32_t c = (uint32_t)(i - row * a.dim), t = (uint32_t)(row / a.kv_heads), h = (uint32_t)(row - (uint64_t)t * a.kv_heads);
  if (a.starts && (int64_t)t < a.starts[0]) return;
  if (a.starts && (int64_t)t >= a.starts[a.batch]) return;
  Pack<float, V> sum = *(const Pack<float, V>*)(p.parts + i);
  for (uint32_t s = 1; s < p.splits; ++s) {
    const Pack<float, V> x = *(const Pack<float, V>*)(p.parts + s * all + i);
#pragma unroll
    for (int e = 0; e < V; ++e) sum.v[e] += x.v[e];
  }
  Pack<T, V> y;
#pragma unroll
  for (int e = 0; e < V; ++e) y.v[e] = (T)sum.v[e];
  *(Pack<T, V>*)(out + (int64_t)t * stride0 + (int64_t)h * stride1 + c) = y;
}

bool rows_aligned(const void* p, const int64_t* stride, uint32_t e) {
  return (uintptr_t)p % 16 == 0 && (uint64_t)stride[0] * e % 16 == 0 && (uint64_t)stride[1] * e % 16 == 0;
}

// 16 rows lie within 2 GiB: a tile's offsets have 32 bits.
bool near(const int64_t* stride) { return stride[0] >= 0 && stride[0] < 1 << 26; }

template <typename T, int DP>
hipError_t launch_prompt_d(const PromptParams& p, hipStream_t s) {
  const dim3 grid(p.places * p.a.q_heads), block(256);
  if constexpr (sizeof(T) == 2) {
    const gts_prompt_args& a = p.a;
    if (p.vec && a.dim % 8 == 0 && rows_aligned(a.out, a.out_stride, 2) && near(a.k_stride) && near(a.v_stride)) {
      prompt_tile_kernel<T, DP><<<grid, block, 0, s>>>(p);
      return hipGetLastError();
    }
  }
  prompt_kernel<T, DP><<<grid, block, 0, s>>>(p);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_prompt_t(const gts_prompt_args& a, hipStream_t s) {
  PromptParams p{a, a.q_heads / a.kv_heads, places_of(a.batch, a.tokens, kRows), false};
  p.vec = rows_aligned(a.q, a.q_stride, sizeof(T)) && rows_aligned(a.k, a.k_stride, sizeof(T)) &&
          rows_aligned(a.v, a.v_stride, sizeof(T));
  if (a.dim <= 64) return launch_prompt_d<T, 64>(p, s);
  if (a.dim <= 128) return launch_prompt_d<T, 128>(p, s);
  return launch_prompt_d<T, 256>(p, s);
}

// Parts of the sum over a key-value head's query heads: where its workgroups do not fill the chip
// twice over, the most that divide the group and give no more than that.  By sizes alone.
uint32_t splits_of(uint32_t tokens, uint32_t q_heads, uint32_t kv_heads) {
  const uint32_t group = q_heads / kv_heads;
  const uint64_t groups = (uint64_t)(tokens / kKeys + 1) * kv_heads;
  uint32_t n = 1;
  for (uint32_t s = 2; s <= group && groups * s <= 1024; ++s)
    if (group % s == 0) n = s;
  return n;
}
uint64_t parts_bytes(uint32_t tokens, uint32_t q_heads, uint32_t kv_heads, uint32_t dim) {
  const uint32_t s = splits_of(tokens, q_heads, kv_heads);
  return s > 1 ? ((4ull * s * tokens * kv_heads * dim + 15) & ~15ull) : 0;
}

template <typename T, int DP>
hipError_t launch_prompt_grad_d(const PromptGradParams& p, hipStream_t s) {
  const gts_prompt_grad_args& a = p.a;
  const dim3 rows(p.places * a.q_heads), keys(p.places * a.kv_heads * p.splits), block(256);
  stats_kernel<T><<<dim3((a.tokens + 63) / 64 * a.q_heads + 1), block, 0, s>>>(p);
  if constexpr (sizeof(T) == 2) {
    if (p.vec && a.dim % 8 == 0 && rows_aligned(a.dq, a.dq_stride, 2) && rows_aligned(a.dk, a.dk_stride, 2) &&
        rows_aligned(a.dv, a.dv_stride, 2) && near(a.k_stride) && near(a.v_stride) && near(a.q_stride) && near(a.dout_stride)) {
      dq_tile_kernel<T, DP><<<rows, block, 0, s>>>(p);
      const dim3 groups(p.key_places * a.kv_heads * p.splits);
      const dim3 join = grid_of(((uint64_t)a.tokens * a.kv_heads * a.dim / 4 + 255) / 256);
      dkv_tile_kernel<T, DP, false><<<groups, block, 0, s>>>(p);
      if (p.splits > 1) join_parts_kernel<T, 4><<<join, block, 0, s>>>(p, (T*)a.dk, a.dk_stride[0], a.dk_stride[1]);
      dkv_tile_kernel<T, DP, true><<<groups, block, 0, s>>>(p);
      if (p.splits > 1) join_parts_kernel<T, 4><<<join, block, 0, s>>>(p, (T*)a.dv, a.dv_stride[0], a.dv_stride[1]);
      return hipGetLastError();
    }
  }
  dq_kernel<T, DP><<<rows, block, 0, s>>>(p);
  if (DP == 256 || p.splits > 1) {  // no registers for both, or no memory for both's parts
    const dim3 join = grid_of(((uint64_t)a.tokens * a.kv_heads * a.dim + 255) / 256);
    dkv_kernel<T, DP, 1><<<keys, block, 0, s>>>(p);
    if (p.splits > 1) join_parts_kernel<T, 1><<<join, block, 0, s>>>(p, (T*)a.dv, a.dv_stride[0], a.dv_stride[1]);
    dkv_kernel<T, DP, 2><<<keys, block, 0, s>>>(p);
    if (p.splits > 1) join_parts_kernel<T, 1><<<join, block, 0, s>>>(p, (T*)a.dk, a.dk_stride[0], a.dk_stride[1]);
  } else if constexpr (DP < 256) {
    dkv_kernel<T, DP, 3><<<keys, block, 0, s>>>(p);
  }
  return hipGetLastError();
}
template <typename T>
hipError_t launch_prompt_grad_t(const gts_prompt_grad_args& a, hipStream_t s) {
  PromptGradParams p{};
  p.a = a;
  p.group = a.q_heads / a.kv_heads;
  p.places = places_of(a.batch, a.tokens, kRows);
  p.key_places = places_of(a.batch, a.tokens, kKeys);
  p.splits = splits_of(a.tokens, a.q_heads, a.kv_heads);
  p.parts = (float*)a.scratch;
  p.lse = (float*)((char*)a.scratch + parts_bytes(a.tokens, a.q_heads, a.kv_heads, a.dim));
  p.delta = p.lse + (uint64_t)a.tokens * a.q_heads;
  p.order = (uint32_t*)(p.delta + (uint64_t)a.tokens * a.q_heads);
  p.vec = rows_aligned(a.q, a.q_stride, sizeof(T)) && rows_aligned(a.k, a.k_stride, sizeof(T)) &&
          rows_aligned(a.v, a.v_stride, sizeof(T)) && rows_aligned(a.dout, a.dout_stride, sizeof(T));
  if (a.dim <= 64) return launch_prompt_grad_d<T, 64>(p, s);
  if (a.dim <= 128) return launch_prompt_grad_d<T, 128>(p, s);
  return launch_prompt_grad_d<T, 256>(p, s);
}

}  // namespace

uint64_t prompt_groups(uint32_t batch, uint32_t tokens, uint32_t heads) {
  return (uint64_t)places_of(batch, tokens, kKeys) * heads;  // the most of any kernel
}

hipError_t launch_prompt(const gts_prompt_args& a, hipStream_t s) {
  if (a.dtype == GTS_F32) return launch_prompt_t<float>(a, s);
  if (a.dtype == GTS_BF16) return launch_prompt_t<__bf16>(a, s);
  return launch_prompt_t<_Float16>(a, s);
}

uint64_t prompt_grad_scratch(uint32_t batch, uint32_t tokens, uint32_t q_heads, uint32_t kv_heads, uint32_t dim) {
  return parts_bytes(tokens, q_heads, kv_heads, dim) + 8ull * tokens * q_heads + 4ull * places_of(batch, tokens, kKeys);
}

hipError_t launch_prompt_grad(const gts_prompt_grad_args& a, hipStream_t s) {
  if (a.dtype == GTS_F32) return launch_prompt_grad_t<float>(a, s);
  if (a.dtype == GTS_BF16) return launch_prompt_grad_t<__bf16>(a, s);
  return launch_prompt_grad_t<_Float16>(a, s);
}

}  // namespace gts
