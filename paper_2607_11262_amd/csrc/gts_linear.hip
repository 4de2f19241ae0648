// gts_linear.hip — matrix products with bias, activation, gate and residual in the
// epilogue, and the elementwise part of their gradient.
//
//   z = sum_k a[m][k] b[n][k] + bias[n],  out = act(z) gate[m][n] + residual[m][n]
//   dz = dy gate act'(z),  dgate = dy act(z),  dbias[n] = sum_m dz[m][n]
//
// Either operand may be stored with the sum's index as its rows (the products of a
// backward pass), so nothing is transposed in memory.
#include <type_traits>

#include "gts_ops.h"
#include "gts_tile.h"

namespace gts {
namespace {

// ---- activations ---------------------------------------------------------------------

constexpr float kRootHalf = 0.70710678118654752f;   // 1 / sqrt(2)
constexpr float kNormal = 0.39894228040143268f;     // 1 / sqrt(2 pi)
constexpr float kTanhA = 0.79788456080286536f;      // sqrt(2 / pi)
constexpr float kTanhB = 0.044715f;

// One exponential and one reciprocal of the card's, off by a step of 32 bits each; the argument's
// rounding is |x| steps of the exponential.
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + exp2_(-kLog2e * x)); }
// Twice the argument of the tanh form; past 30 its sigmoid is 0 or 1 in 32 bits.
__device__ __forceinline__ float clamp30(float z) { return fminf(fmaxf(z, -30.f), 30.f); }
__device__ __forceinline__ float tanh_arg(float z) { return 2.f * kTanhA * (z + kTanhB * z * z * z); }

// The activation of z and its slope there; what the caller drops is not computed.
struct Shape {
  float y, slope;
};
template <uint32_t ACT>
__device__ __forceinline__ Shape shape_of(float z) {
  if constexpr (ACT == GTS_ACT_RELU) {
    return {z > 0.f || z != z ? z : 0.f, z > 0.f ? 1.f : z != z ? z : 0.f};
  } else if constexpr (ACT == GTS_ACT_GELU) {
    const float below = 0.5f * erfcf(-z * kRootHalf);  // no difference of near numbers for z < 0
    return {z * below, below + z * kNormal * exp2_(-0.5f * kLog2e * z * z)};
  } else if constexpr (ACT == GTS_ACT_GELU_TANH) {
    const float c = clamp30(z), s = sigmoid(tanh_arg(c));
    return {z != z ? z : z * s, z != z ? z : s + c * s * (1.f - s) * 2.f * kTanhA * (1.f + 3.f * kTanhB * c * c)};
  } else if constexpr (ACT == GTS_ACT_SILU) {
    const float s = sigmoid(z);
    return {z * s, s * (1.f + z * (1.f - s))};
  } else {
    return {z, 1.f};
  }
}
template <uint32_t ACT, int N>
__device__ __forceinline__ void activate_all(float* z) {
#pragma unroll
  for (int i = 0; i < N; ++i) z[i] = shape_of<ACT>(z[i]).y;
}
template <int N>
__device__ __forceinline__ void activate(uint32_t act, float* z) {
  switch (act) {
    case GTS_ACT_RELU: return activate_all<GTS_ACT_RELU, N>(z);
    case GTS_ACT_GELU: return activate_all<GTS_ACT_GELU, N>(z);
    case GTS_ACT_GELU_TANH: return activate_all<GTS_ACT_GELU_TANH, N>(z);
    case GTS_ACT_SILU: return activate_all<GTS_ACT_SILU, N>(z);
    default: return;
  }
}

struct MatmulParams {
  gts_matmul_args a;
  uint32_t splits;     // of the sum; more than one: the parts go to the scratch
  uint32_t k_split;    // places of a split
  bool wide;           // eight values of a result, its bias, gate and residual are 16 bytes
};

// What becomes of z = the whole sum of (m, n).
template <typename T>
__device__ __forceinline__ void finish(const gts_matmul_args& a, uint32_t m, uint32_t n, float z) {
  if (a.bias) z += (float)((const T*)a.bias)[n];
  if (a.preact) ((T*)a.preact)[(int64_t)m * a.preact_stride + n] = (T)z;
  activate<1>(a.activation, &z);
  if (a.gate) z *= (float)((const T*)a.gate)[(int64_t)m * a.gate_stride + n];
  if (a.residual) z += (float)((const T*)a.residual)[(int64_t)m * a.residual_stride + n];
  ((T*)a.out)[(int64_t)m * a.out_stride + n] = (T)z;
}

// ---- the general kernel ----------------------------------------------------------------
// Any type, size, stride and alignment.  Four waves take 32 R x 32 R each of a tile of 64 R x
// 64 R; 32 places of the sum at a time go through registers to LDS, their loads two stages ahead of
// the products.  The smaller tile is for small results, where more workgroups a CU hide the loads
// (1021 x 1000 x 777 in 32 bits: 51 us in the larger, 25 in this).  In 32 bits bound by matrix issue, a
// sixteenth of the 16-bit rate (4096 x 4096 x 4096 1021 us, 135 TFLOP/s; a library product 997; with
// loads one stage ahead, in one loop with those of the edges, 1140); in 16 bits by the way through
// registers (4095 x 4097 x 4099 333 us, 413 TFLOP/s).
constexpr uint32_t kTileK = 32;

// LDS of an operand's 64 R rows (or columns) and 32 places: rows of 8 values (16 bytes) more than they
// hold, so that reads of neighbouring rows meet other banks.
template <typename T, bool COLUMNS, int R>
constexpr uint32_t kPitch = COLUMNS ? 64 * R + 8 : kTileK + 16 / sizeof(T);
template <int R>
constexpr uint32_t kTileSize = 64 * R * (kTileK + 8);  // the larger of both

template <typename T, bool COLUMNS, int R>
struct Staged {
  Vec8<T> x[R];
  // Rows r0 .. + 64 R - 1 of `rows`, places k0 .. + 31, which are all there: without a branch, so that
  // nothing waits for the loads.  Rows past the end are the last again (what they give is not stored).
  __device__ __forceinline__ void load_whole(const T* p, int64_t stride, uint32_t r0, uint32_t rows, uint32_t k0) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const uint32_t id = threadIdx.x + 256 * i, r = r0 + id / 4;
      x[i] = COLUMNS ? load_any(p + (int64_t)(k0 + id / (8 * R)) * stride + r0 + id % (8 * R) * 8)
                     : load_any(p + (int64_t)(r < rows ? r : rows - 1) * stride + k0 + id % 4 * 8);
    }
  }
  // The same of the places below `k_end`, or columns of which some may be missing.
  __device__ __forceinline__ void load(const T* p, int64_t stride, uint32_t r0, uint32_t rows, uint32_t k0, uint32_t k_end) {
    if (k0 + kTileK <= k_end && (!COLUMNS || r0 + 64 * R <= rows)) return load_whole(p, stride, r0, rows, k0);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const uint32_t id = threadIdx.x + 256 * i;
      uint32_t row, column;
      int64_t valid;
      if (COLUMNS) {
        row = k0 + id / (8 * R);
        column = r0 + id % (8 * R) * 8;
        valid = row < k_end ? (int64_t)rows - column : 0;
      } else {
        row = r0 + id / 4;
        column = k0 + id % 4 * 8;
        valid = row < rows ? (int64_t)k_end - column : 0;
      }
      x[i] = load8(p + (int64_t)row * stride + column, valid);
    }
  }
  __device__ __forceinline__ void store(T* s) const {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const uint32_t id = threadIdx.x + 256 * i;
      write8(s + (COLUMNS ? id / (8 * R) * kPitch<T, true, R> + id % (8 * R) * 8 : id / 4 * kPitch<T, false, R> + id % 4 * 8), x[i]);
    }
  }
  static __device__ __forceinline__ Vec8<T> frag(const T* s, uint32_t row, uint32_t k, uint32_t lane) {
    if constexpr (COLUMNS)
      return frag_columns<false>(s, kPitch<T, true, R>, k, row, lane);
    else
      return frag_rows(s, kPitch<T, false, R>, row, k, lane);
  }
};

template <typename T, bool AC, bool BC, int R>
__global__ __launch_bounds__(256) void matmul_kernel(MatmulParams p) {
  const gts_matmul_args& a = p.a;
  typedef Staged<T, AC, R> SA;
  typedef Staged<T, BC, R> SB;
  __shared__ __align__(16) T s_a[2][kTileSize<R>], s_b[2][kTileSize<R>];
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
  const uint32_t tiles_n = (a.n + 64 * R - 1) / (64 * R);
  const uint32_t tile = blockIdx.x / p.splits, split = blockIdx.x - tile * p.splits;
  const uint32_t m0 = tile / tiles_n * 64 * R, n0 = tile % tiles_n * 64 * R;
  const uint32_t wm = wave / 2 * 32 * R, wn = wave % 2 * 32 * R;
  const uint64_t k_first = (uint64_t)split * p.k_split, k_last = k_first + p.k_split;
  const uint32_t k0 = k_first < a.k ? (uint32_t)k_first : a.k, k1 = k_last < a.k ? (uint32_t)k_last : a.k;
  f32x16 acc[R][R];
#pragma unroll
  for (int i = 0; i < R * R; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) acc[i / R][i % R][j] = 0.f;
  SA sa[2];
  SB sb[2];
  const uint32_t stages = (k1 - k0 + kTileK - 1) / kTileK;
  const auto load = [&](int set, uint32_t t) {
    sa[set].load((const T*)a.a, a.a_stride, m0, a.m, k0 + t * kTileK, k1);
    sb[set].load((const T*)a.b, a.b_stride, n0, a.n, k0 + t * kTileK, k1);
  };
  const auto store = [&](int set) {
    sa[set].store(s_a[set]);
    sb[set].store(s_b[set]);
  };
  const auto multiply = [&](int at) {
#pragma unroll
    for (uint32_t kk = 0; kk < kTileK; kk += 16) {
      Vec8<T> fa[R], fb[R];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        fa[i] = SA::frag(s_a[at], wm + i * 32, kk, lane);
        fb[i] = SB::frag(s_b[at], wn + i * 32, kk, lane);
      }
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < R; ++j) acc[i][j] = mfma(fa[i], fb[j], acc[i][j]);
    }
  };
  if (stages > 0) load(0, 0);
  if (stages > 1) load(1, 1);
  if (stages > 0) store(0);
  __syncthreads();
  uint32_t t = 0;
  if ((!AC || m0 + 64 * R <= a.m) && (!BC || n0 + 64 * R <= a.n)) {
    for (; t + 4 < stages; t += 2) {  // whole stages, whose loads are without a branch
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        sa[x].load_whole((const T*)a.a, a.a_stride, m0, a.m, k0 + (t + 2 + x) * kTileK);
        sb[x].load_whole((const T*)a.b, a.b_stride, n0, a.n, k0 + (t + 2 + x) * kTileK);
        multiply(x);
        store(x ^ 1);
        __syncthreads();
      }
    }
  }
  for (; t < stages; t += 2) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      if (t + 2 + x < stages) load(x, t + 2 + x);
      if (t + x < stages) multiply(x);
      if (t + 1 + x < stages) store(x ^ 1);
      __syncthreads();
    }
  }
  float* part = (float*)a.scratch + (uint64_t)split * a.m * a.n;
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const uint32_t n = n0 + wn + j * 32 + lane % 32;
    if (n >= a.n) continue;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const uint32_t m = m0 + wm + i * 32 + frag_row(e, lane / 32);
        if (m >= a.m) continue;
        if (p.splits > 1)
          part[(uint64_t)m * a.n + n] = acc[i][j][e];
        else
          finish<T>(a, m, n, acc[i][j][e]);
      }
  }
}

// ---- the tile kernel ---------------------------------------------------------------------
// 16-bit operands whose rows are aligned to 16 bytes.  Stages of 64 places of the sum (whole
// lines of 128 bytes) go straight to LDS, two in turn.  A stage is four matrix steps; the
// fragments of a step are read while the one before is multiplied, also across stages, and the
// one barrier of a stage stands where its last fragments have been read: there the next
// stage has arrived, and the one behind it may be loaded over this one.  Bound by matrix issue,
// which is busy 59 % of the time: 8192 x 8192 x 8192 in bfloat16 955 us with rows x rows (1151 TFLOP/s), 915
// with b by columns, 920 with both; 4096 x 4096 x 4096 123 us.  Stages of 32 places, four in turn, reached
// 1050 TFLOP/s with rows x rows where these reached 1204.
constexpr uint32_t kStage = 64;
constexpr int kSteps = kStage / 16;

__device__ __align__(16) const uint32_t g_nothing[4] = {};  // 16 bytes of zeros

// An operand's ROWS rows, 64 places a stage, loaded by W waves.  In LDS chunk c (16 bytes) of
// a row stands at c ^ swizzle, so that the reads of a fragment touch all 64 banks once.
template <typename T, bool COLUMNS, int ROWS, int W>
struct Operand {
  static constexpr int C = COLUMNS ? ROWS / 8 : 8;          // chunks of a row of LDS
  static constexpr int N = ROWS * kStage / 8 / (64 * W);    // loads of a wave
  static constexpr int SIZE = ROWS * kStage;                // values of a stage
  static_assert(ROWS * kStage / 8 % (64 * W) == 0 && (!COLUMNS || C >= 16), "whole loads");
  static __device__ __forceinline__ uint32_t swizzle(uint32_t r) {
    return COLUMNS ? ((r & 3) << 2) | ((r >> 2) & 3) : (r >> 1) & 7;
  }
  const char* base;   // of the tile's first value, the stage's first place
  int64_t step;       // bytes from a stage to the next
  uint32_t off[N];    // bytes to this lane's chunk
  uint32_t chunk[N];  // its place in the stage (rows: the first of 8)

  // Rows past the operand's end are its last ones again (whole chunks of them, if it is stored
  // by columns): what they give is not stored.
  __device__ __forceinline__ void start(const void* p, int64_t stride, uint32_t r0, uint32_t rows, uint32_t k0,
                                        uint32_t wave) {
    const uint32_t lane = threadIdx.x & 63u;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t id = (wave * N + i) * 64 + lane, r = id / C, c = id % C ^ swizzle(r);
      if constexpr (COLUMNS) {
        const uint32_t m = r0 + c * 8 + 8 <= rows ? c * 8 : rows - 8 - r0;
        off[i] = 2 * (r * (uint32_t)stride + m);
        chunk[i] = r;
      } else {
        const uint32_t m = r0 + r < rows ? r : rows - 1 - r0;
        off[i] = 2 * (m * (uint32_t)stride + c * 8);
        chunk[i] = c * 8;
      }
    }
    base = (const char*)((const T*)p + (COLUMNS ? (int64_t)k0 * stride + r0 : (int64_t)r0 * stride + k0));
    step = COLUMNS ? 2 * kStage * stride : 2 * kStage;
  }
  // left: places from the stage's first on; those past it are zeros.
  __device__ __forceinline__ void load(T* s, uint32_t wave, uint32_t left) {
    if (left >= kStage) {
#pragma unroll
      for (int i = 0; i < N; ++i) load_to_lds(base, off[i], s + (wave * N + i) * 512);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        load_to_lds(chunk[i] < left ? (const void*)(base + off[i]) : (const void*)g_nothing, s + (wave * N + i) * 512);
    }
    base += step;
  }
  // Rows row + lane % 32, places 16 kk + 8 half ..
  static __device__ __forceinline__ Vec8<T> frag(const T* s, uint32_t row, int kk, uint32_t lane) {
    if constexpr (COLUMNS) {
      typedef __attribute__((address_space(3))) i16x4* lds_t;
      const uint32_t k = kk * 16 + lane / 32 * 8 + lane % 16 / 4, c = row / 8 + lane / 16 % 2 * 2 + lane % 4 / 2;
      union {
        i16x4 h[2];
        Vec8<T> v;
      } u;
      const T* at = s + k * ROWS + lane % 2 * 4;
      u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(at + (c ^ swizzle(k)) * 8));
      u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(at + 4 * ROWS + (c ^ swizzle(k + 4)) * 8));
      return u.v;
    } else {
      const uint32_t r = row + lane % 32;
      return *(const Vec8<T>*)(s + r * kStage + ((2 * kk + lane / 32) ^ swizzle(r)) * 8);
    }
  }
};

// Eight values of a row at once; `wide`: everything is aligned to that.
template <typename T>
__device__ __forceinline__ void finish8(const gts_matmul_args& a, uint32_t m, uint32_t n, const float* zs, bool wide) {
  if (!wide) {
    for (uint32_t i = 0; i < 8 && n + i < a.n; ++i) finish<T>(a, m, n + i, zs[i]);
    return;
  }
  float z[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) z[i] = zs[i];
  if (a.bias) {
    const Pack<T, 8> b = *(const Pack<T, 8>*)((const T*)a.bias + n);
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] += (float)b.v[i];
  }
  Pack<T, 8> y;
  if (a.preact) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y.v[i] = (T)z[i];
    *(Pack<T, 8>*)((T*)a.preact + (int64_t)m * a.preact_stride + n) = y;
  }
  activate<8>(a.activation, z);
  if (a.gate) {
    const Pack<T, 8> g = *(const Pack<T, 8>*)((const T*)a.gate + (int64_t)m * a.gate_stride + n);
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] *= (float)g.v[i];
  }
  if (a.residual) {
    const Pack<T, 8> r = *(const Pack<T, 8>*)((const T*)a.residual + (int64_t)m * a.residual_stride + n);
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] += (float)r.v[i];
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) y.v[i] = (T)z[i];
  *(Pack<T, 8>*)((T*)a.out + (int64_t)m * a.out_stride + n) = y;
}

// WR x WC waves, MB x NB blocks of 32 x 32 each.
template <typename T, bool AC, bool BC, int WR, int WC, int MB, int NB>
__global__ __launch_bounds__(WR * WC * 64, 2) void tile_kernel(MatmulParams p) {
  constexpr int W = WR * WC;
  constexpr uint32_t TM = WR * MB * 32, TN = WC * NB * 32;
  typedef Operand<T, AC, TM, W> OA;
  typedef Operand<T, BC, TN, W> OB;
  constexpr int kLoads = OA::N + OB::N;
  const gts_matmul_args& a = p.a;
  __shared__ __align__(16) T s_ab[2 * (OA::SIZE + OB::SIZE)];
  const uint32_t lane = threadIdx.x & 63u, wave = uni(threadIdx.x >> 6);
  // Workgroups go round the eight XCDs: each takes a run of the tiles, in columns of eight, so
  // that those at work at one time share rows of both operands in its L2.
  const uint32_t tiles_m = (a.m + TM - 1) / TM, tiles_n = (a.n + TN - 1) / TN;
  const uint32_t xcd = blockIdx.x & 7u, share = gridDim.x / 8, extra = gridDim.x % 8;
  const uint32_t id = xcd * share + (xcd < extra ? xcd : extra) + (blockIdx.x >> 3);
  const uint32_t split = id / (tiles_m * tiles_n), tile = id - split * (tiles_m * tiles_n);
  const uint32_t band = tile / (8 * tiles_n), in = tile - band * 8 * tiles_n;
  const uint32_t height = tiles_m - band * 8 < 8 ? tiles_m - band * 8 : 8;
  const uint32_t m0 = (band * 8 + in % height) * TM, n0 = in / height * TN;
  const uint32_t wm = wave / WC * MB * 32, wn = wave % WC * NB * 32;
  const uint64_t k_first = (uint64_t)split * p.k_split;
  const uint32_t places = k_first >= a.k ? 0 : a.k - k_first < p.k_split ? (uint32_t)(a.k - k_first) : p.k_split;
  const uint32_t stages = (places + kStage - 1) / kStage;
  OA oa;
  OB ob;
  oa.start(a.a, a.a_stride, m0, a.m, (uint32_t)k_first, wave);
  ob.start(a.b, a.b_stride, n0, a.n, (uint32_t)k_first, wave);
  const auto sa = [&](uint32_t t) { return s_ab + (t & 1) * (OA::SIZE + OB::SIZE); };
  const auto load = [&](uint32_t t) {
    const uint32_t left = places - t * kStage;
    oa.load(sa(t), wave, left);
    ob.load(sa(t) + OA::SIZE, wave, left);
  };
  f32x16 acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  Vec8<T> fa[2][MB], fb[2][NB];
  const auto read = [&](uint32_t t, int kk) {
    const T* s = sa(t);
#pragma unroll
    for (int j = 0; j < NB; ++j) fb[kk & 1][j] = OB::frag(s + OA::SIZE, wn + j * 32, kk, lane);
#pragma unroll
    for (int i = 0; i < MB; ++i) fa[kk & 1][i] = OA::frag(s, wm + i * 32, kk, lane);
  };
  const auto multiply = [&](int kk) {
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = mfma(fa[kk & 1][i], fb[kk & 1][j], acc[i][j]);
  };
  if (stages) load(0);
  if (stages > 1) {
    load(1);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
  } else {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");  // no read of LDS moves before the barrier
  if (stages) read(0, 0);
  for (uint32_t t = 0; t < stages; ++t) {
#pragma unroll
    for (int kk = 0; kk < kSteps; ++kk) {
      if (kk + 1 < kSteps) {
        read(t, kk + 1);
      } else {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (t + 2 < stages) load(t + 2);
        if (t + 1 < stages) read(t + 1, 0);
      }
      multiply(kk);
    }
  }
  // Results: through LDS, a block of 32 rows of the wave at a time, so that whole rows are
  // written (and gate and residual read).
  constexpr uint32_t P = NB * 32 + 4;
  static_assert(W * 32 * P * 4 <= sizeof(s_ab), "the results fit the stages' LDS");
  __syncthreads();
  float* s = (float*)s_ab + wave * 32 * P;
  float* part = (float*)a.scratch + (uint64_t)split * a.m * a.n;
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    asm volatile("" ::: "memory");  // a wave's accesses to LDS keep their order
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[frag_row(e, lane / 32) * P + j * 32 + lane % 32] = acc[i][j][e];
    asm volatile("" ::: "memory");
#pragma unroll 1
    for (int x = 0; x < NB * 2; ++x) {
      const uint32_t at = x * 64 + lane, r = at / (NB * 4), c = at % (NB * 4) * 8;
      const uint32_t m = m0 + wm + i * 32 + r, n = n0 + wn + c;
      if (m >= a.m || n >= a.n) continue;
      float z[8];
      *(f32x4*)z = *(const f32x4*)(s + r * P + c);
      *(f32x4*)(z + 4) = *(const f32x4*)(s + r * P + c + 4);
      if (p.splits > 1) {
        float* to = part + (uint64_t)m * a.n + n;
        if (a.n % 8 == 0) {
          *(f32x4*)to = *(const f32x4*)z;
          *(f32x4*)(to + 4) = *(const f32x4*)(z + 4);
        } else {
          for (uint32_t y = 0; y < 8 && n + y < a.n; ++y) to[y] = z[y];
        }
      } else {
        finish8<T>(a, m, n, z, p.wide);
      }
    }
  }
}

// The sums of the splits, in order; eight values of a row a thread.
template <typename T>
__global__ __launch_bounds__(256) void join_splits_kernel(MatmulParams p) {
  const gts_matmul_args& a = p.a;
  const uint32_t per = (a.n + 7) / 8;
  const uint64_t i = block_number() * 256 + threadIdx.x, all = (uint64_t)a.m * a.n;
  if (i >= (uint64_t)a.m * per) return;
  const uint32_t m = (uint32_t)(i / per), n = (uint32_t)(i - (uint64_t)m * per) * 8;
  const float* part = (const float*)a.scratch + (uint64_t)m * a.n + n;
  float z[8] = {};
  if (a.n % 8 == 0) {
    for (uint32_t s = 0; s < p.splits; ++s)
#pragma unroll
      for (int x = 0; x < 8; x += 4) {
        const f32x4 y = *(const f32x4*)(part + s * all + x);
#pragma unroll
        for (int e = 0; e < 4; ++e) z[x + e] += y[e];
      }
  } else {
    for (uint32_t s = 0; s < p.splits; ++s)
      for (uint32_t x = 0; x < 8 && n + x < a.n; ++x) z[x] += part[s * all + x];
  }
  finish8<T>(a, m, n, z, p.wide);
}

// ---- few rows ----------------------------------------------------------------------------
// Up to 16 rows of a: the rows of b are streamed through registers, each read once, 16 of
// them a workgroup; its four waves take 64 places of the sum in turn and join their sums in
// LDS: one launch where the tiles take two.  Bound by the loads of b (16 rows at a time: 3.5 TB/s);
// a comes from the L2s.  3 x 1024 x 1024 4.2 us (tiles with splits 7.4), 1 x 4096 x 4096 7.1 (11.1),
// 8 x 6144 x 4096 14.4 (14.6); past 2^25 values of b the tiles are faster (16 x 4096 x 14336 27.0, 25.1).
constexpr uint64_t kFewValues = 1ull << 25;
constexpr uint32_t kFew = 16;
constexpr int kAhead = 4;  // steps of 64 places whose loads are on their way together

__device__ __forceinline__ f32x4 mfma16(Vec8<__bf16> a, Vec8<__bf16> b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(Vec8<_Float16> a, Vec8<_Float16> b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

template <typename T>
__global__ __launch_bounds__(256) void few_kernel(MatmulParams p) {
  const gts_matmul_args& a = p.a;
  constexpr uint32_t W = 4;
  __shared__ __align__(16) float s_sum[W][16][20];
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, r = lane % 16, quarter = lane / 16;
  const uint32_t n0 = blockIdx.x * 16;
  // rows past the end are the last again: what they give is not stored
  const T* pa = (const T*)a.a + (int64_t)(r < a.m ? r : a.m - 1) * a.a_stride;
  const T* pb = (const T*)a.b + (int64_t)(n0 + r < a.n ? n0 + r : a.n - 1) * a.b_stride;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  const uint32_t steps = (a.k + 63) / 64;
  // 16 bytes of a row at step s, half x of its places; zeros behind the end
  const auto at = [&](const T* row, uint32_t s, int x) {
    const uint64_t k = (uint64_t)s * 64 + x * 32 + quarter * 8;
    return *(const Vec8<T>*)(k < a.k ? row + k : (const T*)g_nothing);
  };
  Vec8<T> fa[2][kAhead][2], fb[2][kAhead][2];
  const auto load = [&](int to, uint32_t s) {
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        fa[to][y][x] = at(pa, s + y * W, x);
        fb[to][y][x] = at(pb, s + y * W, x);
      }
    __builtin_amdgcn_sched_barrier(0);  // the loads stay ahead of the products
  };
  const auto multiply = [&](int from) {
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
#pragma unroll
      for (int x = 0; x < 2; ++x) acc = mfma16(fb[from][y][x], fa[from][y][x], acc);
  };
  // loads past the end are of 16 bytes that are in every L2
  load(0, wave);
  for (uint32_t s = wave; s < steps; s += 2 * kAhead * W) {
    load(1, s + kAhead * W);
    multiply(0);
    load(0, s + 2 * kAhead * W);
    multiply(1);
  }
  // a lane has row r of a, and four rows of b side by side
  *(f32x4*)&s_sum[wave][r][quarter * 4] = acc;
  __syncthreads();
  if (threadIdx.x < 32) {
    const uint32_t m = threadIdx.x / 2, c = threadIdx.x % 2 * 8;
    if (m >= a.m || n0 + c >= a.n) return;
    float z[8] = {};
#pragma unroll
    for (uint32_t w = 0; w < W; ++w)
#pragma unroll
      for (int x = 0; x < 8; ++x) z[x] += s_sum[w][m][c + x];
    finish8<T>(a, m, n0 + c, z, p.wide);
  }
}

uint64_t size(int64_t x) { return (uint64_t)(x < 0 ? -x : x); }
bool rows_aligned(const void* p, int64_t stride, uint32_t e) {
  return (uintptr_t)p % 16 == 0 && size(stride) * e % 16 == 0;
}

// How a product is cut: its tile, and the splits of its sum.  By sizes alone: the scratch is
// asked for before the layout is known.
struct Cut {
  uint32_t tile;  // of kCuts
  uint32_t splits;
};
// Microseconds that a stage of 64 places takes: a workgroup alone on its CU, and what each adds
// where several share one (or take turns).  Fitted to products of 64 to 8192 rows and columns with
// 1024 to 14336 places.
struct TileCost {
  uint32_t m, n;
  float alone, shared;
};
constexpr TileCost kCuts[] = {
    // the tile kernel
    {256, 256, 1.45f, 1.6f},
    {256, 128, 0.9f, 0.98f},
    {128, 128, 0.72f, 0.52f},
    {64, 128, 0.56f, 0.33f},
    // the general kernel, and in 32 bits: a sixteenth of the matrix rate
    {128, 128, 1.6f, 0.9f},
    {64, 64, 1.0f, 0.35f},
    {128, 128, 6.0f, 4.4f},
    {64, 64, 1.75f, 1.2f}};
constexpr uint32_t kUnits = 256;  // CUs
// A launch with a workgroup's begin and end, the join's, a byte of the parts written and read.
constexpr float kBegin = 4.f, kJoin = 4.f, kPartBytes = 1.f / 2.4e6f;

float cost_of(const TileCost& c, uint32_t m, uint32_t n, uint32_t k, uint32_t splits) {
  const uint64_t tiles = (uint64_t)((m + c.m - 1) / c.m) * ((n + c.n - 1) / c.n);
  const uint64_t groups = tiles * splits;
  if (groups > kMostGroups) return INFINITY;  // never tiles of 128 x 128 in one split: the sizes were checked for them
  const float shared = c.shared * (groups < kUnits ? (float)groups / kUnits : (float)((groups + kUnits - 1) / kUnits));
  const uint32_t stages = ((k + 63) / 64 + splits - 1) / splits;
  const float join = splits > 1 ? kJoin + kPartBytes * 4.f * splits * (float)m * (float)n : 0.f;
  return kBegin + (float)stages * (shared > c.alone ? shared : c.alone) + join;
}
// kLargeTiles: a is stored by columns, of which a tile has 128 at least.
enum Kind { kGeneral, kTiles, kLargeTiles, kGeneral32 };
Cut cut_of(uint32_t m, uint32_t n, uint32_t k, Kind kind) {
  const uint32_t from = kind == kGeneral ? 4 : kind == kGeneral32 ? 6 : 0;
  const uint32_t to = kind == kGeneral ? 6 : kind == kGeneral32 ? 8 : kind == kTiles ? 4 : 3;
  Cut best{from, 1};
  float least = INFINITY;
  for (uint32_t t = from; t < to; ++t)
    for (const uint32_t splits : {1u, 2u, 3u, 4u, 6u, 8u, 12u, 16u, 24u, 32u}) {
      if (splits > 1 && splits * 128 > k) break;
      const float c = cost_of(kCuts[t], m, n, k, splits);
      if (c < least) {
        least = c;
        best = {t, splits};
      }
    }
  return best;
}
uint64_t parts_bytes(uint32_t m, uint32_t n, uint32_t splits) { return splits > 1 ? 4ull * splits * m * n : 0; }

// An operand's stages as the tile kernel loads them: 16 bytes at a time, whole chunks, a tile's
// offsets in 32 bits.
bool fits_tiles(const void* p, int64_t stride, uint32_t rows, uint32_t k, bool columns) {
  return rows_aligned(p, stride, 2) && stride >= 0 && stride < 1 << 22 && (columns ? rows : k) % 8 == 0;
}

template <typename T>
void launch_join(const MatmulParams& p, hipStream_t s) {
  const uint64_t all = (uint64_t)p.a.m * ((p.a.n + 7) / 8);
  join_splits_kernel<T><<<grid_of((all + 255) / 256), dim3(256), 0, s>>>(p);
}

template <typename T, bool AC, bool BC, int WR, int WC, int MB, int NB>
void launch_tiles(const MatmulParams& p, hipStream_t s) {
  const gts_matmul_args& a = p.a;
  constexpr uint32_t TM = WR * MB * 32, TN = WC * NB * 32;
  const uint64_t tiles = (uint64_t)((a.m + TM - 1) / TM) * ((a.n + TN - 1) / TN);
  tile_kernel<T, AC, BC, WR, WC, MB, NB><<<dim3((uint32_t)(tiles * p.splits)), dim3(WR * WC * 64), 0, s>>>(p);
}

template <typename T, bool AC, bool BC>
hipError_t launch_layout(MatmulParams& p, hipStream_t s) {
  const gts_matmul_args& a = p.a;
  if constexpr (sizeof(T) == 2) {
    if (fits_tiles(a.a, a.a_stride, a.m, a.k, AC) && fits_tiles(a.b, a.b_stride, a.n, a.k, BC)) {
      if constexpr (!AC && !BC) {
        if (a.m <= kFew && (uint64_t)a.n * a.k <= kFewValues) {
          few_kernel<T><<<dim3((a.n + 15) / 16), dim3(256), 0, s>>>(p);
          return hipGetLastError();
        }
      }
      const Cut cut = cut_of(a.m, a.n, a.k, AC ? kLargeTiles : kTiles);
      p.splits = cut.splits;
      p.k_split = ((a.k + p.splits - 1) / p.splits + kStage - 1) / kStage * kStage;
      if (cut.tile == 0)
        launch_tiles<T, AC, BC, 2, 4, 4, 2>(p, s);
      else if (cut.tile == 1)
        launch_tiles<T, AC, BC, 4, 2, 2, 2>(p, s);
      else if (cut.tile == 2)
        launch_tiles<T, AC, BC, 2, 2, 2, 2>(p, s);
      else if constexpr (!AC)
        launch_tiles<T, AC, BC, 1, 4, 2, 1>(p, s);
      if (p.splits > 1) launch_join<T>(p, s);
      return hipGetLastError();
    }
  }
  const Cut cut = cut_of(a.m, a.n, a.k, sizeof(T) == 4 ? kGeneral32 : kGeneral);
  p.splits = cut.splits;
  p.k_split = ((a.k + p.splits - 1) / p.splits + kTileK - 1) / kTileK * kTileK;
  const uint32_t edge = kCuts[cut.tile].m;
  const uint64_t groups = (((uint64_t)a.m + edge - 1) / edge) * (((uint64_t)a.n + edge - 1) / edge) * p.splits;
  if (edge == 128)
    matmul_kernel<T, AC, BC, 2><<<dim3((uint32_t)groups), dim3(256), 0, s>>>(p);
  else
    matmul_kernel<T, AC, BC, 1><<<dim3((uint32_t)groups), dim3(256), 0, s>>>(p);
  if (p.splits > 1) launch_join<T>(p, s);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_matmul_t(const gts_matmul_args& a, hipStream_t s) {
  MatmulParams p{};
  p.a = a;
  p.wide = a.n % 8 == 0 && rows_aligned(a.out, a.out_stride, sizeof(T)) &&
           rows_aligned(a.preact, a.preact ? a.preact_stride : 0, sizeof(T)) &&
           rows_aligned(a.gate, a.gate ? a.gate_stride : 0, sizeof(T)) &&
           rows_aligned(a.residual, a.residual ? a.residual_stride : 0, sizeof(T)) && (uintptr_t)a.bias % 16 == 0;
  const bool ac = a.flags & GTS_MATMUL_A_COLUMNS, bc = a.flags & GTS_MATMUL_B_COLUMNS;
  if (ac) return bc ? launch_layout<T, true, true>(p, s) : launch_layout<T, true, false>(p, s);
  return bc ? launch_layout<T, false, true>(p, s) : launch_layout<T, false, false>(p, s);
}

// ---- the elementwise part of the gradient ------------------------------------------------
// A wave takes 64 V columns of a strip of rows, and keeps its part of dbias in registers.  Two rows are
// on their way at a time; bound by HBM (2048 x 14336 with silu and gate in bfloat16, 294 MB: 55 us, 5.3 TB/s).
struct LinearGradParams {
  gts_linear_grad_args a;
  float* db;  // [strips][n], NULL if not wanted
  uint32_t strips;
};

template <typename T, int V, uint32_t ACT>
__global__ __launch_bounds__(256) void linear_grad_kernel(LinearGradParams p) {
  const gts_linear_grad_args& a = p.a;
  const uint32_t strip = blockIdx.y * 4 + (threadIdx.x >> 6);
  const uint64_t at = ((uint64_t)blockIdx.x * 64 + (threadIdx.x & 63u)) * V;
  if (strip >= p.strips || at >= a.n) return;
  float db[V] = {};
  constexpr int R = 2;  // rows whose loads are on their way together
  for (uint64_t m0 = strip; m0 < a.m; m0 += (uint64_t)R * p.strips) {
    Pack<T, V> dy[R], z[R] = {}, g[R] = {};
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const uint64_t m = m0 + (uint64_t)k * p.strips;
      if (m >= a.m) break;
      dy[k] = *(const Pack<T, V>*)((const T*)a.dy + (int64_t)m * a.dy_stride + at);
      if (a.preact) z[k] = *(const Pack<T, V>*)((const T*)a.preact + (int64_t)m * a.preact_stride + at);
      if (a.gate) g[k] = *(const Pack<T, V>*)((const T*)a.gate + (int64_t)m * a.gate_stride + at);
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const uint64_t m = m0 + (uint64_t)k * p.strips;
      if (m >= a.m) break;
      Pack<T, V> dg, dz;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float d = (float)dy[k].v[i];
        const Shape at_z = shape_of<ACT>((float)z[k].v[i]);
        if (a.dgate) dg.v[i] = (T)(d * at_z.y);
        if (a.gate) d *= (float)g[k].v[i];
        if constexpr (ACT != GTS_ACT_NONE) d *= at_z.slope;
        dz.v[i] = (T)d;
        db[i] += d;
      }
      if (a.dz) *(Pack<T, V>*)((T*)a.dz + (int64_t)m * a.dz_stride + at) = dz;
      if (a.dgate) *(Pack<T, V>*)((T*)a.dgate + (int64_t)m * a.dgate_stride + at) = dg;
    }
  }
  if (p.db) {
#pragma unroll
    for (int i = 0; i < V; ++i) p.db[(uint64_t)strip * a.n + at + i] = db[i];
  }
}

// Strips of rows: 16 rows each, but no more than keep the chip busy, so that the parts
// of dbias stay small beside the rows.
uint32_t strips_of(uint32_t m, uint32_t n) {
  const uint64_t waves = ((uint64_t)n + 511) / 512;
  uint64_t most = 16384 / (waves ? waves : 1);
  if (most < 16) most = 16;
  const uint64_t want = ((uint64_t)m + 15) / 16;
  return (uint32_t)(want < 1 ? 1 : want < most ? want : most);
}

template <typename T>
void launch_linear_grad_t(const LinearGradParams& p, hipStream_t s) {
  constexpr uint32_t V = 16 / sizeof(T);
  const gts_linear_grad_args& a = p.a;
  const bool wide = a.n % V == 0 && rows_aligned(a.dy, a.dy_stride, sizeof(T)) &&
                    rows_aligned(a.preact, a.preact ? a.preact_stride : 0, sizeof(T)) &&
                    rows_aligned(a.gate, a.gate ? a.gate_stride : 0, sizeof(T)) &&
                    rows_aligned(a.dz, a.dz ? a.dz_stride : 0, sizeof(T)) &&
                    rows_aligned(a.dgate, a.dgate ? a.dgate_stride : 0, sizeof(T));
  const uint32_t v = wide ? V : 1;
  const dim3 grid((uint32_t)(((uint64_t)a.n + 64 * v - 1) / (64 * v)), (p.strips + 3) / 4);
  const auto launch = [&](auto act) {
    constexpr uint32_t A = decltype(act)::value;
    if (wide)
      linear_grad_kernel<T, V, A><<<grid, dim3(256), 0, s>>>(p);
    else
      linear_grad_kernel<T, 1, A><<<grid, dim3(256), 0, s>>>(p);
  };
  switch (a.activation) {
    case GTS_ACT_RELU: return launch(std::integral_constant<uint32_t, GTS_ACT_RELU>{});
    case GTS_ACT_GELU: return launch(std::integral_constant<uint32_t, GTS_ACT_GELU>{});
    case GTS_ACT_GELU_TANH: return launch(std::integral_constant<uint32_t, GTS_ACT_GELU_TANH>{});
    case GTS_ACT_SILU: return launch(std::integral_constant<uint32_t, GTS_ACT_SILU>{});
    default: return launch(std::integral_constant<uint32_t, GTS_ACT_NONE>{});
  }
}

}  // namespace

uint64_t matmul_scratch(uint32_t m, uint32_t n, uint32_t k) {
  uint32_t most = 1;
  for (const Kind kind : {kGeneral, kTiles, kLargeTiles, kGeneral32}) {
    const uint32_t splits = cut_of(m, n, k, kind).splits;
    most = splits > most ? splits : most;
  }
  return parts_bytes(m, n, most);
}

hipError_t launch_matmul(const gts_matmul_args& a, hipStream_t s) {
  if (a.dtype == GTS_F32) return launch_matmul_t<float>(a, s);
  if (a.dtype == GTS_BF16) return launch_matmul_t<__bf16>(a, s);
  return launch_matmul_t<_Float16>(a, s);
}

uint64_t linear_grad_scratch(uint32_t m, uint32_t n) { return 4ull * strips_of(m, n) * n; }

hipError_t launch_linear_grad(const gts_linear_grad_args& a, hipStream_t s) {
  LinearGradParams p{a, a.dbias ? (float*)a.scratch : nullptr, strips_of(a.m, a.n)};
  if (a.dtype == GTS_F32)
    launch_linear_grad_t<float>(p, s);
  else if (a.dtype == GTS_BF16)
    launch_linear_grad_t<__bf16>(p, s);
  else
    launch_linear_grad_t<_Float16>(p, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_column_sums(p.db, a.dbias, nullptr, nullptr, p.strips, a.n, a.dtype, s);
}

}  // namespace gts
