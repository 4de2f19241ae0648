// gts_norm.hip — layer norm over rows, centered or not, and its gradient.
//
//   forward   mu = mean(x) (0 without centering), r = 1 / sqrt(mean((x - mu)^2) + eps),
//             h = (x - mu) r,  y = h w + b
//   backward  g = dy w,  dx = r (g - mean(g) - h mean(g h)) (no mean(g) without
//             centering),  dw = sum_rows(dy h),  db = sum_rows(dy)
//
// A row belongs to a team: 16 lanes, a wave, four or eight, the fewest whose registers hold it
// (16 values a lane, or 32), so x is read once and the variance is of the differences, not a
// difference of sums.  Longer rows are read again from memory for each pass over them.
// Bound by HBM when large (32768 rows of 4096 in bfloat16: 4.9 TB/s forward, 5.1 backward) and by
// the launch when small.
#include "gts_ops.h"
#include "gts_tile.h"

namespace gts {
namespace {

constexpr int kHeld = 32;                   // values of a row that a lane holds
constexpr uint32_t kLongest = 512 * kHeld;  // longest row that a team holds

// Sums over a team of L lanes; every lane gets them.  s: one slot a wave and sum, twice, used in
// turn so that one barrier a call is enough.
template <int L>
struct Team {
  static constexpr int W = L / 64;
  float (*s)[2][16];
  uint32_t turn = 0;
  __device__ __forceinline__ static float lanes_sum(float x) {
#pragma unroll
    for (int k = L < 64 ? L / 2 : 32; k; k >>= 1) x += __shfl_xor(x, k);
    return x;
  }
  __device__ __forceinline__ void sum2(float& a, float& b) {
    a = lanes_sum(a);
    b = lanes_sum(b);
    if constexpr (W > 1) {
      float(*t)[16] = s[turn & 1];
      ++turn;
      const uint32_t wave = threadIdx.x >> 6;
      if ((threadIdx.x & 63u) == 0) {
        t[0][wave] = a;
        t[1][wave] = b;
      }
      __syncthreads();
      a = b = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        a += t[0][i];
        b += t[1][i];
      }
    }
  }
  __device__ __forceinline__ float sum(float a) {
    float b = 0.f;
    sum2(a, b);
    return a;
  }
};

template <int L>
constexpr int kThreads = L < 256 ? 256 : L;
template <int L>
constexpr int kTeams = kThreads<L> / L;

// V values of a row, loaded and stored at any alignment.
template <typename T, int V>
struct __attribute__((packed, aligned(sizeof(T)))) Anywhere {
  T v[V];
};
// A lane's c-th access to a row: V values from column `at` on.  WHOLE: V divides the row.  Else
// the last access of a row reaches back over `skip` values that are another lane's: they are left
// out of sums, and stored by both.
template <typename T, int V, int L, bool WHOLE>
struct Access {
  uint32_t at, skip;
  bool in;
  __device__ __forceinline__ Access(int c, uint32_t lane, uint32_t dim) : at((c * L + lane) * V), skip(0), in(at < dim) {
    if (!WHOLE && in && at + V > dim) {
      skip = at + V - dim;
      at -= skip;
    }
  }
  __device__ __forceinline__ Anywhere<T, V> load(const T* row) const {
    Anywhere<T, V> x = {};
    if (in) x = *reinterpret_cast<const Anywhere<T, V>*>(row + at);
    return x;
  }
  __device__ __forceinline__ void store(T* row, const Anywhere<T, V>& x) const {
    if (in) *reinterpret_cast<Anywhere<T, V>*>(row + at) = x;
  }
  // Whether value i is the lane's own (one outside the row is zero).
  __device__ __forceinline__ bool own(int i) const { return WHOLE || i >= (int)skip; }
};

template <typename T, int V, int L, int C, bool WHOLE>
__global__ __launch_bounds__(kThreads<L>) void norm_kernel(gts_norm_args a) {
  __shared__ float s_sum[2][2][16];
  Team<L> team{s_sum};
  const uint32_t lane = threadIdx.x % L;
  const uint64_t row = block_number<kThreads<L>>() * kTeams<L> + threadIdx.x / L;
  if (row >= a.rows) return;
  const bool center = a.flags & GTS_NORM_CENTER;
  const T* x = (const T*)a.x + (int64_t)row * a.x_stride;
  const float n = 1.f / (float)a.dim;
  Anywhere<T, V> v[C];
#pragma unroll
  for (int c = 0; c < C; ++c) v[c] = Access<T, V, L, WHOLE>(c, lane, a.dim).load(x);
  float mu = 0.f;
  if (center) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Access<T, V, L, WHOLE> at(c, lane, a.dim);
#pragma unroll
      for (int i = 0; i < V; ++i) mu += at.own(i) ? (float)v[c].v[i] : 0.f;
    }
    mu = team.sum(mu) * n;
  }
  float q = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const Access<T, V, L, WHOLE> at(c, lane, a.dim);
    if (!at.in) continue;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float d = at.own(i) ? (float)v[c].v[i] - mu : 0.f;
      q += d * d;
    }
  }
  const float r = 1.f / sqrtf(team.sum(q) * n + a.eps);
  if (lane == 0) {
    if (a.mean) a.mean[row] = mu;
    if (a.rstd) a.rstd[row] = r;
  }
  T* y = (T*)a.out + (int64_t)row * a.out_stride;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const Access<T, V, L, WHOLE> at(c, lane, a.dim);
    if (!at.in) continue;
    Anywhere<T, V> w = {}, b = {}, o;
    if (a.weight) w = at.load((const T*)a.weight);
    if (a.bias) b = at.load((const T*)a.bias);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float h = ((float)v[c].v[i] - mu) * r;
      if (a.weight) h *= (float)w.v[i];
      if (a.bias) h += (float)b.v[i];
      o.v[i] = (T)h;
    }
    at.store(y, o);
  }
}

// Rows of any other length: three passes over memory, sums of a thread in order.
template <typename T>
__global__ __launch_bounds__(1024) void norm_long_kernel(gts_norm_args a) {
  __shared__ float s_sum[2][2][16];
  Team<1024> team{s_sum};
  const uint64_t row = block_number<1024>();
  if (row >= a.rows) return;
  const T* x = (const T*)a.x + (int64_t)row * a.x_stride;
  T* y = (T*)a.out + (int64_t)row * a.out_stride;
  float mu = 0.f, q = 0.f;
  if (a.flags & GTS_NORM_CENTER) {
    for (uint32_t i = threadIdx.x; i < a.dim; i += 1024) mu += (float)x[i];
    mu = team.sum(mu) / (float)a.dim;
  }
  for (uint32_t i = threadIdx.x; i < a.dim; i += 1024) {
    const float d = (float)x[i] - mu;
    q += d * d;
  }
  const float r = 1.f / sqrtf(team.sum(q) / (float)a.dim + a.eps);
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[row] = mu;
    if (a.rstd) a.rstd[row] = r;
  }
  for (uint32_t i = threadIdx.x; i < a.dim; i += 1024) {
    float h = ((float)x[i] - mu) * r;
    if (a.weight) h *= (float)((const T*)a.weight)[i];
    if (a.bias) h += (float)((const T*)a.bias)[i];
    y[i] = (T)h;
  }
}

// The gradient.  A team takes every (gridDim.x x teams)-th row and keeps its part of dw and db in
// registers: columns of a lane are the same in every row.  The teams of a workgroup join theirs in
// LDS; the parts, one row of scratch a workgroup, are added up in order by column_sums_kernel.
struct NormGradParams {
  gts_norm_grad_args a;
  float *dw, *db;  // [groups][dim], NULL if not wanted
};

template <typename T, int V, int L, int C, bool WHOLE>
__global__ __launch_bounds__(kThreads<L>) void norm_grad_kernel(NormGradParams p) {
  __shared__ float s_sum[2][2][16];
  const gts_norm_grad_args& a = p.a;
  Team<L> team{s_sum};
  const uint32_t lane = threadIdx.x % L, mine = threadIdx.x / L;
  const float n = 1.f / (float)a.dim;
  const bool center = a.flags & GTS_NORM_CENTER;
  float dw[C][V] = {}, db[C][V] = {};
  Anywhere<T, V> w[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (a.weight) {
      w[c] = Access<T, V, L, WHOLE>(c, lane, a.dim).load((const T*)a.weight);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) w[c].v[i] = (T)1.f;
    }
  }
  // The next row is on its way while a row's sums are taken (32768 rows of 4096 in bfloat16: 252
  // us without, 168 with).
  Anywhere<T, V> xv[C], dv[C];
  float mu = 0.f, r = 0.f;
  const uint64_t step = (uint64_t)gridDim.x * kTeams<L>;
  const auto load = [&](uint64_t row) {
    const T* x = (const T*)a.x + (int64_t)row * a.x_stride;
    const T* dy = (const T*)a.dy + (int64_t)row * a.dy_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Access<T, V, L, WHOLE> at(c, lane, a.dim);
      xv[c] = at.load(x);
      dv[c] = at.load(dy);
    }
    mu = center ? a.mean[row] : 0.f;
    r = a.rstd[row];
  };
  uint64_t row = (uint64_t)blockIdx.x * kTeams<L> + mine;
  if (row < a.rows) load(row);
  for (; row < a.rows; row += step) {
    float h[C][V], g[C][V], sg = 0.f, sgh = 0.f;
    const float rs = r;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Access<T, V, L, WHOLE> at(c, lane, a.dim);
      if (!at.in) continue;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = (float)dv[c].v[i];
        h[c][i] = ((float)xv[c].v[i] - mu) * r;
        g[c][i] = d * (float)w[c].v[i];
        if (at.own(i)) {
          sg += g[c][i];
          sgh += g[c][i] * h[c][i];
        }
        dw[c][i] += d * h[c][i];
        db[c][i] += d;
      }
    }
    if (row + step < a.rows) load(row + step);
    team.sum2(sg, sgh);
    const float mg = center ? sg * n : 0.f, mgh = sgh * n;
    if (!a.dx) continue;
    T* dx = (T*)a.dx + (int64_t)row * a.dx_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Access<T, V, L, WHOLE> at(c, lane, a.dim);
      if (!at.in) continue;
      Anywhere<T, V> o;
#pragma unroll
      for (int i = 0; i < V; ++i) o.v[i] = (T)((g[c][i] - mg - h[c][i] * mgh) * rs);
      at.store(dx, o);
    }
  }
  const uint64_t part = (uint64_t)blockIdx.x * a.dim;
  if constexpr (kTeams<L> == 1) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const Access<T, V, L, WHOLE> at(c, lane, a.dim);
      if (!at.in) continue;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (!at.own(i)) continue;
        if (p.dw) p.dw[part + at.at + i] = dw[c][i];
        if (p.db) p.db[part + at.at + i] = db[c][i];
      }
    }
  } else {
    __shared__ float s_part[kTeams<L>][C * L * V];
    for (int which = 0; which < 2; ++which) {
      float* to = which ? p.db : p.dw;
      if (!to) continue;
      __syncthreads();
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const Access<T, V, L, WHOLE> at(c, lane, a.dim);
        if (!at.in) continue;
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (at.own(i)) s_part[mine][at.at + i] = which ? db[c][i] : dw[c][i];
      }
      __syncthreads();
      for (uint32_t at = threadIdx.x; at < a.dim; at += kThreads<L>) {
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < kTeams<L>; ++t) sum += s_part[t][at];
        to[part + at] = sum;
      }
    }
  }
}

// Rows of any length.  dw and db: a column's sum over a strip of rows.
template <typename T>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(gts_norm_grad_args a) {
  __shared__ float s_sum[2][2][16];
  Team<1024> team{s_sum};
  const uint64_t row = block_number<1024>();
  if (row >= a.rows) return;
  const T* x = (const T*)a.x + (int64_t)row * a.x_stride;
  const T* dy = (const T*)a.dy + (int64_t)row * a.dy_stride;
  T* dx = (T*)a.dx + (int64_t)row * a.dx_stride;
  const bool center = a.flags & GTS_NORM_CENTER;
  const float mu = center ? a.mean[row] : 0.f, r = a.rstd[row];
  float sg = 0.f, sgh = 0.f;
  for (uint32_t i = threadIdx.x; i < a.dim; i += 1024) {
    const float g = (float)dy[i] * (a.weight ? (float)((const T*)a.weight)[i] : 1.f);
    sg += g;
    sgh += g * (((float)x[i] - mu) * r);
  }
  team.sum2(sg, sgh);
  const float mg = center ? sg / (float)a.dim : 0.f, mgh = sgh / (float)a.dim;
  for (uint32_t i = threadIdx.x; i < a.dim; i += 1024) {
    const float g = (float)dy[i] * (a.weight ? (float)((const T*)a.weight)[i] : 1.f);
    dx[i] = (T)((g - mg - ((float)x[i] - mu) * r * mgh) * r);
  }
}
template <typename T>
__global__ __launch_bounds__(256) void norm_columns_kernel(NormGradParams p) {
  const gts_norm_grad_args& a = p.a;
  const uint32_t at = blockIdx.x * 256 + threadIdx.x;
  if (at >= a.dim) return;
  const bool center = a.flags & GTS_NORM_CENTER;
  float dw = 0.f, db = 0.f;
  for (uint64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const float d = (float)((const T*)a.dy)[(int64_t)row * a.dy_stride + at];
    const float x = (float)((const T*)a.x)[(int64_t)row * a.x_stride + at];
    dw += d * ((x - (center ? a.mean[row] : 0.f)) * a.rstd[row]);
    db += d;
  }
  if (p.dw) p.dw[(uint64_t)blockIdx.y * a.dim + at] = dw;
  if (p.db) p.db[(uint64_t)blockIdx.y * a.dim + at] = db;
}

// The team of a row: the fewest lanes whose registers hold it, with 16 values a lane (16 or 64 lanes) or 32.
template <int L>
constexpr uint32_t kMost = L < 256 ? L * kHeld / 2 : L * kHeld;  // values of a row
static_assert(kMost<512> == kLongest, "the largest team holds the longest row");
uint32_t lanes_of(uint32_t dim) { return dim <= kMost<16> ? 16 : dim <= kMost<64> ? 64 : dim <= kMost<256> ? 256 : 512; }

// The accesses of 16 bytes that each lane makes.  Shorter rows (up to `below`) have a smaller team.
template <template <typename, int, int, int> class K, typename T, int L, typename P>
void launch_lanes(const P& p, uint32_t dim, uint32_t groups, hipStream_t s) {
  constexpr int V = 16 / sizeof(T), C = kHeld / V;
  constexpr uint32_t below = L == 16 ? 0 : L == 64 ? kMost<16> : L == 256 ? kMost<64> : kMost<256>;
  if constexpr (below < L * kHeld / 4)
    if (dim <= L * kHeld / 4) return K<T, V, L, C / 4>::go(p, groups, s);
  if constexpr (below < L * kHeld / 2)
    if (dim <= L * kHeld / 2) return K<T, V, L, C / 2>::go(p, groups, s);
  if constexpr (kMost<L> > L * kHeld / 2) K<T, V, L, C>::go(p, groups, s);
}
// Rows that teams take: neither longer than they hold nor shorter than an access.
template <typename T>
bool held(uint32_t dim) {
  return dim <= kLongest && dim >= 16 / sizeof(T);
}
template <template <typename, int, int, int> class K, typename T, typename P>
void launch_team(const P& p, uint32_t dim, uint32_t groups, hipStream_t s) {
  switch (lanes_of(dim)) {
    case 16: return launch_lanes<K, T, 16>(p, dim, groups, s);
    case 64: return launch_lanes<K, T, 64>(p, dim, groups, s);
    case 256: return launch_lanes<K, T, 256>(p, dim, groups, s);
    default: return launch_lanes<K, T, 512>(p, dim, groups, s);
  }
}
template <typename T, int V, int L, int C>
struct Forward {
  static void go(const gts_norm_args& a, uint32_t, hipStream_t s) {
    const dim3 grid = grid_of<kThreads<L>>(((uint64_t)a.rows + kTeams<L> - 1) / kTeams<L>);
    if (a.dim % V == 0)
      norm_kernel<T, V, L, C, true><<<grid, dim3(kThreads<L>), 0, s>>>(a);
    else
      norm_kernel<T, V, L, C, false><<<grid, dim3(kThreads<L>), 0, s>>>(a);
  }
};
template <typename T, int V, int L, int C>
struct Gradient {
  static void go(const NormGradParams& p, uint32_t groups, hipStream_t s) {
    if (p.a.dim % V == 0)
      norm_grad_kernel<T, V, L, C, true><<<dim3(groups), dim3(kThreads<L>), 0, s>>>(p);
    else
      norm_grad_kernel<T, V, L, C, false><<<dim3(groups), dim3(kThreads<L>), 0, s>>>(p);
  }
};

template <typename T>
void launch_norm_t(const gts_norm_args& a, hipStream_t s) {
  if (!held<T>(a.dim))
    norm_long_kernel<T><<<grid_of<1024>(a.rows), dim3(1024), 0, s>>>(a);
  else
    launch_team<Forward, T>(a, a.dim, 0, s);
}

// Workgroups of the gradient, and so rows of parts: eight rows a team, so that the parts stay small
// beside the rows, but 128 of them where there are two rows for each team, and 512 at most (no
// rows: sums of nothing).
uint32_t grad_groups(uint32_t rows, uint32_t dim) {
  const uint32_t lanes = lanes_of(dim), teams = lanes < 256 ? 256 / lanes : 1;
  const auto groups = [&](uint32_t each) { return (uint32_t)(((uint64_t)rows + each * teams - 1) / (each * teams)); };
  const uint32_t few = groups(2) < 128 ? groups(2) : 128, n = groups(8) > few ? groups(8) : few;
  return n < 1 ? 1 : n < 512 ? n : 512;
}

template <typename T>
void launch_grad_t(const NormGradParams& p, hipStream_t s) {
  const gts_norm_grad_args& a = p.a;
  const uint32_t groups = grad_groups(a.rows, a.dim);
  if (!held<T>(a.dim)) {
    // first what only reads: dx may be dy or x
    if (p.dw || p.db) norm_columns_kernel<T><<<dim3((a.dim + 255) / 256, groups), dim3(256), 0, s>>>(p);
    if (a.dx && a.rows) norm_grad_long_kernel<T><<<grid_of<1024>(a.rows), dim3(1024), 0, s>>>(a);
    return;
  }
  launch_team<Gradient, T>(p, a.dim, groups, s);
}

}  // namespace

hipError_t launch_norm(const gts_norm_args& a, hipStream_t s) {
  if (a.dtype == GTS_F32)
    launch_norm_t<float>(a, s);
  else if (a.dtype == GTS_BF16)
    launch_norm_t<__bf16>(a, s);
  else
    launch_norm_t<_Float16>(a, s);
  return hipGetLastError();
}

uint64_t norm_grad_scratch(uint32_t rows, uint32_t dim) { return 8ull * grad_groups(rows, dim) * dim; }

hipError_t launch_norm_grad(const gts_norm_grad_args& a, hipStream_t s) {
  NormGradParams p{a, nullptr, nullptr};
  const uint32_t parts = grad_groups(a.rows, a.dim);
  if (a.dweight) p.dw = (float*)a.scratch;
  if (a.dbias) p.db = (float*)a.scratch + (uint64_t)parts * a.dim;
  if (a.dtype == GTS_F32)
    launch_grad_t<float>(p, s);
  else if (a.dtype == GTS_BF16)
    launch_grad_t<__bf16>(p, s);
  else
    launch_grad_t<_Float16>(p, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_column_sums(p.dw, a.dweight, p.db, a.dbias, parts, a.dim, a.dtype, s);
}

// ---- sums of parts ------------------------------------------------------------------

// out[c] = the sum over parts p of in[p][c], p in the same order on every run: a workgroup takes
// 64 columns, a wave every 16th part, eight loads on their way.
template <typename T>
__global__ __launch_bounds__(1024) void column_sums_kernel(const float* in0, void* out0, const float* in1, void* out1,
                                                           uint32_t parts, uint32_t n) {
  __shared__ float s[16][64];
  const float* in = blockIdx.y ? in1 : in0;
  T* out = (T*)(blockIdx.y ? out1 : out0);
  if (!in) return;
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  float sum = 0.f;
  if (c < n) {
    uint32_t i = wave;
    for (; i + 112 < parts; i += 128) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = in[(uint64_t)(i + 16 * k) * n + c];
#pragma unroll
      for (int k = 0; k < 8; ++k) sum += v[k];
    }
    for (; i < parts; i += 16) sum += in[(uint64_t)i * n + c];
  }
  s[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && c < n) {
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) sum += s[k][lane];
    out[c] = (T)sum;
  }
}

hipError_t launch_column_sums(const float* in0, void* out0, const float* in1, void* out1, uint32_t parts, uint32_t n,
                              uint32_t dtype, hipStream_t s) {
  if (!in0 && !in1) return hipSuccess;
  const dim3 grid((n + 63) / 64, in1 ? 2 : 1), block(1024);
  if (dtype == GTS_F32)
    column_sums_kernel<float><<<grid, block, 0, s>>>(in0, out0, in1, out1, parts, n);
  else if (dtype == GTS_BF16)
    column_sums_kernel<__bf16><<<grid, block, 0, s>>>(in0, out0, in1, out1, parts, n);
  else
    column_sums_kernel<_Float16><<<grid, block, 0, s>>>(in0, out0, in1, out1, parts, n);
  return hipGetLastError();
}

}  // namespace gts
