// gts_norm.hip — layer norm over rows, centered or not, and its gradient.
//
//   forward   mu = mean(x) (0 without centering), r = 1 / sqrt(mean((x - mu)^2) + eps),
//             h = (x - mu) r,  y = h w + b
//   backward  g = dy w,  dx = r (g - mean(g) - h mean(g h)) (no mean(g) without
//             centering),  dw = sum_rows(dy h),  db = sum_rows(dy)
//
// A row belongs to a team: one wave, four or sixteen, the fewest whose registers
// hold it (32 values a thread), so x is read once and the variance is of the
// differences, not a difference of sums.  Longer rows are read again from memory for
// each pass over them.  Bound by HBM when large and by the launch when small.
#include "gts_ops.h"
#include "gts_tile.h"

namespace gts {
namespace {

constexpr int kHeld = 32;  // values of a row that a thread holds

// Sums over a team of W waves; every lane gets them.  s: one slot a wave and sum,
// twice, used in turn so that one barrier a call is enough.
template <int W>
struct Team {
  float (*s)[2][16];
  uint32_t turn = 0;
  __device__ __forceinline__ static float wave_sum(float x) {
#pragma unroll
    for (int k = 32; k; k >>= 1) x += __shfl_xor(x, k);
    return x;
  }
  __device__ __forceinline__ void sum2(float& a, float& b) {
    a = wave_sum(a);
    b = wave_sum(b);
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

// Threads of a workgroup: teams of one wave share one of four.
template <int W>
constexpr int kThreads = W == 1 ? 256 : W * 64;
template <int W>
constexpr int kTeams = W == 1 ? 4 : 1;

// V values at column at of a row, zeros behind its end (V divides the row's length, so
// an access is inside or outside as a whole).
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> columns(const T* row, uint32_t at, uint32_t dim) {
  Pack<T, V> x = {};
  if (at < dim) x = *reinterpret_cast<const Pack<T, V>*>(row + at);
  return x;
}

template <typename T, int V, int W, int C>
__global__ __launch_bounds__(kThreads<W>) void norm_kernel(gts_norm_args a) {
  __shared__ float s_sum[2][2][16];
  Team<W> team{s_sum};
  const uint32_t lane = W == 1 ? threadIdx.x & 63u : threadIdx.x;
  const uint64_t row = block_number() * kTeams<W> + (W == 1 ? threadIdx.x >> 6 : 0);
  if (row >= a.rows) return;
  const bool center = a.flags & GTS_NORM_CENTER;
  const T* x = (const T*)a.x + (int64_t)row * a.x_stride;
  const float n = 1.f / (float)a.dim;
  Pack<T, V> v[C];
#pragma unroll
  for (int c = 0; c < C; ++c) v[c] = columns<T, V>(x, (c * W * 64 + lane) * V, a.dim);
  float mu = 0.f;
  if (center) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) mu += (float)v[c].v[i];
    mu = team.sum(mu) * n;
  }
  float q = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c)
    if ((c * W * 64 + lane) * V < a.dim) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = (float)v[c].v[i] - mu;
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
    const uint32_t at = (c * W * 64 + lane) * V;
    if (at >= a.dim) continue;
    const Pack<T, V> w = a.weight ? *reinterpret_cast<const Pack<T, V>*>((const T*)a.weight + at) : Pack<T, V>{};
    const Pack<T, V> b = a.bias ? *reinterpret_cast<const Pack<T, V>*>((const T*)a.bias + at) : Pack<T, V>{};
    Pack<T, V> o;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float h = ((float)v[c].v[i] - mu) * r;
      if (a.weight) h *= (float)w.v[i];
      if (a.bias) h += (float)b.v[i];
      o.v[i] = (T)h;
    }
    *reinterpret_cast<Pack<T, V>*>(y + at) = o;
  }
}

// Rows of any length: three passes over memory, sums of a thread in order.
template <typename T>
__global__ __launch_bounds__(1024) void norm_long_kernel(gts_norm_args a) {
  __shared__ float s_sum[2][2][16];
  Team<16> team{s_sum};
  const uint64_t row = block_number();
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

// The gradient.  A workgroup takes every gridDim.x-th group of rows and keeps its part
// of dw and db in registers: columns of a thread are the same in every row.  The
// parts, one row of scratch a workgroup, are added up in order by sum_kernel.
struct NormGradParams {
  gts_norm_grad_args a;
  float *dw, *db;  // [groups][dim], NULL if not wanted
};

template <typename T, int V, int W, int C>
__global__ __launch_bounds__(kThreads<W>) void norm_grad_kernel(NormGradParams p) {
  __shared__ float s_sum[2][2][16];
  const gts_norm_grad_args& a = p.a;
  Team<W> team{s_sum};
  const uint32_t lane = W == 1 ? threadIdx.x & 63u : threadIdx.x, mine = W == 1 ? threadIdx.x >> 6 : 0;
  const float n = 1.f / (float)a.dim;
  const bool center = a.flags & GTS_NORM_CENTER;
  float dw[C][V] = {}, db[C][V] = {};
  Pack<T, V> w[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const uint32_t at = (c * W * 64 + lane) * V;
    if (a.weight) {
      w[c] = columns<T, V>((const T*)a.weight, at, a.dim);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) w[c].v[i] = (T)1.f;
    }
  }
  for (uint64_t row = (uint64_t)blockIdx.x * kTeams<W> + mine; row < a.rows; row += (uint64_t)gridDim.x * kTeams<W>) {
    const T* x = (const T*)a.x + (int64_t)row * a.x_stride;
    const T* dy = (const T*)a.dy + (int64_t)row * a.dy_stride;
    Pack<T, V> xv[C], dv[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const uint32_t at = (c * W * 64 + lane) * V;
      xv[c] = columns<T, V>(x, at, a.dim);
      dv[c] = columns<T, V>(dy, at, a.dim);
    }
    const float mu = center ? a.mean[row] : 0.f, r = a.rstd[row];
    float sg = 0.f, sgh = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
      if ((c * W * 64 + lane) * V < a.dim) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float h = ((float)xv[c].v[i] - mu) * r, d = (float)dv[c].v[i], g = d * (float)w[c].v[i];
          sg += g;
          sgh += g * h;
          dw[c][i] += d * h;
          db[c][i] += d;
        }
      }
    team.sum2(sg, sgh);
    const float mg = center ? sg * n : 0.f, mgh = sgh * n;
    T* dx = (T*)a.dx + (int64_t)row * a.dx_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const uint32_t at = (c * W * 64 + lane) * V;
      if (at >= a.dim) continue;
      Pack<T, V> o;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float h = ((float)xv[c].v[i] - mu) * r;
        o.v[i] = (T)(((float)dv[c].v[i] * (float)w[c].v[i] - mg - h * mgh) * r);
      }
      if (a.dx) *reinterpret_cast<Pack<T, V>*>(dx + at) = o;
    }
  }
  const uint64_t part = ((uint64_t)blockIdx.x * kTeams<W> + mine) * a.dim;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const uint32_t at = (c * W * 64 + lane) * V;
    if (at >= a.dim) continue;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (p.dw) p.dw[part + at + i] = dw[c][i];
      if (p.db) p.db[part + at + i] = db[c][i];
    }
  }
}

// Rows of any length.  dw and db: a column's sum over a strip of rows.
template <typename T>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(gts_norm_grad_args a) {
  __shared__ float s_sum[2][2][16];
  Team<16> team{s_sum};
  const uint64_t row = block_number();
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

bool wide(uint64_t bytes, uint64_t elements, uint32_t v, uint32_t e) { return bytes % (v * e) == 0 && elements % v == 0; }
uint64_t size(int64_t x) { return (uint64_t)(x < 0 ? -x : x); }

template <typename T, int V, int W>
void launch_norm_w(const gts_norm_args& a, hipStream_t s) {
  const uint32_t per = W * 64 * V;
  const dim3 grid = grid_of(((uint64_t)a.rows + kTeams<W> - 1) / kTeams<W>), block(kThreads<W>);
  constexpr int C = kHeld / V;
  if (C >= 4 && a.dim <= per * (C / 4))
    norm_kernel<T, V, W, C / 4 ? C / 4 : 1><<<grid, block, 0, s>>>(a);
  else if (C >= 2 && a.dim <= per * (C / 2))
    norm_kernel<T, V, W, C / 2 ? C / 2 : 1><<<grid, block, 0, s>>>(a);
  else
    norm_kernel<T, V, W, C><<<grid, block, 0, s>>>(a);
}

template <typename T, int V>
void launch_norm_v(const gts_norm_args& a, hipStream_t s) {
  if (a.dim <= 64 * kHeld / 2)
    launch_norm_w<T, V, 1>(a, s);
  else if (a.dim <= 256 * kHeld)
    launch_norm_w<T, V, 4>(a, s);
  else
    launch_norm_w<T, V, 16>(a, s);
}

template <typename T>
void launch_norm_t(const gts_norm_args& a, hipStream_t s) {
  constexpr int V = 16 / sizeof(T);
  if (a.dim > 1024 * kHeld) {
    norm_long_kernel<T><<<grid_of(a.rows), dim3(1024), 0, s>>>(a);
    return;
  }
  const uint64_t bytes = (uint64_t)(uintptr_t)a.x | (uint64_t)(uintptr_t)a.out | (uint64_t)(uintptr_t)a.weight |
                         (uint64_t)(uintptr_t)a.bias;
  if (wide(bytes, size(a.x_stride) | size(a.out_stride) | a.dim, V, sizeof(T)))
    launch_norm_v<T, V>(a, s);
  else
    launch_norm_v<T, 1>(a, s);
}

// Workgroups of the gradient: rows enough for each, and two a CU at most, so that
// the parts stay small beside the rows.
constexpr uint32_t kGradGroups = 512;
uint32_t grad_groups(uint32_t rows) {
  const uint64_t n = ((uint64_t)rows + 3) / 4;
  return n < 1 ? 1 : n < kGradGroups ? (uint32_t)n : kGradGroups;  // no rows: sums of nothing
}
// Rows of parts: four a workgroup where a team is one wave.
uint32_t grad_parts(uint32_t rows, uint32_t dim) { return grad_groups(rows) * (dim <= 64 * kHeld / 2 ? 4 : 1); }

template <typename T, int V, int W>
void launch_grad_w(const NormGradParams& p, hipStream_t s) {
  const uint32_t per = W * 64 * V;
  const dim3 grid(grad_groups(p.a.rows)), block(kThreads<W>);
  constexpr int C = kHeld / V;
  if (C >= 4 && p.a.dim <= per * (C / 4))
    norm_grad_kernel<T, V, W, C / 4 ? C / 4 : 1><<<grid, block, 0, s>>>(p);
  else if (C >= 2 && p.a.dim <= per * (C / 2))
    norm_grad_kernel<T, V, W, C / 2 ? C / 2 : 1><<<grid, block, 0, s>>>(p);
  else
    norm_grad_kernel<T, V, W, C><<<grid, block, 0, s>>>(p);
}
template <typename T, int V>
void launch_grad_v(const NormGradParams& p, hipStream_t s) {
  if (p.a.dim <= 64 * kHeld / 2)
    launch_grad_w<T, V, 1>(p, s);
  else if (p.a.dim <= 256 * kHeld)
    launch_grad_w<T, V, 4>(p, s);
  else
    launch_grad_w<T, V, 16>(p, s);
}
template <typename T>
void launch_grad_t(const NormGradParams& p, hipStream_t s) {
  const gts_norm_grad_args& a = p.a;
  constexpr int V = 16 / sizeof(T);
  if (a.dim > 1024 * kHeld) {
    if (a.dx && a.rows) norm_grad_long_kernel<T><<<grid_of(a.rows), dim3(1024), 0, s>>>(a);
    if (p.dw || p.db)
      norm_columns_kernel<T><<<dim3((a.dim + 255) / 256, grad_parts(a.rows, a.dim)), dim3(256), 0, s>>>(p);
    return;
  }
  const uint64_t bytes = (uint64_t)(uintptr_t)a.x | (uint64_t)(uintptr_t)a.dy | (uint64_t)(uintptr_t)a.weight |
                         (uint64_t)(uintptr_t)a.dx;
  if (wide(bytes, size(a.x_stride) | size(a.dy_stride) | size(a.dx_stride) | a.dim, V, sizeof(T)))
    launch_grad_v<T, V>(p, s);
  else
    launch_grad_v<T, 1>(p, s);
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

uint64_t norm_grad_scratch(uint32_t rows, uint32_t dim) { return 8ull * grad_parts(rows, dim) * dim; }

hipError_t launch_norm_grad(const gts_norm_grad_args& a, hipStream_t s) {
  NormGradParams p{a, nullptr, nullptr};
  const uint32_t parts = grad_parts(a.rows, a.dim);
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

// out[c] = the sum over parts p of in[p][c], p in the same order on every run: a
// workgroup takes 64 columns, a wave every fourth part.
template <typename T>
__global__ __launch_bounds__(256) void column_sums_kernel(const float* in0, void* out0, const float* in1, void* out1,
                                                          uint32_t parts, uint32_t n) {
  __shared__ float s[4][64];
  const float* in = blockIdx.y ? in1 : in0;
  T* out = (T*)(blockIdx.y ? out1 : out0);
  if (!in) return;
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  float sum = 0.f;
  if (c < n) {
    // eight loads on their way
    uint32_t i = wave;
    for (; i + 28 < parts; i += 32) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = in[(uint64_t)(i + 4 * k) * n + c];
#pragma unroll
      for (int k = 0; k < 8; ++k) sum += v[k];
    }
    for (; i < parts; i += 4) sum += in[(uint64_t)i * n + c];
  }
  s[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && c < n) out[c] = (T)((s[0][lane] + s[1][lane]) + (s[2][lane] + s[3][lane]));
}

hipError_t launch_column_sums(const float* in0, void* out0, const float* in1, void* out1, uint32_t parts, uint32_t n,
                              uint32_t dtype, hipStream_t s) {
  if (!in0 && !in1) return hipSuccess;
  const dim3 grid((n + 63) / 64, in1 ? 2 : 1), block(256);
  if (dtype == GTS_F32)
    column_sums_kernel<float><<<grid, block, 0, s>>>(in0, out0, in1, out1, parts, n);
  else if (dtype == GTS_BF16)
    column_sums_kernel<__bf16><<<grid, block, 0, s>>>(in0, out0, in1, out1, parts, n);
  else
    column_sums_kernel<_Float16><<<grid, block, 0, s>>>(in0, out0, in1, out1, parts, n);
  return hipGetLastError();
}

}  // namespace gts
