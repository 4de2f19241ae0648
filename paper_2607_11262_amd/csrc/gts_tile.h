// gts_tile.h — device helpers of the operators' tile kernels: matrix instructions,
// exchanges between the halves of a wave, loads to LDS, values that are not finite.
#pragma once
#include "gts_ops.h"

#ifdef __HIPCC__
namespace gts {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
template <typename T>
using Vec8 = T __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x16 mfma(Vec8<__bf16> a, Vec8<__bf16> b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma(Vec8<_Float16> a, Vec8<_Float16> b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ uint32_t uni(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t uni(uint64_t x) {
  return ((uint64_t)uni((uint32_t)(x >> 32)) << 32) | uni((uint32_t)x);
}
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
// The lane's number as a value of its own: what is computed from it stays where
// it is used, instead of being kept in registers across the loops around.
__device__ __forceinline__ uint32_t fresh_lane() {
  uint32_t lane = threadIdx.x & 63u;
  asm volatile("" : "+v"(lane));
  return lane;
}
// The value of the lane 32 away joined with this lane's.
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float add_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// 16 bytes a lane from memory to LDS, lane after lane from `to` on (the same in
// all lanes).  Nothing waits for it but the wait for all loads before the barrier
// that hands the tile over: written as the compiler's builtin, it waits for every
// such load before the next LDS read, whatever that reads, and no tile is on its
// way while another is worked on.  M0, the LDS address, is the compiler's: it gets
// its value back.
__device__ __forceinline__ void load_to_lds(const void* from, void* to) {
  const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)to;
  uint32_t m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\ts_mov_b32 m0, %0"
               : "=&s"(m0)
               : "s"(at), "v"(from)
               : "memory");
}

// The same from a base that all lanes share and an offset in bytes below 2^32.
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t offset, void* to) {
  const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)to;
  uint32_t m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
               : "=&s"(m0)
               : "s"(at), "v"(offset), "s"(base)
               : "memory");
}

__device__ __forceinline__ bool not_finite(float x) { return !(__builtin_fabsf(x) < INFINITY); }
template <typename T>
__device__ __forceinline__ bool any_not_finite(u32x4 v) {
  constexpr uint32_t kExp = __is_same(T, __bf16) ? 0x7F80u : 0x7C00u;
  bool found = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) found |= (v[i] & kExp) == kExp || (v[i] >> 16 & kExp) == kExp;
  return found;
}
template <typename T>
__device__ __forceinline__ u32x4 finite_only(u32x4 v) {
  constexpr uint32_t kExp = __is_same(T, __bf16) ? 0x7F80u : 0x7C00u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((v[i] & kExp) == kExp) v[i] &= 0xFFFF0000u;
    if ((v[i] >> 16 & kExp) == kExp) v[i] &= 0xFFFFu;
  }
  return v;
}

// 32 bits: eight instructions of two products each.  Element j of lane half h is the
// same place of the sum in both operands, as in the 16-bit instructions.
__device__ __forceinline__ f32x16 mfma(Vec8<float> a, Vec8<float> b, f32x16 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

// ---- fragments of a 32 x 32 product, 16 places of the sum at a time ------------------
// Operands: a lane has row (of A) or column (of B) lane % 32 and eight places of the
// sum, by its half.  Result: column lane % 32, row frag_row(i, half) for i < 16.
__device__ __forceinline__ uint32_t frag_row(int i, uint32_t half) { return 8 * (i / 4) + 4 * half + i % 4; }

// Eight values side by side, aligned to 16 bytes.
template <typename T>
struct alignas(16) Eight {
  T v[8];
};
template <typename T>
__device__ __forceinline__ Vec8<T> read8(const T* p) {
  const Eight<T> x = *reinterpret_cast<const Eight<T>*>(p);
  Vec8<T> r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = x.v[i];
  return r;
}
template <typename T>
__device__ __forceinline__ void write8(T* p, Vec8<T> x) {
  Eight<T> y;
#pragma unroll
  for (int i = 0; i < 8; ++i) y.v[i] = x[i];
  *reinterpret_cast<Eight<T>*>(p) = y;
}
// From LDS rows of `pitch` values that hold the sum's places side by side.
template <typename T>
__device__ __forceinline__ Vec8<T> frag_rows(const T* s, uint32_t pitch, uint32_t row, uint32_t k, uint32_t lane) {
  return read8(s + (row + lane % 32) * pitch + k + 8 * (lane / 32));
}
// From LDS rows that are the sum's places, turned on the way: places 8 half .. + 7, or,
// as a result of a product has them (TURNED), 4 half .. + 3 and 8 further.
template <bool TURNED, typename T>
__device__ __forceinline__ Vec8<T> frag_columns(const T* s, uint32_t pitch, uint32_t k, uint32_t column, uint32_t lane) {
  const uint32_t half = lane / 32;
  if constexpr (sizeof(T) == 2) {
    typedef __attribute__((address_space(3))) i16x4* lds_t;
    const uint32_t row = k + (TURNED ? 4 : 8) * half + lane % 16 / 4, c = column + lane / 16 % 2 * 16 + lane % 4 * 4;
    union {
      i16x4 h[2];
      Vec8<T> v;
    } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(s + row * pitch + c));
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(s + (row + (TURNED ? 8 : 4)) * pitch + c));
    return u.v;
  } else {
    Vec8<T> r;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      r[i] = s[(k + (TURNED ? 4 * half + i % 4 + i / 4 * 8 : 8 * half + i)) * pitch + column + lane % 32];
    return r;
  }
}
// Eight values from memory at any alignment (the card loads 16 bytes from any address of a
// value), or the first `valid` of them with zeros behind.
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) EightAnywhere {
  T v[8];
};
template <typename T>
__device__ __forceinline__ Vec8<T> load_any(const T* p) {
  const EightAnywhere<T> x = *reinterpret_cast<const EightAnywhere<T>*>(p);
  Vec8<T> r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = x.v[i];
  return r;
}
template <typename T>
__device__ __forceinline__ Vec8<T> load8(const T* p, int64_t valid) {
  if (valid >= 8) return load_any(p);
  Vec8<T> r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = i < valid ? p[i] : (T)0.f;
  return r;
}
template <typename T>
__device__ __forceinline__ bool clear_not_finite(Vec8<T>& x) {
  bool found = false;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (not_finite((float)x[i])) {
      found = true;
      x[i] = (T)0.f;
    }
  return found;
}

}  // namespace gts
#endif
