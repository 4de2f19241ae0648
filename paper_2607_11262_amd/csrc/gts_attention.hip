// gts_attention.hip — attention of new tokens over a paged cache and the
// prefix that all sequences share.
//
// Two kernels and a join.
//
// The tile kernel takes 16-bit caches whose rows can be loaded 16 bytes at a
// time.  All work is cut into tiles of 64 keys of one key-value head against
// up to 128 query rows (a row: one new token's one query head).  For the
// prefix the rows are those of all tokens of the batch, so its keys are read
// once for everybody; for a sequence's own keys they are its tokens'.  The
// tiles of all segments (rows with the keys that they see) stand in one line,
// with as many places as they cost, behind some for a segment's begin and end.
// The line is the same for every key-value head; it is cut into equal stretches,
// wherever they start and end, one for each workgroup of the head: ragged
// lengths and few rows fill the chip alike, and the workgroups of all heads walk
// the same pages at the same time, where the heads of a token lie side by side.
// Where the prefix has many rows, its segments are first dealt out whole, or in
// equal pieces, one for each workgroup: they then walk the same keys at the same
// time, and all but the first of an XCD find them in its L2.  (All of it in the
// line: 8 TB/s from behind the L2s, twice the time.)
// A stretch leaves one partial result per segment of which it has tiles
// (unnormalised sum, running maximum and sum of the softmax, 32 bits), and the join
// adds up the partials of each row.
// Measured (tile kernel and join, back to back, heads 32 / 8 of 128 in bfloat16): 64
// ragged decodes of 601491 keys 396 us (6.2 TB/s, bound by the loads), 2113 prompt tokens
// behind 32768 shared keys 1320 to 1390 us (820 to 860 TFLOP/s, bound by matrix and vector
// instructions that do not overlap), 64 decodes behind 8192 shared keys 49 us and one of 512
// keys 15 us (bound by chains of loads at a stretch's begin and end).  In the prompts the
// matrix units are busy 38 % of the time, vector instructions take 43 % and LDS reads 20 %.
//
// The row kernel: one wavefront per (token, query head) walks the row's keys 64
// at a time, one key a lane, with the running maximum and sum of the softmax;
// the weighted values are summed with a lane per group of dims.  Takes every
// type, head dim, stride and alignment; every row reads its keys by itself.
#include "gts_ops.h"

namespace gts {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr uint32_t kTile = 64;        // keys of a tile
constexpr uint32_t kMostRows = 128;   // query rows of a segment
constexpr uint32_t kGroups = 512;     // most workgroups: two a CU
// Rows from which a wave of the join takes four: 2048 rows take 8.0 us by one, 9.1 by
// four; 67616 rows 96 and 26.
constexpr uint32_t kFourRows = 4096;

// Places in the line (of about half a microsecond): a segment's begin and end,
// and a tile, by the segment's row groups.  Measured with few rows 5 us and 1 us
// (nothing else running), with 128 rows 12 us and 2.6 us (two workgroups a CU).
constexpr uint32_t kMostPlaces = 5, kLeastStretch = 5;
__host__ __device__ __forceinline__ uint32_t segment_places(uint32_t row_groups) { return row_groups == 1 ? 10 : 24; }
__host__ __device__ __forceinline__ uint32_t tile_places(uint32_t row_groups) {
  return row_groups == 1 ? 2 : row_groups == 2 ? 3 : kMostPlaces;
}

// What the kernels need beside the arguments.
struct AttnParams {
  gts_attention_args a;
  uint32_t page_shift;
  uint32_t group;       // query heads of a key-value head
  FastDiv by_group, by_q_heads;
  bool near_rows;       // see Loader
  uint32_t cuts;        // stretches of a head's line: so many workgroups for each head
  uint32_t part_rows;   // rows that a cut between workgroups may add to the partials
  uint32_t pieces;      // of each segment of the prefix
  uint32_t whole;       // pieces that each workgroup takes before its stretch of the line
};

// Scratch: the plan (what the tile kernel's first workgroup leaves for the
// join), then the partials: maximum and sum of each row, then its sums.
struct Plan {
  uint64_t per;    // places of a workgroup
  double per_inv;  // 1 / per
  // Which workgroup has place x (below 2^53), without a 64-bit division.
  __device__ __forceinline__ uint32_t group_of(uint64_t x) const {
    uint64_t g = (uint64_t)((double)x * per_inv);
    if (g * per > x) --g;
    if ((g + 1) * per <= x) ++g;
    return (uint32_t)g;
  }
};
struct Scratch {
  uint64_t begin, stats, sums, bytes;  // offsets; begin: [batch] first place of each sequence
};
__host__ __device__ inline uint64_t up256(uint64_t x) { return (x + 255) & ~255ull; }
// Rows of partials: every row's of the prefix and of its own keys, and what the
// cuts between workgroups add: a segment's rows each, once more for pieces.
__host__ __device__ inline uint64_t head_partials(uint64_t rows, uint64_t cut_rows) { return 2 * rows + 2 * cut_rows; }
__host__ __device__ inline Scratch scratch_layout(uint32_t batch, uint64_t rows, uint64_t cut_rows, uint32_t dim) {
  Scratch s;
  s.begin = 256;
  s.stats = s.begin + up256(8ull * batch);
  const uint64_t n = head_partials(rows, cut_rows);
  s.sums = s.stats + up256(8 * n);
  s.bytes = s.sums + up256(4 * n * dim);
  return s;
}

// A page table: global memory, said in the type, because a load that might be from
// LDS makes every LDS read wait for it.
typedef const __attribute__((address_space(1))) int32_t* pages_t;

// Page of own or prefix key j, -1 when none holds it.
__device__ __forceinline__ int32_t key_page(const gts_attention_args& a, pages_t pages, uint32_t n, uint32_t shift,
                                            uint32_t j) {
  const uint32_t at = j >> shift;
  if (at >= n) return -1;
  const int32_t p = pages[at];
  return p >= 0 && (uint32_t)p < a.cache.n_pages ? p : -1;
}

// ---- the tile kernel -------------------------------------------------------------

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

// Rows of a segment for n query rows: 32 rg.  rg = 1: the stream below; 2 and 4:
// so many of the four waves take rows of their own (with 2, the others take the
// other half of the keys).
__host__ __device__ __forceinline__ uint32_t row_groups(uint32_t rows) { return rows <= 32 ? 1 : rows <= 64 ? 2 : 4; }

// New tokens and own keys of sequence b.
struct Seq {
  uint32_t first, n;  // first token, tokens
  int64_t len;        // own keys by lens
  uint32_t keys;      // of these, those that pages can hold
};
__device__ __forceinline__ Seq make_seq(const AttnParams& p, int32_t s0, int32_t s1, int32_t len) {
  const bool ok = s0 >= 0 && s1 > s0 && (uint32_t)s1 <= p.a.batch.tokens;
  Seq s;
  s.first = ok ? (uint32_t)s0 : 0;
  s.n = ok ? (uint32_t)(s1 - s0) : 0;
  s.len = len;
  const uint64_t cap = (uint64_t)p.a.batch.max_pages << p.page_shift;
  const int64_t k = s.len < 0 || p.a.cache.n_pages == 0 ? 0 : s.len;
  s.keys = (uint32_t)((uint64_t)k < cap ? (uint64_t)k : cap);
  return s;
}
__device__ __forceinline__ Seq load_seq(const AttnParams& p, uint32_t b) {
  const gts_kv_batch& kb = p.a.batch;
  const uint32_t n = kb.tokens / kb.batch;
  return kb.starts ? make_seq(p, kb.starts[b], kb.starts[b + 1], kb.lens[b])
                   : make_seq(p, (int32_t)(b * n), (int32_t)(b * n + n), kb.lens[b]);
}
// Own keys that token i of the sequence sees.
__device__ __forceinline__ uint32_t seen(const Seq& s, uint32_t i) {
  const int64_t v = s.len - s.n + i + 1;
  return v < 0 ? 0 : v < (int64_t)s.keys ? (uint32_t)v : s.keys;
}
// Tiles of the rt-th segment of a sequence (rows rt * 32 rg ..): as far as its
// last row sees.
__device__ __forceinline__ uint32_t own_tiles(const AttnParams& p, const Seq& s, uint32_t rg, uint32_t rt) {
  const uint32_t rows = s.n * p.group, end = (rt + 1) * 32 * rg;
  const uint32_t last = p.by_group.div((rows < end ? rows : end) - 1);
  return (seen(s, last) + kTile - 1) / kTile;
}
__device__ __forceinline__ uint64_t places(uint32_t tiles, uint32_t rg) {
  return tiles ? (uint64_t)tiles * tile_places(rg) + segment_places(rg) : 0;
}
// Places of a sequence's segments.
__device__ __forceinline__ uint64_t seq_places(const AttnParams& p, const Seq& s) {
  const uint32_t rows = s.n * p.group;
  if (rows == 0 || s.keys == 0) return 0;
  const uint32_t rg = row_groups(rows), n = (rows + 32 * rg - 1) / (32 * rg);
  uint64_t t = 0;
  for (uint32_t rt = 0; rt < n; ++rt) t += places(own_tiles(p, s, rg, rt), rg);
  return t;
}

// One stretch of one segment.
struct Work {
  pages_t pages;
  uint32_t n_pages, keys;    // keys: of the segment's last row
  uint32_t head, rg, rows;   // key-value head, row groups, valid rows
  uint32_t first_row;        // token * group + query head within the group
  uint32_t tile, n_tiles;    // first tile and number of tiles of the stretch
  uint32_t low;              // keys that its first row sees
  int64_t see;               // row r sees see + token keys; own == false: all
  bool own;
  uint64_t part;             // first row of its partial
};

template <typename T, int DP>
struct Tiles {
  static constexpr int C = DP / 8;         // 16-byte chunks of a row
  static constexpr int RPI = 64 / C;       // rows that one load of a wave covers
  static constexpr int NL = 16 / RPI;      // loads of a wave for its 16 rows of a tile
  static constexpr int KK = DP / 16;       // matrix steps over the head
  static constexpr int MB = DP / 32;       // blocks of 32 output dims
  static constexpr int N = kTile * DP;     // values of a tile of keys
  // Chunk c of row r stands at c ^ swizzle(r): the 16-byte reads of 16 rows
  // at one chunk (keys), and the reads of 4 rows x 64 bytes that are turned
  // on the way (values), each touch all 64 banks once.
  static __device__ __forceinline__ uint32_t swizzle_k(uint32_t r) { return C >= 16 ? r & 15 : (r >> 1) & 7; }
  static __device__ __forceinline__ uint32_t swizzle_v(uint32_t r) {
    return C >= 16 ? ((r & 3) << 2) | ((r >> 2) & 3) : ((r & 2) << 1) | ((r >> 2) & 3);
  }
};

// What rows of a tile that do not exist are loaded from.
__device__ __align__(16) const uint32_t g_zeros[GTS_OPS_MAX_ATTN / 2] = {};  // a row
// What the page of a key that does not exist is loaded from.
__device__ const int32_t g_no_page = -1;

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

// Loads tiles of keys and values from the cache straight into LDS (no
// registers in between, so nothing is held while the tile before is worked
// on).  A wave loads 16 rows of a tile; rows past the segment's keys, or without
// a page, become zeros.  Chunks past the head are not loaded where whole rows
// are: the LDS holds zeros there from the stretch's beginning on.
template <typename T, int DP>
struct Loader {
  using L = Tiles<T, DP>;
  uint32_t k_off[L::NL], v_off[L::NL];  // bytes from the wave's first row to this lane's chunk
  int32_t page;                         // page of the wave's rows in the next tile (pages of 16 or more)
  uint32_t wave;
  bool near;  // pages of 16 or more, and 16 rows lie within 2 GiB: k_off and v_off serve

  __device__ __forceinline__ void start(const AttnParams& p, const Work& w, uint32_t wave_) {
    const gts_kv_cache& kc = p.a.cache;
    wave = wave_;
    near = p.near_rows;
    const uint32_t lane = fresh_lane(), c = lane % L::C, r0 = lane / L::C;
#pragma unroll
    for (int n = 0; n < L::NL; ++n) {
      const uint32_t r = n * L::RPI + r0;
      k_off[n] = 2 * (r * (uint32_t)kc.k_stride[1] + (c ^ L::swizzle_k(r)) * 8);
      v_off[n] = 2 * (r * (uint32_t)kc.v_stride[1] + (c ^ L::swizzle_v(r)) * 8);
    }
    page = p.page_shift >= 4 ? next_page(p, w, w.tile) : 0;
  }
  // By a vector load, though it is the same for all lanes: LDS reads wait for
  // every scalar load before them (one counter), and this one may be long.
  __device__ __forceinline__ int32_t next_page(const AttnParams& p, const Work& w, uint32_t tile) const {
    const uint32_t at = (tile * kTile + wave * 16) >> p.page_shift;
    uint32_t zero = 0;
    asm volatile("" : "+v"(zero));
    return at < w.n_pages ? (w.pages + at)[zero] : -1;
  }

  // Returns the wave's rows inside the segment that no page holds (one bit
  // each, the same in all lanes).
  __device__ __forceinline__ uint32_t load(const AttnParams& p, const Work& w, uint32_t tile, T* sk, T* sv) {
    const gts_kv_cache& kc = p.a.cache;
    const uint32_t j0 = tile * kTile + wave * 16;
    const uint32_t pg0 = uni((uint32_t)page);
    if (near && pg0 < kc.n_pages && j0 + 16 <= w.keys) {
      const uint32_t slot = j0 & (kc.page - 1);
      const char* kp = (const char*)((const T*)kc.k + (int64_t)pg0 * kc.k_stride[0] + (int64_t)slot * kc.k_stride[1] +
                                     (int64_t)w.head * kc.k_stride[2]);
      const char* vp = (const char*)((const T*)kc.v + (int64_t)pg0 * kc.v_stride[0] + (int64_t)slot * kc.v_stride[1] +
                                     (int64_t)w.head * kc.v_stride[2]);
      if (kc.dim == DP) {
#pragma unroll
        for (int n = 0; n < L::NL; ++n) {
          const uint32_t at = (wave * 16 + n * L::RPI) * DP;
          load_to_lds(kp + k_off[n], sk + at);
          load_to_lds(vp + v_off[n], sv + at);
        }
      } else {
        const uint32_t lane = fresh_lane(), c = lane % L::C, r0 = lane / L::C;
#pragma unroll
        for (int n = 0; n < L::NL; ++n) {
          const uint32_t at = (wave * 16 + n * L::RPI) * DP, r = n * L::RPI + r0;
          if ((c ^ L::swizzle_k(r)) * 8 < kc.dim) load_to_lds(kp + k_off[n], sk + at);
          if ((c ^ L::swizzle_v(r)) * 8 < kc.dim) load_to_lds(vp + v_off[n], sv + at);
        }
      }
      page = next_page(p, w, tile + 1);
      return 0;
    }
    // the general way: every row by itself
    const uint32_t lane = fresh_lane(), c = lane % L::C, r0 = lane / L::C;
    uint32_t missing = 0;
#pragma unroll 1
    for (int n = 0; n < L::NL; ++n) {
      const uint32_t r = n * L::RPI + r0, j = j0 + r;
      const bool in = j < w.keys;
      const int32_t pg = in ? key_page(p.a, w.pages, w.n_pages, p.page_shift, j) : -1;
      const uint64_t lost = __ballot(in && pg < 0);
      for (int i = 0; i < L::RPI; ++i) missing |= (uint32_t)(lost >> (i * L::C) & 1) << (n * L::RPI + i);
      const int64_t slot = j & (kc.page - 1);
      const uint32_t ck = (c ^ L::swizzle_k(r)) * 8, cv = (c ^ L::swizzle_v(r)) * 8;
      const T* kp = (const T*)kc.k + (int64_t)pg * kc.k_stride[0] + slot * kc.k_stride[1] + (int64_t)w.head * kc.k_stride[2] + ck;
      const T* vp = (const T*)kc.v + (int64_t)pg * kc.v_stride[0] + slot * kc.v_stride[1] + (int64_t)w.head * kc.v_stride[2] + cv;
      kp = pg >= 0 && ck < kc.dim ? kp : (const T*)g_zeros;
      vp = pg >= 0 && cv < kc.dim ? vp : (const T*)g_zeros;
      const uint32_t at = (wave * 16 + n * L::RPI) * DP;
      load_to_lds(kp, sk + at);
      load_to_lds(vp, sv + at);
    }
    if (p.page_shift >= 4) page = next_page(p, w, tile + 1);
    return missing;
  }
};

// Values of 8 keys at one dim, as the matrix instruction takes them: keys
// key .. + 3 and key + 8 .. + 11 of this lane's half (the sum over keys may
// take them in any order as long as the weights come in the same).
template <typename T, int DP>
__device__ __forceinline__ Vec8<T> load_v(const T* sv, uint32_t lane, uint32_t key, uint32_t mb) {
  using L = Tiles<T, DP>;
  const uint32_t g = lane / 16, r = 4 * (g / 2) + (lane % 16) / 4;  // key is a multiple of 16
  const uint32_t c = (g % 2) * 2 + (lane % 4) / 2;
  typedef __attribute__((address_space(3))) i16x4* lds_t;
  union {
    i16x4 h[2];
    Vec8<T> v;
  } u;
  const T* at = sv + (key + r) * DP + (lane % 2) * 4;
  u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(at + ((c ^ L::swizzle_v(r)) ^ (mb * 4)) * 8));
  u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(at + 8 * DP + ((c ^ L::swizzle_v(r + 8)) ^ (mb * 4)) * 8));
  return u.v;
}

// Values that are not finite, in a block of keys that some rows do not see to
// its end: 0 times one of them would reach rows that must not see it.  So they
// are cleared in the copy that is multiplied, and added here, from the cache,
// to the rows that see them.  `add(key, d, x)` gets four values x from dim d on.
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
template <typename T>
__device__ __forceinline__ const T* value_row(const AttnParams& p, const Work& w, uint32_t j) {
  const gts_kv_cache& kc = p.a.cache;
  const int32_t page = j < w.keys ? key_page(p.a, w.pages, w.n_pages, p.page_shift, j) : -1;
  if (page < 0) return nullptr;
  return (const T*)kc.v + (int64_t)page * kc.v_stride[0] + (int64_t)(j & (kc.page - 1)) * kc.v_stride[1] +
         (int64_t)w.head * kc.v_stride[2];
}

// What a wave holds: 32 query rows against its keys.  Scores are computed as
// keys x rows, so a lane has 16 of 32 keys of one row: maximum and sum need one
// exchange with the lane 32 away, and the weights are already where the
// second product (dims x rows) wants them.
template <typename T, int DP>
struct Rows {
  using L = Tiles<T, DP>;
  Vec8<T> q[L::KK];
  f32x16 o[L::MB];
  float m, l;  // reference maximum of q.k (unscaled), sum of this half's weights

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < L::MB; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    m = -INFINITY;
    l = 0.f;
  }

  // NS blocks of 32 keys from LDS row `key` on (key number j0 of the segment).
  template <int NS>
  __device__ __forceinline__ void step(uint32_t lane, const T* sk, const T* sv, uint32_t key, uint32_t j0, float c, bool mask,
                                       uint64_t missing, uint32_t sees) {
    const uint32_t half = lane / 32;
    f32x16 s[NS];
    const T* ka = sk + (key + lane % 32) * DP;
    const uint32_t kc = half ^ L::swizzle_k(lane % 32);
#pragma unroll
    for (int b = 0; b < NS; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
    // The fragments of two matrix steps are read while the two before are
    // multiplied; the fences keep that order.
    Vec8<T> kf[2][2][NS];
    const auto read = [&](int at, int kk) {
#pragma unroll
      for (int b = 0; b < NS; ++b) {
        kf[at][0][b] = *(const Vec8<T>*)(ka + b * 32 * DP + (kc ^ (2 * kk)) * 8);
        kf[at][1][b] = *(const Vec8<T>*)(ka + b * 32 * DP + (kc ^ (2 * kk + 2)) * 8);
      }
    };
    read(0, 0);
#pragma unroll
    for (int kk = 0; kk < L::KK; kk += 2) {
      if (kk + 2 < L::KK) read(kk / 2 + 1 & 1, kk + 2);
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
        for (int i = 0; i < 16; ++i) {
          const uint32_t r = b * 32 + 8 * (i / 4) + 4 * half + i % 4;
          const bool ok = j0 + r < sees && !(missing >> (key + r) & 1);
          s[b][i] = ok ? s[b][i] : -INFINITY;
        }
    }
    float mx = s[0][0];
#pragma unroll
    for (int b = 0; b < NS; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[b][i]);
    mx = max_halves(mx);
    // The reference follows the maximum only when that is 2^8 ahead: weights
    // up to 256 are as exact, and sums and output are rescaled rarely.
    if (__any((mx - m) * c > 8.f || (m == -INFINITY && mx > m))) {
      const float m1 = fmaxf(m, mx);
      const float alpha = m == -INFINITY ? 0.f : exp2_((m - m1) * c);
      l *= alpha;
#pragma unroll
      for (int b = 0; b < L::MB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] *= alpha;
      m = m1;
    }
    const float base = m == -INFINITY ? 0.f : -m * c;
    // The weights are multiplied in the cache's type, as the matrix instruction
    // takes them, and summed in 32 bits, which lse keeps.  The result's error against 64
    // bits is 2.2e-3 of its size in bfloat16 (weights in 32 bits: 1.7e-3, the rounding of the
    // result) and 2.2e-4 in float16 (2.1e-4).
    float sum[2] = {0.f, 0.f};
    Vec8<T> pw[2 * NS];
    const auto weigh = [&](int kb, int i) {
      const float e = exp2_(__builtin_fmaf(s[kb / 2][kb % 2 * 8 + i], c, base));
      sum[i & 1] += e;
      pw[kb][i] = (T)e;
    };
    // The weights of 16 keys are computed, and the values of 16 keys read,
    // between the products of the 16 keys before.
    Vec8<T> vf[2][L::MB];
#pragma unroll
    for (int mb = 0; mb < L::MB; ++mb) vf[0][mb] = load_v<T, DP>(sv, lane, key, mb);
#pragma unroll
    for (int i = 0; i < 8; ++i) weigh(0, i);
#pragma unroll
    for (int kb = 0; kb < 2 * NS; ++kb) {
      if (kb + 1 < 2 * NS) {
#pragma unroll
        for (int mb = 0; mb < L::MB; ++mb) vf[kb + 1 & 1][mb] = load_v<T, DP>(sv, lane, key + kb * 16 + 16, mb);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int mb = 0; mb < L::MB; ++mb) {
        o[mb] = mfma(vf[kb & 1][mb], pw[kb], o[mb]);
        if (kb + 1 < 2 * NS) {
#pragma unroll
          for (int i = mb * 8 / L::MB; i < (mb + 1) * 8 / L::MB; ++i) weigh(kb + 1, i);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    l += sum[0] + sum[1];
  }

  // See not_finite: keys j0 .. j0 + 31.
  __device__ __forceinline__ void add_odd(const AttnParams& p, const Work& w, uint32_t lane, uint32_t j0, uint32_t sees) {
#pragma unroll 1
    for (uint32_t j = j0; j < j0 + 32; ++j) {
      const T* v = value_row<T>(p, w, j);
      if (!v) continue;
#pragma unroll
      for (int x = 0; x < L::MB * 4; ++x) {
        const uint32_t d = x / 4 * 32 + 8 * (x % 4) + 4 * (lane / 32);
        if (d >= p.a.cache.dim) continue;
        const Pack<T, 4> y = *(const Pack<T, 4>*)(v + d);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (not_finite((float)y.v[i]) && j < sees) o[x / 4][x % 4 * 4 + i] += (float)y.v[i];
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
};

// Flags that the waves of a workgroup leave each other for a tile.
struct Flags {
  uint16_t missing[2][4];  // rows without a page
  uint32_t odd[4];         // values that are not finite
};

// Tiles i0 .. i1 of a stretch, the first of them already on its way.  One tile is
// worked on while the next is on its way to the other half of the LDS; one
// barrier a tile.
template <int NS, typename T, int DP>
__device__ __forceinline__ void run_tiles(const AttnParams& p, const Work& w, Loader<T, DP>& ld, Rows<T, DP>& r,
                                          uint32_t i0, uint32_t i1, uint32_t wave, uint32_t kgroup, T* s_kv,
                                          Flags* flags, float c, uint32_t sees) {
  using L = Tiles<T, DP>;
  for (uint32_t i = i0; i < i1; ++i) {
    const uint32_t tile = w.tile + i, j0 = tile * kTile;
    T* sk = s_kv + (i & 1) * 2 * L::N;
    T* sv = sk + L::N;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const uint64_t missing = uni(*(const uint64_t*)flags->missing[i & 1]);
    if (i + 1 < w.n_tiles) {
      T* next = s_kv + ((i + 1) & 1) * 2 * L::N;
      const uint32_t miss = ld.load(p, w, tile + 1, next, next + L::N);
      if ((threadIdx.x & 63u) == 0) flags->missing[(i + 1) & 1][wave] = (uint16_t)miss;
    }
    const bool edge = j0 + kTile > w.low;  // some row does not see all of the tile
    const bool mask = edge || missing;
    if constexpr (NS == 2) {
      r.template step<2>(fresh_lane(), sk, sv, 0, j0, c, mask, missing, sees);
    } else {
      bool odd = false;
      if (edge && w.low < w.keys) {
        bool found = false;
        for (uint32_t x = threadIdx.x; x < L::N / 8; x += 256) found |= any_not_finite<T>(*(const u32x4*)(sv + x * 8));
        const bool any = __any(found);
        if ((threadIdx.x & 63u) == 0) flags->odd[wave] = any;
        __syncthreads();
        odd = uni(flags->odd[0] | flags->odd[1] | flags->odd[2] | flags->odd[3]);
        if (odd)
          for (uint32_t x = threadIdx.x; x < L::N / 8; x += 256)
            *(u32x4*)(sv + x * 8) = finite_only<T>(*(const u32x4*)(sv + x * 8));
        __syncthreads();
      }
      // one key group takes all of a tile, two take a half each
#pragma unroll 1
      for (uint32_t x = kgroup * 32; x < kTile; x += w.rg == 4 ? 32 : kTile) {
        r.template step<1>(fresh_lane(), sk, sv, x, j0 + x, c, mask, missing, sees);
        if (odd) r.add_odd(p, w, fresh_lane(), j0 + x, sees);
      }
    }
  }
}

template <typename T, int DP>
__device__ __forceinline__ void run_stretch(const AttnParams& p, const Work& w, T* s_kv, Flags* flags, float* stats,
                                            float* sums) {
  using L = Tiles<T, DP>;
  const gts_attention_args& a = p.a;
  const uint32_t lane = fresh_lane(), wave = uni(threadIdx.x >> 6), half = lane / 32;
  const uint32_t rgroup = wave % w.rg, kgroup = wave / w.rg;
  const uint32_t row = rgroup * 32 + lane % 32;
  const bool valid = row < w.rows;
  const uint32_t flat = w.first_row + (valid ? row : 0);
  const uint32_t token = p.by_group.div(flat), gq = flat - token * p.group;
  const float scale = a.scale;
  const float c = scale == 0.f ? 1.f : __builtin_fabsf(scale) * kLog2e;

  Loader<T, DP> ld;
  ld.start(p, w, wave);
  __syncthreads();  // LDS of the stretch before is free
  if (a.cache.dim < DP) {
    for (uint32_t x = threadIdx.x; x < 4 * L::N / 8; x += 256) *(u32x4*)(s_kv + x * 8) = u32x4{0, 0, 0, 0};
    __syncthreads();
  }
  const uint32_t missing0 = ld.load(p, w, w.tile, s_kv, s_kv + L::N);
  if (lane == 0) flags->missing[0][wave] = (uint16_t)missing0;

  Rows<T, DP> r;
  r.clear();
  {
    // scale's sign (and 0) go into the queries: the maximum of q.k is then
    // that of the scaled scores
    const T* q = (const T*)a.q + (int64_t)token * a.q_stride[0] + (int64_t)(w.head * p.group + gq) * a.q_stride[1];
#pragma unroll
    for (int kk = 0; kk < L::KK; ++kk) {
      const uint32_t d = kk * 16 + half * 8;
      const bool in = valid && d < a.cache.dim;
      u32x4 x = *(const u32x4*)(q + (in ? d : 0));
      const uint32_t keep = in ? ~0u : 0u, flip = scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = (x[i] & keep) ^ flip;
      if (scale == 0.f) x = u32x4{0, 0, 0, 0};
      r.q[kk] = __builtin_bit_cast(Vec8<T>, x);
    }
  }
  uint32_t sees = w.keys;
  if (w.own) {
    const int64_t v = w.see + token;
    sees = !valid ? w.keys : v < 0 ? 0 : v < (int64_t)w.keys ? (uint32_t)v : w.keys;
  }

  // Tiles of which every row sees all keys, or a segment whose rows all see
  // the same: with rows for all four waves, 64 keys a step.
  // (Heads of 256 leave no registers for it.)
  uint32_t plain = 0;
  if (DP <= 128 && w.rg == 4) {
    plain = w.n_tiles;
    if (w.low < w.keys) {
      const uint32_t full = w.low / kTile;  // tiles before the first that a row does not see to its end
      plain = full <= w.tile ? 0 : full - w.tile < w.n_tiles ? full - w.tile : w.n_tiles;
    }
    if constexpr (DP <= 128) run_tiles<2>(p, w, ld, r, 0, plain, wave, kgroup, s_kv, flags, c, sees);
  }
  if (plain < w.n_tiles) run_tiles<1>(p, w, ld, r, plain, w.n_tiles, wave, kgroup, s_kv, flags, c, sees);

  // two waves that took other keys of the same rows: the second hands its to
  // the first
  r.l = add_halves(r.l);
  if (w.rg == 2) {
    constexpr int N = L::MB * 16 + 2;
    static_assert(2 * N * 64 * 4 <= 4 * L::N * sizeof(T), "partials of two waves fit the tiles' LDS");
    float* other = (float*)s_kv + rgroup * N * 64 + lane;
    __syncthreads();
    if (kgroup == 1) {
#pragma unroll
      for (int i = 0; i < L::MB * 16; ++i) other[i * 64] = r.o[i / 16][i % 16];
      other[(N - 2) * 64] = r.m;
      other[(N - 1) * 64] = r.l;
    }
    __syncthreads();
    if (kgroup == 0) {
      const float mo = other[(N - 2) * 64], lo = other[(N - 1) * 64];
      const float m1 = fmaxf(r.m, mo);
      const float fa = r.m == -INFINITY ? 1.f : exp2_((r.m - m1) * c);
      const float fb = mo == -INFINITY ? 1.f : exp2_((mo - m1) * c);
#pragma unroll
      for (int i = 0; i < L::MB * 16; ++i) r.o[i / 16][i % 16] = r.o[i / 16][i % 16] * fa + other[i * 64] * fb;
      r.l = r.l * fa + lo * fb;
      r.m = m1;
    }
  }
  if (kgroup == 0 && valid) {
    const uint64_t at = w.part + row;
    if (half == 0) {
      stats[2 * at] = r.m * c;  // base 2 from here on
      stats[2 * at + 1] = r.l;
    }
    float* dst = sums + at * a.cache.dim;
#pragma unroll
    for (int mb = 0; mb < L::MB; ++mb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t d = mb * 32 + 8 * i + 4 * half;
        if (d < a.cache.dim)
          *(float4*)(dst + d) = make_float4(r.o[mb][4 * i], r.o[mb][4 * i + 1], r.o[mb][4 * i + 2], r.o[mb][4 * i + 3]);
      }
  }
}

// ---- few rows: a stream of keys per wave -------------------------------------------
//
// With at most 32 rows the products are small beside the bytes: every wave
// takes blocks of 32 keys of its own and waits for nobody.  Whole rows of keys and
// values go to registers, and from there to the wave's part of the LDS when the
// block before is done with it: 16 KiB a wave (head dim 128) are on their way
// while it computes.  (Keys loaded as the matrix instruction takes them, 64
// bytes of each of 16 rows, without LDS: 7 % slower on 64 ragged sequences.)
// 16 x 16 tiles, because decode has few rows (query heads of a key-value head).
__device__ __forceinline__ f32x4 mfma16(Vec8<__bf16> a, Vec8<__bf16> b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(Vec8<_Float16> a, Vec8<_Float16> b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
// Joins the values of the four lanes with the same number modulo 16.
__device__ __forceinline__ float max_quarters(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float add_quarters(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return add_halves(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

constexpr uint32_t kBlock = 32;  // keys of a block

template <typename T, int DP>
struct Stream {
  static constexpr int C = DP / 8;           // 16-byte chunks of a row
  static constexpr int RPI = 64 / C;         // rows that one load of values covers
  static constexpr int NV = kBlock / RPI;    // loads of values for a block (16 keys are a whole number)
  static constexpr int KK = DP / 32;         // matrix steps over the head
  static constexpr int DB = DP / 16;         // blocks of 16 output dims
  // Chunk c of row r stands at c ^ swizzle(r), for the reads of 16 rows at one
  // chunk (keys) and of 16 rows x 32 bytes (values).
  static __device__ __forceinline__ uint32_t swizzle_k(uint32_t r) { return C >= 16 ? r & 15 : (r >> 1) & 7; }
  static __device__ __forceinline__ uint32_t swizzle_v(uint32_t r) { return C >= 16 ? (r & 7) << 1 : r & 6; }

  u32x4 k[NV], v[NV];

  // Lane i (and i + 32): what the page table says for key i of the block at j0,
  // or -1 past the end.  One load whatever the lanes need, and nothing here
  // looks at its result: it is on its way until known_pages.
  static __device__ __forceinline__ int32_t load_pages(const AttnParams& p, const Work& w, uint32_t lane, uint32_t end,
                                                       uint32_t j0) {
    const uint32_t j = j0 + (lane & 31u), at = j >> p.page_shift;
    uint64_t x = (uint64_t)(j < end && at < w.n_pages ? w.pages + at : (pages_t)&g_no_page);
    asm volatile("" : "+v"(x));
    return *(pages_t)x;
  }
  static __device__ __forceinline__ int32_t known_pages(const AttnParams& p, int32_t pages) {
    return (uint32_t)pages < p.a.cache.n_pages ? pages : -1;
  }

  // The block at j0, whose keys' pages are in `pages` and `there` (a bit for
  // each key that has one).  Addresses come from one branch or the other, the
  // loads from neither: the compiler then knows how many are on their way.
  static __device__ __forceinline__ void load(const AttnParams& p, const Work& w, const void* base,
                                              const int64_t* stride, uint32_t j0, int32_t pages, uint32_t there,
                                              u32x4 (&to)[NV]) {
    const uint32_t lane = fresh_lane();
    const char* x[NV];
    if (p.near_rows && there == ~0u) {  // all there, 16 keys on one page
      const uint32_t off = 2 * (lane / C * (uint32_t)stride[1]);
#pragma unroll
      for (int n = 0; n < NV; ++n)
        x[n] = page_row(p, w, base, stride, j0, n * RPI / 16 * 16, pages) + n * RPI % 16 * stride[1] * 2 + off;
    } else {
#pragma unroll
      for (int n = 0; n < NV; ++n) x[n] = any_row(p, w, base, stride, j0, n * RPI + lane / C, pages);
    }
    const uint32_t d = lane % C * 8;
#pragma unroll
    for (int n = 0; n < NV; ++n) to[n] = load16((d < p.a.cache.dim ? x[n] : (const char*)g_zeros) + d * 2);
  }
  // Read once: without the hint that says so, 6.1 instead of 6.8 TB/s for the
  // loads alone.
  static __device__ __forceinline__ u32x4 load16(const char* x) {
    return __builtin_nontemporal_load((const __attribute__((address_space(1))) u32x4*)(uint64_t)x);
  }
  // Row r0 of the block (the same in all lanes), or a row of each lane's own
  // (the zeros, when it has no page).
  static __device__ __forceinline__ const char* page_row(const AttnParams& p, const Work& w, const void* base,
                                                         const int64_t* stride, uint32_t j0, uint32_t r0, int32_t pages) {
    return (const char*)((const T*)base + (int64_t)__builtin_amdgcn_readlane(pages, r0) * stride[0] +
                         (int64_t)((j0 + r0) & (p.a.cache.page - 1)) * stride[1] + (int64_t)w.head * stride[2]);
  }
  static __device__ __forceinline__ const char* any_row(const AttnParams& p, const Work& w, const void* base,
                                                        const int64_t* stride, uint32_t j0, uint32_t r, int32_t pages) {
    const int32_t page = __shfl(pages, (int)r);
    const T* x = (const T*)base + (int64_t)page * stride[0] + (int64_t)((j0 + r) & (p.a.cache.page - 1)) * stride[1] +
                 (int64_t)w.head * stride[2];
    return page < 0 ? (const char*)g_zeros : (const char*)x;
  }
};

template <int NR, typename T, int DP>
__device__ __forceinline__ void run_stream(const AttnParams& p, const Work& w, T* s_kv, float* s_ml, float* stats,
                                           float* sums) {
  using S = Stream<T, DP>;
  const gts_attention_args& a = p.a;
  const uint32_t lane = fresh_lane(), wave = uni(threadIdx.x >> 6), quarter = lane / 16;
  const float scale = a.scale;
  const float c = scale == 0.f ? 1.f : __builtin_fabsf(scale) * kLog2e;
  const uint32_t begin = w.tile * kTile;
  const uint32_t end = begin + w.n_tiles * kTile < w.keys ? begin + w.n_tiles * kTile : w.keys;
  T* sk = s_kv + wave * 2 * kBlock * DP;  // this wave's block of keys, then of values
  T* sv = sk + kBlock * DP;

  S st;
  uint32_t j0 = begin + wave * kBlock;
  int32_t pages = S::load_pages(p, w, lane, end, j0);  // of the block to load next
  int32_t later = S::load_pages(p, w, lane, end, j0 + 4 * kBlock);
  pages = S::known_pages(p, pages);
  uint32_t there = (uint32_t)__ballot(pages >= 0);  // keys of the block in k and v
  S::load(p, w, a.cache.k, a.cache.k_stride, j0, pages, there, st.k);
  S::load(p, w, a.cache.v, a.cache.v_stride, j0, pages, there, st.v);
  pages = later;

  Vec8<T> q[S::KK][NR];
  f32x4 o[S::DB][NR];
  float m[NR], l[NR];
  uint32_t sees[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const uint32_t row = r * 16 + lane % 16;
    const bool valid = row < w.rows;
    const uint32_t flat = w.first_row + (valid ? row : 0);
    const uint32_t token = p.by_group.div(flat), gq = flat - token * p.group;
    // scale's sign (and 0) go into the queries: the maximum of q.k is then
    // that of the scaled scores
    const T* x = (const T*)a.q + (int64_t)token * a.q_stride[0] + (int64_t)(w.head * p.group + gq) * a.q_stride[1];
#pragma unroll
    for (int kk = 0; kk < S::KK; ++kk) {
      const uint32_t d = kk * 32 + quarter * 8;
      const bool in = valid && d < a.cache.dim && scale != 0.f;
      u32x4 y = *(const u32x4*)(in ? x + d : (const T*)g_zeros);
      if (scale < 0.f) y ^= u32x4{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
      q[kk][r] = __builtin_bit_cast(Vec8<T>, y);
    }
    sees[r] = w.keys;
    if (w.own && valid) {
      const int64_t n = w.see + token;
      sees[r] = n < 0 ? 0 : n < (int64_t)w.keys ? (uint32_t)n : w.keys;
    }
    m[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int d = 0; d < S::DB; ++d) o[d][r] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __syncthreads();  // LDS of the stretch before is free

  for (; j0 < end; j0 += 4 * kBlock) {
    // the page numbers of the block after next are asked for first: waiting for
    // them later leaves the loads behind them on their way
    const uint32_t lane = fresh_lane(), quarter = lane / 16;
    later = S::load_pages(p, w, lane, end, j0 + 8 * kBlock);
    const uint32_t here = there;
    pages = S::known_pages(p, pages);
    there = (uint32_t)__ballot(pages >= 0);
    const uint32_t next = j0 + 4 * kBlock;
#pragma unroll
    for (int n = 0; n < S::NV; ++n) {
      const uint32_t row = n * S::RPI + lane / S::C;
      *(u32x4*)(sk + row * DP + ((lane % S::C) ^ S::swizzle_k(row)) * 8) = st.k[n];
    }
    __builtin_amdgcn_sched_barrier(0);
    S::load(p, w, a.cache.k, a.cache.k_stride, next, pages, there, st.k);
    __builtin_amdgcn_sched_barrier(0);
    f32x4 s[2][NR];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int r = 0; r < NR; ++r) s[t][r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < S::KK; ++kk) {
        const uint32_t row = lane % 16;
        const Vec8<T> x =
            *(const Vec8<T>*)(sk + (t * 16 + row) * DP + (quarter ^ S::swizzle_k(row) ^ (4 * kk)) * 8);
#pragma unroll
        for (int r = 0; r < NR; ++r) s[t][r] = mfma16(x, q[kk][r], s[t][r]);
      }
    }
    // values to LDS; one that is not finite matters where some rows do not see
    // every key
    const bool edge = j0 + kBlock > w.low, mask = edge || here != ~0u;
    bool odd = false;
    if (edge && w.low < w.keys) {
#pragma unroll
      for (int n = 0; n < S::NV; ++n) odd |= any_not_finite<T>(st.v[n]);
      odd = __any(odd);
      if (odd) {
#pragma unroll
        for (int n = 0; n < S::NV; ++n) st.v[n] = finite_only<T>(st.v[n]);
      }
    }
#pragma unroll
    for (int n = 0; n < S::NV; ++n) {
      const uint32_t row = n * S::RPI + lane / S::C;
      *(u32x4*)(sv + row * DP + ((lane % S::C) ^ S::swizzle_v(row)) * 8) = st.v[n];
    }
    __builtin_amdgcn_sched_barrier(0);
    S::load(p, w, a.cache.v, a.cache.v_stride, next, pages, there, st.v);
    pages = later;
    __builtin_amdgcn_sched_barrier(0);

    Vec8<T> pw[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      if (mask) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t key = i / 4 * 16 + 4 * quarter + i % 4;
          s[i / 4][r][i % 4] = j0 + key < sees[r] && (here >> key & 1) ? s[i / 4][r][i % 4] : -INFINITY;
        }
      }
      float mx = s[0][r][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[i / 4][r][i % 4]);
      mx = max_quarters(mx);
      // as in Rows::step
      if (__any((mx - m[r]) * c > 8.f || (m[r] == -INFINITY && mx > m[r]))) {
        const float m1 = fmaxf(m[r], mx);
        const float alpha = m[r] == -INFINITY ? 0.f : exp2_((m[r] - m1) * c);
        l[r] *= alpha;
#pragma unroll
        for (int d = 0; d < S::DB; ++d) o[d][r] *= alpha;
        m[r] = m1;
      }
      const float base = m[r] == -INFINITY ? 0.f : -m[r] * c;
      float sum = 0.f;
      // rounded and summed as in Rows::step
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float e = exp2_(__builtin_fmaf(s[i / 4][r][i % 4], c, base));
        sum += e;
        pw[r][i] = (T)e;
      }
      l[r] += sum;
    }
    // Values of 8 keys at one dim: keys 4 quarter .. + 3 and 16 further.
    const uint32_t vr = 4 * quarter + lane % 16 / 4;
    const T* va = sv + vr * DP + lane % 2 * 4;
    const uint32_t vc = lane % 4 / 2 ^ S::swizzle_v(vr);
    typedef __attribute__((address_space(3))) i16x4* lds_t;
    const auto turned = [&](int d) {
      union {
        i16x4 h[2];
        Vec8<T> v;
      } u;
      const T* x = va + (vc ^ (2 * d)) * 8;
      u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)x);
      u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(x + 16 * DP));
      return u.v;
    };
#pragma unroll
    for (int d = 0; d < S::DB; ++d) {
      const Vec8<T> x = turned(d);
#pragma unroll
      for (int r = 0; r < NR; ++r) o[d][r] = mfma16(x, pw[r], o[d][r]);
    }
    if (odd) {
#pragma unroll 1
      for (uint32_t j = j0; j < j0 + kBlock; ++j) {
        const T* x = value_row<T>(p, w, j);
        if (!x) continue;
#pragma unroll
        for (int d = 0; d < S::DB; ++d) {
          const uint32_t at = d * 16 + 4 * quarter;
          if (at >= a.cache.dim) continue;
          const Pack<T, 4> y = *(const Pack<T, 4>*)(x + at);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < NR; ++r)
              if (not_finite((float)y.v[i]) && j < sees[r]) o[d][r][i] += (float)y.v[i];
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }

  // the four waves' sums, rows in order, joined by all threads
  __syncthreads();
  float* mine = (float*)s_kv + wave * (NR * 16) * DP;
  static_assert(4 * NR * 16 * DP * 4 <= 4 * kTile * DP * sizeof(T), "the sums fit the tiles' LDS");
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const uint32_t row = r * 16 + lane % 16;
    const float sum = add_quarters(l[r]);
    if (row < w.rows) {
      if (quarter == 0) {
        s_ml[(wave * 32 + row) * 2] = m[r];
        s_ml[(wave * 32 + row) * 2 + 1] = sum;
      }
#pragma unroll
      for (int d = 0; d < S::DB; ++d) *(f32x4*)(mine + row * DP + ((d * 4 + quarter) ^ (row & 15)) * 4) = o[d][r];
    }
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < w.rows * (DP / 4); i += 256) {
    const uint32_t row = i / (DP / 4), d = i % (DP / 4);
    if (d * 4 >= a.cache.dim) continue;
    float mw[4], top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      mw[x] = s_ml[(x * 32 + row) * 2];
      top = fmaxf(top, mw[x]);
    }
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float f = mw[x] == -INFINITY ? 1.f : exp2_((mw[x] - top) * c);
      sum += s_ml[(x * 32 + row) * 2 + 1] * f;
      acc += *(const f32x4*)((float*)s_kv + (x * NR * 16 + row) * DP + (d ^ (row & 15)) * 4) * f;
    }
    const uint64_t at = w.part + row;
    *(f32x4*)(sums + at * a.cache.dim + d * 4) = acc;
    if (d == 0) *(float2*)(stats + 2 * at) = make_float2(top * c, sum);  // base 2 from here on
  }
}

// Of a segment's tiles [from, to), whose places begin at seg, those that a
// stretch from place t to place stop has: tile i begins at seg +
// segment_places + (i - from) * tile_places, and is the stretch's in which it
// begins.
__device__ __forceinline__ void cut_tiles(uint64_t t, uint64_t stop, uint64_t seg, uint32_t rg, uint32_t& from,
                                          uint32_t& to) {
  const uint32_t each = tile_places(rg);
  const uint64_t zero = seg + segment_places(rg);
  const uint64_t a = t > zero ? (t - zero + each - 1) / each : 0, b = stop > zero ? (stop - zero + each - 1) / each : 0;
  const uint32_t n = to - from;
  to = from + (uint32_t)(b < n ? b : n);
  from += (uint32_t)(a < n ? a : n);
}

template <typename T, int DP>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void tile_kernel(AttnParams p) {
  const gts_attention_args& a = p.a;
  const uint32_t B = a.batch.batch, hkv = a.cache.heads, P = a.cache.n_pages ? a.batch.prefix_len : 0;
  __shared__ __align__(16) T s_kv[4 * kTile * DP];
  __shared__ uint64_t s_sum[256];
  __shared__ uint64_t s_wave[4];
  __shared__ __align__(8) Flags s_flags;
  __shared__ __align__(8) float s_ml[4 * 32 * 2];
  const uint32_t tid = threadIdx.x, lane = tid & 63u;

  // The plan: places of every sequence, summed.  Thread i takes sequences
  // [i per, (i + 1) per).
  const uint32_t per_thread = (B + 255) / 256;
  const uint32_t prows = a.batch.tokens * p.group;
  const uint32_t prg = row_groups(prows), n_prt = (prows + 32 * prg - 1) / (32 * prg);
  const uint32_t ptiles = (P + kTile - 1) / kTile;
  // pieces of the prefix: piece i is part i / n_prt of segment i % n_prt
  const uint32_t whole = P ? p.whole : 0, line_piece = whole * p.cuts;  // the first in the line
  const uint64_t piece_places = places((ptiles + p.pieces - 1) / p.pieces, prg);
  const uint64_t prefix_places = P ? piece_places * (n_prt * p.pieces - line_piece) : 0;
  uint64_t mine = 0;
  for (uint32_t i = 0; i < per_thread; ++i) {
    const uint32_t b = tid * per_thread + i;
    if (b < B) mine += seq_places(p, load_seq(p, b));
  }
  uint64_t scan = mine;
  for (int i = 1; i < 64; i <<= 1) {
    const uint64_t x = __shfl_up(scan, i);
    if ((int)lane >= i) scan += x;
  }
  if (lane == 63) s_wave[tid >> 6] = scan;
  __syncthreads();
  uint64_t before = prefix_places;
  for (uint32_t i = 0; i < tid >> 6; ++i) before += s_wave[i];
  s_sum[tid] = before + scan - mine;  // first place of this thread's sequences
  const uint64_t total = uni(prefix_places + s_wave[0] + s_wave[1] + s_wave[2] + s_wave[3]);
  // at least a tile's: then every stretch between a segment's first and last
  // tile begins one
  uint64_t per = (total + p.cuts - 1) / p.cuts;
  if (per < kLeastStretch) per = kLeastStretch;
  const uint64_t rows = (uint64_t)a.batch.tokens * a.q_heads;
  const uint64_t cut_rows = (uint64_t)p.part_rows * p.cuts;  // of a head
  const Scratch sc = scratch_layout(B, rows, cut_rows * hkv, a.cache.dim);
  char* scratch = (char*)a.scratch;
  if (blockIdx.x == 0) {
    uint64_t t = s_sum[tid];
    for (uint32_t i = 0; i < per_thread; ++i) {
      const uint32_t b = tid * per_thread + i;
      if (b >= B) break;
      ((uint64_t*)(scratch + sc.begin))[b] = t;
      t += seq_places(p, load_seq(p, b));
    }
    if (tid == 0) *(Plan*)scratch = Plan{per, 1.0 / (double)per};
  }
  __syncthreads();

  // Workgroups go round the eight XCDs: each takes a run of the (head, stretch)
  // pairs, so that rows which share keys also share an L2, and the heads of a
  // token are read at the same time (taking the heads in turn reads 4 % slower).
  const uint32_t xcd = blockIdx.x & 7u, share = gridDim.x / 8, extra = gridDim.x % 8;
  const uint32_t id = xcd * share + (xcd < extra ? xcd : extra) + (blockIdx.x >> 3);
  const uint32_t head = id / p.cuts, g = id - head * p.cuts;
  uint64_t t = (uint64_t)g * per, end = t + per;
  if (end > total) end = total;
  uint32_t dealt = 0;
  while (dealt < whole || t < end) {
    Work w;
    uint64_t stop = t;   // place behind what is done of the line
    uint32_t from, to;   // tiles of the segment
    if (dealt < whole || t < prefix_places) {
      const uint32_t piece = dealt < whole ? dealt * p.cuts + g : line_piece + (uint32_t)(t / piece_places);
      const uint32_t j = piece / n_prt, rt = piece - j * n_prt;
      w.pages = (pages_t)a.prefix_pages;
      w.n_pages = a.n_prefix_pages;
      w.keys = w.low = P;
      w.rg = prg;
      w.first_row = rt * 32 * prg;
      w.rows = prows - w.first_row < 32 * prg ? prows - w.first_row : 32 * prg;
      w.own = false;
      w.see = 0;
      w.part = (uint64_t)j * prows + w.first_row;
      from = (uint32_t)((uint64_t)ptiles * j / p.pieces);
      to = (uint32_t)((uint64_t)ptiles * (j + 1) / p.pieces);
      if (dealt < whole) {
        ++dealt;
      } else {
        const uint64_t seg = (uint64_t)(piece - line_piece) * piece_places;
        stop = seg + piece_places < end ? seg + piece_places : end;
        cut_tiles(t, stop, seg, w.rg, from, to);
        w.part += (uint64_t)p.part_rows * g;
      }
    } else {
      // the last thread whose sequences start at or before t, then its
      // sequences one by one (one, up to 256 sequences)
      uint32_t who = 0;
      for (uint32_t i = 0; i < 4; ++i) who += (uint32_t)__popcll(__ballot(s_sum[i * 64 + lane] <= t));
      who = uni(who - 1);
      uint32_t b = who * per_thread;
      uint64_t first = uni(s_sum[who]);
      Seq s = load_seq(p, b < B ? b : B - 1);
      for (uint32_t i = 1; i < per_thread && t >= first + seq_places(p, s); ++i) {
        first += seq_places(p, s);
        s = load_seq(p, ++b);
      }
      w.rg = row_groups(s.n * p.group);
      uint32_t rt = 0, tiles = own_tiles(p, s, w.rg, 0);
      uint64_t seg = first;
      while (t >= seg + places(tiles, w.rg)) {
        seg += places(tiles, w.rg);
        tiles = own_tiles(p, s, w.rg, ++rt);
      }
      const uint32_t srows = s.n * p.group, r0 = rt * 32 * w.rg;
      w.pages = (pages_t)(a.batch.page_table + (int64_t)b * a.batch.table_stride);
      w.n_pages = a.batch.max_pages;
      w.rows = srows - r0 < 32 * w.rg ? srows - r0 : 32 * w.rg;
      w.first_row = s.first * p.group + r0;
      w.low = seen(s, p.by_group.div(r0));
      w.keys = seen(s, p.by_group.div(r0 + w.rows - 1));
      w.own = true;
      w.see = s.len - s.n + 1 - (int64_t)s.first;
      w.part = (uint64_t)p.pieces * prows + s.first * p.group + r0 + (uint64_t)p.part_rows * g;
      stop = seg + places(tiles, w.rg) < end ? seg + places(tiles, w.rg) : end;
      from = 0;
      to = tiles;
      cut_tiles(t, stop, seg, w.rg, from, to);
    }
    w.head = head;
    if (to > from) {
      // the same in all lanes: kept in scalar registers
      w.pages = (pages_t)uni((uint64_t)w.pages);
      w.n_pages = uni(w.n_pages);
      w.keys = uni(w.keys);
      w.low = uni(w.low);
      w.head = uni(w.head);
      w.rg = uni(w.rg);
      w.rows = uni(w.rows);
      w.first_row = uni(w.first_row);
      w.see = (int64_t)uni((uint64_t)w.see);
      w.part = uni((uint64_t)(w.part + head_partials(prows, cut_rows) * head));
      w.tile = uni(from);
      w.n_tiles = uni(to - from);
      float *stats = (float*)(scratch + sc.stats), *sums = (float*)(scratch + sc.sums);
      // 32 rows of 256 values do not fit the stream's registers: half the tile
      // path's rows stay empty
      if (DP > 128 && w.rows > 16 && w.rg == 1) w.rg = 2;
      if (w.rg > 1) {
        run_stretch<T, DP>(p, w, s_kv, &s_flags, stats, sums);
      } else if (w.rows <= 16) {
        run_stream<1, T, DP>(p, w, s_kv, s_ml, stats, sums);
      } else {
        if constexpr (DP <= 128) run_stream<2, T, DP>(p, w, s_kv, s_ml, stats, sums);
      }
    }
    t = uni(stop);
  }
}

// Whether a page holds one of keys 0 .. keys - 1.  All 64 lanes, 64 pages a load.
__device__ __forceinline__ bool any_page(const AttnParams& p, pages_t pages, uint32_t n, uint32_t keys) {
  for (uint32_t first = 0; (uint64_t)first << p.page_shift < keys; first += 64) {
    const uint32_t at = first + (threadIdx.x & 63u);
    const bool in = at < n && (uint64_t)at << p.page_shift < keys;
    if (__any(in && (uint32_t)pages[at] < p.a.cache.n_pages)) return true;
  }
  return false;
}
// Whether new token t sees a key: what a row whose weights are all zero is asked.
// With a key (their scores are all -inf) it is 0 / 0; without one it is zeros.
__device__ __forceinline__ bool sees_key(const AttnParams& p, uint32_t t) {
  const gts_kv_batch& kb = p.a.batch;
  uint32_t seq, index, count;
  if (!find_sequence(kb, t, &seq, &index, &count)) return false;
  return any_page(p, (pages_t)p.a.prefix_pages, p.a.n_prefix_pages, kb.prefix_len) ||
         any_page(p, (pages_t)(kb.page_table + (int64_t)seq * kb.table_stride), kb.max_pages,
                  seen(load_seq(p, seq), index));
}

// The sequence of new token t, the token's number in it and the first of its
// places; false when no sequence has it.  Up to 63 sequences: one load of each kind
// whose latencies pass together, instead of one behind the other.
__device__ __forceinline__ bool find_places(const AttnParams& p, const uint64_t* begin, uint32_t t, Seq* s, uint32_t* index,
                                            uint64_t* place) {
  const gts_kv_batch& kb = p.a.batch;
  const uint32_t lane = threadIdx.x & 63u;
  if (!kb.starts || kb.batch > 63) {
    uint32_t seq, count;
    if (!find_sequence(kb, t, &seq, index, &count)) return false;
    *s = load_seq(p, seq);
    *place = begin[seq];
    return true;
  }
  const bool in = lane < kb.batch;
  const int32_t start = lane <= kb.batch ? kb.starts[lane] : 0, len = in ? kb.lens[lane] : 0;
  const uint64_t first = in ? begin[lane] : 0;
  const uint64_t m = __ballot(lane == 0 || (lane <= kb.batch && start <= (int32_t)t));
  const uint32_t seq = 63u - (uint32_t)__builtin_clzll(m);
  if (seq >= kb.batch) return false;
  *s = make_seq(p, __builtin_amdgcn_readlane(start, seq), __builtin_amdgcn_readlane(start, seq + 1),
                __builtin_amdgcn_readlane(len, seq));
  if (t < s->first || t >= s->first + s->n) return false;
  *index = t - s->first;
  *place = (uint64_t)__builtin_amdgcn_readlane((uint32_t)(first >> 32), seq) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((uint32_t)first, seq);
  return true;
}

// The join: a wavefront takes ROWS rows, W lanes each.  Lane i of a row takes the
// maximum and sum of partial i, then all of them add up the partials, four dims
// each (ND times).  Bound by its chain of loads (place, then statistics and
// sums together), so with many rows a wave takes four: query heads of one token
// and key-value head, which have one place.
template <int N>
struct Ahead {
  static constexpr int n = N;
};
template <typename T, int ND, int ROWS>
__global__ __launch_bounds__(256) void join_kernel(AttnParams p) {
  constexpr uint32_t W = 64 / ROWS;
  const gts_attention_args& a = p.a;
  const uint32_t lane = threadIdx.x & 63u, sub = lane / W, li = lane % W;
  const uint32_t rows = a.batch.tokens * a.q_heads, row = uni(((uint32_t)block_number() * 4 + (threadIdx.x >> 6)) * ROWS);
  if (row >= rows) return;
  const uint32_t t = p.by_q_heads.div(row), hq = row - t * a.q_heads;
  const uint32_t head = p.by_group.div(hq), gq = hq - head * p.group, D = a.cache.dim;
  const uint32_t prows = a.batch.tokens * p.group;  // of a head
  const uint64_t cut_rows = (uint64_t)p.part_rows * p.cuts;
  const Scratch sc = scratch_layout(a.batch.batch, rows, cut_rows * a.cache.heads, D);
  const char* scratch = (const char*)a.scratch;
  const Plan plan = *(const Plan*)scratch;
  const float* stats = (const float*)(scratch + sc.stats);
  const float* sums = (const float*)(scratch + sc.sums);

  // Three runs of partials, each count[] rows from at[] on, step[] apart: the
  // pieces of the prefix that were dealt out, one in the line (of a row's pieces
  // at most one is, when any are dealt out), and the own keys.
  uint32_t count[3] = {0, 0, 0};
  uint64_t at[3] = {0, 0, 0}, step[3] = {prows, p.part_rows, p.part_rows};
  Seq s;
  uint32_t index;
  uint64_t place;
  if (find_places(p, (const uint64_t*)(scratch + sc.begin), t, &s, &index, &place)) {
    const uint64_t base = head_partials(prows, cut_rows) * head;
    const uint32_t P = a.cache.n_pages ? a.batch.prefix_len : 0;
    const auto locate = [&](int run, uint64_t place, uint32_t tiles, uint32_t rg, uint64_t x) {
      if (tiles == 0) return;
      place += segment_places(rg);
      const uint32_t first = plan.group_of(place);
      count[run] = plan.group_of(place + (uint64_t)(tiles - 1) * tile_places(rg)) - first + 1;
      at[run] = base + x + (uint64_t)p.part_rows * first;
    };
    if (P) {
      const uint32_t ptiles = (P + kTile - 1) / kTile, rg = row_groups(prows), n_rt = (prows + 32 * rg - 1) / (32 * rg);
      const uint32_t r = t * p.group + gq, rt = r / (32 * rg), line = p.whole * p.cuts;
      // piece j of this row has number j n_rt + rt; those below `line` were dealt out
      const uint32_t dealt = line > rt ? (line - rt + n_rt - 1) / n_rt : 0;
      count[0] = dealt < p.pieces ? dealt : p.pieces;
      at[0] = base + r;
      if (count[0] < p.pieces) {
        const uint32_t j = count[0];
        const uint32_t tiles = (uint32_t)((uint64_t)ptiles * (j + 1) / p.pieces - (uint64_t)ptiles * j / p.pieces);
        locate(1, places((ptiles + p.pieces - 1) / p.pieces, rg) * (j * n_rt + rt - line), tiles, rg,
               (uint64_t)j * prows + r);
      }
    }
    if (s.keys) {
      const uint32_t rg = row_groups(s.n * p.group), r = index * p.group + gq, rt = r / (32 * rg);
      if (rt) {  // behind rt segments: 64 at a time (8 x 4096 tokens have 128 a sequence)
        uint64_t before = 0;
        for (uint32_t i = lane; i < rt; i += 64) before += places(own_tiles(p, s, rg, i), rg);
        for (int k = 32; k; k >>= 1) before += __shfl_xor(before, k);
        place += uni(before);
      }
      locate(2, place, own_tiles(p, s, rg, rt), rg, (uint64_t)p.pieces * prows + s.first * p.group + r);
    }
  }
  const uint32_t n01 = count[0] + count[1], n = n01 + count[2];
  const auto part = [&](uint32_t i) {
    return i < count[0] ? at[0] + step[0] * i : i < n01 ? at[1] + step[1] * (i - count[0]) : at[2] + step[2] * (i - n01);
  };

  float m = -INFINITY, l = 0.f;
  f32x4 o[ND] = {};
  for (uint32_t i0 = 0; i0 < n; i0 += W) {
    const uint32_t here = n - i0 < W ? n - i0 : W;
    float mi = -INFINITY, sum = 0.f;
    if (li < here) {
      const float2 x = *(const float2*)(stats + 2 * (part(i0 + li) + sub));
      mi = x.x;
      sum = x.y;
    }
    float f = 0.f;  // weight of partial i0 + li
    const auto weigh = [&] {
      float m1 = mi;
      for (int k = W / 2; k; k >>= 1) m1 = fmaxf(m1, __shfl_xor(m1, k));
      m1 = fmaxf(m1, m);
      f = mi == -INFINITY ? 1.f : exp2_(mi - m1);
      const float old = m == -INFINITY ? 1.f : exp2_(m - m1);
      sum *= f;
      for (int k = W / 2; k; k >>= 1) sum += __shfl_xor(sum, k);
      l = l * old + sum;
      m = m1;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] *= old;
    };
    // A loads of the sums on their way, the first of them before the weights are
    // known.  Past the end the last once more, left out of the sum: a branch
    // around a load would make the next one wait for it.
    const auto add_up = [&](auto ahead) {
      constexpr int A = decltype(ahead)::n;
      for (uint32_t k0 = 0; k0 < here; k0 += A) {
        f32x4 v[A][ND];
#pragma unroll
        for (int y = 0; y < A; ++y) {
          const float* src = sums + (part(i0 + (k0 + y < here ? k0 + y : here - 1)) + sub) * D;
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            const uint32_t c = (d * W + li) * 4;
            v[y][d] = *(const f32x4*)(src + (c < D ? c : 0));
          }
        }
        if (k0 == 0) weigh();
#pragma unroll
        for (int y = 0; y < A; ++y) {
          if (k0 + y >= here) break;
          const float w = ROWS == 1 ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), k0 + y))
                                    : __shfl(f, (int)(sub * W + k0 + y));
#pragma unroll
          for (int d = 0; d < ND; ++d) o[d] += v[y][d] * w;
        }
      }
    };
    if (here <= 2)
      add_up(Ahead<2>{});
    else
      add_up(Ahead<8 / ND>{});
  }
  float inv = 1.f / l;
  if (__any(l == 0.f)) {
    const float none = sees_key(p, t) ? __builtin_nanf("") : 0.f;
    if (l == 0.f) inv = none;
  }
  T* out = (T*)a.out + (int64_t)t * a.out_stride[0] + (int64_t)(hq + sub) * a.out_stride[1];
#pragma unroll
  for (int d = 0; d < ND; ++d) {
    const uint32_t c = (d * W + li) * 4;
    if (c >= D) continue;
    const f32x4 y = o[d] * inv;
    // rows of the output are aligned to four bytes at least
    *(Pack<T, 2>*)(out + c) = Pack<T, 2>{(T)y[0], (T)y[1]};
    *(Pack<T, 2>*)(out + c + 2) = Pack<T, 2>{(T)y[2], (T)y[3]};
  }
  if (a.lse && li == 0) a.lse[row + sub] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

template <typename T>
void launch_join(const AttnParams& p, hipStream_t stream) {
  const uint64_t rows = (uint64_t)p.a.batch.tokens * p.a.q_heads;
  const dim3 one = grid_of((rows + 3) / 4), four = grid_of((rows + 15) / 16), block(256);
  if (p.group % 4 == 0 && rows >= kFourRows) {
    if (p.a.cache.dim <= 64)
      join_kernel<T, 1, 4><<<four, block, 0, stream>>>(p);
    else if (p.a.cache.dim <= 128)
      join_kernel<T, 2, 4><<<four, block, 0, stream>>>(p);
    else
      join_kernel<T, 4, 4><<<four, block, 0, stream>>>(p);
  } else {
    join_kernel<T, 1, 1><<<one, block, 0, stream>>>(p);
  }
}

// ---- the row kernel --------------------------------------------------------------

template <typename T>
__global__ __launch_bounds__(256) void row_kernel(AttnParams p) {
  const gts_attention_args& a = p.a;
  __shared__ float s_q[4][GTS_OPS_MAX_ATTN];
  const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63u;
  const uint64_t row = block_number() * 4 + wave;
  if (row >= (uint64_t)a.batch.tokens * a.q_heads) return;
  const uint32_t t = (uint32_t)(row / a.q_heads), hq = (uint32_t)(row % a.q_heads), h = hq / p.group;
  const uint32_t D = a.cache.dim;
  uint32_t seq = 0, index = 0, count = 0;
  const bool has = find_sequence(a.batch, t, &seq, &index, &count);
  const uint32_t own = has ? seen(load_seq(p, seq), index) : 0;
  const uint32_t n_prefix = has && a.cache.n_pages ? a.batch.prefix_len : 0;
  const T* q = (const T*)a.q + (int64_t)t * a.q_stride[0] + (int64_t)hq * a.q_stride[1];
  for (uint32_t d = lane; d < D; d += 64) s_q[wave][d] = (float)q[d];
  float m = -INFINITY, l = 0.f, o[GTS_OPS_MAX_ATTN / 64] = {};
  const float scale = a.scale * kLog2e;
  for (int part = 0; part < 2; ++part) {
    const uint32_t n = part ? own : n_prefix;
    const pages_t pages = (pages_t)(part ? a.batch.page_table + (int64_t)seq * a.batch.table_stride : a.prefix_pages);
    const uint32_t n_pages = part ? a.batch.max_pages : a.n_prefix_pages;
    for (uint32_t j0 = 0; j0 < n; j0 += 64) {
      const uint32_t j = j0 + lane;
      const int32_t page = j < n ? key_page(a, pages, n_pages, p.page_shift, j) : -1;
      const uint32_t slot = j & (a.cache.page - 1);
      float s = -INFINITY;
      if (page >= 0) {
        const T* k = (const T*)a.cache.k + (int64_t)page * a.cache.k_stride[0] + (int64_t)slot * a.cache.k_stride[1] +
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
        const int64_t pj = __shfl(page, src);
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
  float inv = 1.f / l;
  if (l == 0.f) inv = sees_key(p, t) ? __builtin_nanf("") : 0.f;  // the same in all lanes
  T* out = (T*)a.out + (int64_t)t * a.out_stride[0] + (int64_t)hq * a.out_stride[1];
#pragma unroll
  for (uint32_t i = 0; i < GTS_OPS_MAX_ATTN / 64; ++i) {
    const uint32_t d = i * 64 + lane;
    if (d < D) out[d] = (T)(o[i] * inv);
  }
  if (a.lse && lane == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

}  // namespace

// Rows that a cut may add: a segment's, at most all rows of a head.
static uint32_t part_rows(uint32_t tokens, uint32_t group) {
  const uint64_t rows = (uint64_t)tokens * group;
  return rows > 64 ? kMostRows : rows > 32 ? 64 : 32;
}

// Stretches of a head: two workgroups a CU (one with the largest heads, which
// take all of its LDS) over all heads, at least one each.
static uint32_t cuts(uint32_t kv_heads, uint32_t dim) {
  const uint32_t n = (dim > 128 ? kGroups / 2 : kGroups) / kv_heads;
  return n ? n : 1;
}

uint64_t attention_scratch(uint32_t batch, uint32_t tokens, uint32_t q_heads, uint32_t kv_heads, uint32_t dim) {
  return scratch_layout(batch, (uint64_t)tokens * q_heads,
                        (uint64_t)part_rows(tokens, q_heads / kv_heads) * cuts(kv_heads, dim) * kv_heads, dim)
      .bytes;
}

// How the prefix is dealt out: segments whole where there are more than
// workgroups, else in the fewest equal pieces that give each workgroup one, if
// those are 8 tiles or more (shorter ones cost more to begin than they save).
// pieces * segments is below workgroups + segments, so that what is left over
// for the line is less than a piece of each segment.
static void deal_prefix(AttnParams& p) {
  const uint32_t rows = p.a.batch.tokens * p.group, rg = row_groups(rows), n = (rows + 32 * rg - 1) / (32 * rg);
  const uint32_t tiles = (p.a.batch.prefix_len + kTile - 1) / kTile;
  p.pieces = 1;
  if (n > 1 && n < p.cuts && tiles / ((p.cuts + n - 1) / n) >= 8) p.pieces = (p.cuts + n - 1) / n;
  p.whole = n > 1 && tiles ? n * p.pieces / p.cuts : 0;
}

// The tile kernel's loads: 16-bit values, every row of q, k and v and every 16
// bytes of it aligned to 16 bytes.
static bool tiles_fit(const gts_attention_args& a) {
  const gts_kv_cache& c = a.cache;
  if (c.dtype == GTS_F32 || c.dim % 8 != 0) return false;
  uint64_t bits = ((uint64_t)a.out_stride[0] | (uint64_t)a.out_stride[1]) % 2;
  for (int i = 0; i < 3; ++i) bits |= (uint64_t)c.k_stride[i] | (uint64_t)c.v_stride[i];
  for (int i = 0; i < 2; ++i) bits |= (uint64_t)a.q_stride[i];
  const uint64_t addr = (uint64_t)(uintptr_t)a.q | (uint64_t)(uintptr_t)c.k | (uint64_t)(uintptr_t)c.v |
                        (uint64_t)(uintptr_t)a.scratch | (uint64_t)(uintptr_t)a.out % 4 * 4;
  return bits % 8 == 0 && addr % 16 == 0;
}

template <typename T>
static hipError_t launch_typed(AttnParams& p, hipStream_t stream) {
  const gts_attention_args& a = p.a;
  const uint64_t rows = (uint64_t)a.batch.tokens * a.q_heads;
  const dim3 grid = grid_of((rows + 3) / 4), block(256);
  if constexpr (sizeof(T) == 2) {
    if (tiles_fit(a)) {
      p.cuts = cuts(a.cache.heads, a.cache.dim);
      deal_prefix(p);
      const dim3 wgs(p.cuts * a.cache.heads);
      if (a.cache.dim <= 64)
        tile_kernel<T, 64><<<wgs, block, 0, stream>>>(p);
      else if (a.cache.dim <= 128)
        tile_kernel<T, 128><<<wgs, block, 0, stream>>>(p);
      else
        tile_kernel<T, 256><<<wgs, block, 0, stream>>>(p);
      launch_join<T>(p, stream);
      return hipGetLastError();
    }
  }
  row_kernel<T><<<grid, block, 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_attention(const gts_attention_args& a, hipStream_t stream) {
  AttnParams p{};
  p.a = a;
  p.page_shift = (uint32_t)__builtin_ctz(a.cache.page);
  p.group = a.q_heads / a.cache.heads;
  p.by_group = FastDiv(p.group);
  p.by_q_heads = FastDiv(a.q_heads);
  p.part_rows = part_rows(a.batch.tokens, p.group);
  const int64_t far = 1 << 26;  // elements: 16 rows and a chunk stay below 2^31 bytes
  p.near_rows = p.page_shift >= 4 && a.cache.k_stride[1] >= 0 && a.cache.k_stride[1] < far && a.cache.v_stride[1] >= 0 &&
                a.cache.v_stride[1] < far;
  if (a.cache.dtype == GTS_F32) return launch_typed<float>(p, stream);
  if (a.cache.dtype == GTS_BF16) return launch_typed<__bf16>(p, stream);
  return launch_typed<_Float16>(p, stream);
}

}  // namespace gts
