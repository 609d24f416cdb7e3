// What the attention kernels and the rotation of their operands share: argument
// checks, product fragments, the mapping of workgroups to packed segments, and the
// score of a query and a key.
#pragma once

#include "attn_plan.hpp"
#include "nnconv.hpp"

#include <cmath>
#include <initializer_list>
#include <type_traits>

namespace dsmp {

constexpr int MAX_HEADS = 256, MAX_HEAD_DIM = 128;
constexpr int64_t MAX_ROW = (int64_t)1 << 16;   // elements between rows: a tile's rows lie within 32 bits

// Makes the handle's device current for a call's launches.
struct DeviceScope {
  int before = -1;
  explicit DeviceScope(const dsmp_handle* h) {
    int now = -1;
    if (hipGetDevice(&now) == hipSuccess && now != h->device && hipSetDevice(h->device) == hipSuccess) before = now;
  }
  ~DeviceScope() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

struct Matrix {
  const void* p;   // NULL: not there
  int64_t ld, width;
  const char* name;
};

inline dsmp_status check_matrices(dsmp_handle* h, int size, std::initializer_list<Matrix> all) {
  for (const Matrix& m : all) {
    if (!m.p) continue;
    DSMP_CHECK(h, m.ld >= m.width, DSMP_INVALID_ARG, "%s: rows are closer than their values", m.name);
    DSMP_CHECK(h, m.ld <= MAX_ROW, DSMP_UNSUPPORTED, "%s: rows more than %lld elements apart", m.name, (long long)MAX_ROW);
    DSMP_CHECK(h, reinterpret_cast<uintptr_t>(m.p) % 16 == 0 && m.ld * size % 16 == 0, DSMP_INVALID_ARG,
               "%s: rows must be 16-byte aligned", m.name);
  }
  return DSMP_OK;
}

// ------------------------------------------------------------------ fragments
// Eight values of a lane: A[row = l % 32][8 h + e], B[8 h + e][col = l % 32] with h = l / 32,
// 16 deep; the result as in nnconv.hpp.  In float32 eight products 2 deep take element e of
// both halves each, so both types have the same layout.
typedef float f32x8 __attribute__((ext_vector_type(8)));

template <typename T>
struct Frag;
template <>
struct Frag<__bf16> {
  typedef bf16x8 type;
};
template <>
struct Frag<float> {
  typedef f32x8 type;
};

__device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(f32x8 a, f32x8 b, f32x16 c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

// Eight float32 values rounded to the type of the products (to nearest even).
template <typename T>
__device__ __forceinline__ typename Frag<T>::type to_frag(const float* v);
template <>
__device__ __forceinline__ bf16x8 to_frag<__bf16>(const float* v) { return pack_frag<__bf16>(v); }
template <>
__device__ __forceinline__ f32x8 to_frag<float>(const float* v) {
  f32x8 f;
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = v[e];
  return f;
}

// What that rounding left, rounded: the sum of both has 16 bits.
__device__ __forceinline__ bf16x8 rest_frag(const float* v, bf16x8 f) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = v[e] - (float)f[e];
  return to_frag<__bf16>(r);
}

typedef __attribute__((address_space(3))) unsigned char lds_u8;

// A operand from row-major LDS: row r0 + l % 32, values c0 + 8 h + e.
template <typename T>
__device__ __forceinline__ typename Frag<T>::type lds_rows(lds_u8* X, int pitch, int r0, int c0) {
  const int l = threadIdx.x & 63;
  lds_u8* p = X + (r0 + (l & 31)) * pitch + (c0 + 8 * (l >> 5)) * (int)sizeof(T);
  if (sizeof(T) == 4) {
    uint32_t at = (uint32_t)(uintptr_t)p;
    asm volatile("" : "+v"(at));   // formed here: not kept over a loop for each of many calls
    p = (lds_u8*)(uintptr_t)at;
  }
  return *(__attribute__((address_space(3))) typename Frag<T>::type*)p;
}

// A operand from row-major LDS, transposed: A row = column c0 + l % 32, contraction index
// (h, e) = LDS row r0 + 8 (e / 4) + 4 h + e % 4 -- the order in which a lane's eight
// consecutive result registers hold the rows of a 32-row result, which so become the B
// operand as they are.
template <typename T>
__device__ __forceinline__ typename Frag<T>::type lds_columns(lds_u8* X, int pitch, int r0, int c0);
template <>
__device__ __forceinline__ f32x8 lds_columns<float>(lds_u8* X, int pitch, int r0, int c0) {
  const int l = threadIdx.x & 63;
  uint32_t at = (uint32_t)(uintptr_t)(X + (r0 + 4 * (l >> 5)) * pitch + (c0 + (l & 31)) * 4);
  asm volatile("" : "+v"(at));   // as in lds_rows
  lds_u8* p = (lds_u8*)(uintptr_t)at;
  f32x8 f;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    f[e] = *(__attribute__((address_space(3))) float*)(p + (8 * (e / 4) + e % 4) * pitch);
  return f;
}

// Row of register i of a 32-row result.
__device__ __forceinline__ int result_row(int i) { return 8 * (i >> 2) + 4 * ((threadIdx.x & 63) >> 5) + (i & 3); }

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32, 64); }

// LDS pitch of a tile with D values to a row: rows read 16 bytes at a time (ROWS), or in
// transposing reads.
template <typename T, int D, bool ROWS>
constexpr int pitch_of() {
  return D * (int)sizeof(T) + (ROWS || sizeof(T) == 4 ? 16 : 16 * tr_pad_units(D * (int)sizeof(T)));
}

// ------------------------------------------------------------- guarded global reads
// Buffer reads: what begins at or behind `bytes` comes back as zero, in LDS too.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr uint32_t NOWHERE = 0x80000000u;   // an offset behind every tile

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}
__device__ __forceinline__ u32x4 buffer_read(__amdgpu_buffer_rsrc_t r, uint32_t offset) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)offset, 0, 0));
}

// ------------------------------------------------------ tiles of bfloat16 rows in LDS
// Rows of D values without room between them, copied from memory directly (64 lanes write 1,024
// bytes in a row; no registers on the way).  The 16-byte units of row r are permuted by
// XOR with swizzle(r), so that both kinds of reads are free of bank conflicts: 16 rows at the
// same unit at once (tile_rows), and four rows over four units (tile_columns).  LDS has 64 banks of 4
// bytes: a row has 16, 32 or 64 of them, so among 16 rows 4, 8 or all begin at the same bank.
template <int D>
__device__ __forceinline__ int swizzle(int r) {
  if (D == 32) return (r >> 2) & 3;
  if (D == 64) return ((r >> 1) & 1) * 4 + ((r >> 2) & 1) * 2 + ((r >> 3) & 1);
  return (r & 3) * 4 + ((r >> 2) & 3);
}
// what eight rows further on flip in a unit's place
template <int D>
constexpr uint32_t EIGHT_ROWS = 16 * (D == 64 ? 1 : 2);

template <int D, int ROWS>
struct TileCopy {
  static constexpr int RB = 2 * D, UPR = RB / 16, PER = ROWS * UPR / 256, STEP = 256 / UPR;
  static_assert(ROWS * UPR % 256 == 0 && STEP % 16 == 0, "whole loads of a workgroup, rows of one permutation to a lane");
  // a lane's row in its first load, and the unit that it copies there, in bytes
  static __device__ __forceinline__ int row0() { return (int)threadIdx.x / UPR; }
  static __device__ __forceinline__ int unit0() { return ((int)threadIdx.x % UPR ^ swizzle<D>(row0())) * 16; }
  // load i: rows row0 + i STEP, from byte `offset` of the buffer
  static __device__ __forceinline__ void copy(__amdgpu_buffer_rsrc_t from, lds_u8* to, int i, uint32_t offset) {
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(to + (i * 4 + wave) * 1024), 16,
                                             (int)offset, 0, 0, 0);
  }
};

// ------------------------------------------------------------- operands from tiles
// As lds_rows and lds_columns; bfloat16 tiles as above, float32 ones with a pitch of 16 bytes more than a row.
// A lane's place in a bfloat16 tile's first 32 rows: reads of other columns flip bits of it.
struct LanePlace {
  uint32_t rows, columns;
};
template <int D>
__device__ __forceinline__ LanePlace lane_place() {
  const int l = (int)threadIdx.x & 63, g = l >> 4, j = (l >> 2) & 3, q = l & 3, r = l & 31, c = 4 * (g >> 1) + j;
  return {(uint32_t)(r * 2 * D + ((l >> 5) ^ swizzle<D>(r)) * 16),
          (uint32_t)(c * 2 * D + ((2 * (g & 1) + (q >> 1)) ^ swizzle<D>(c)) * 16 + 8 * (q & 1))};
}
// The flipped places are formed where they are used: kept over a loop they would take a register each.
__device__ __forceinline__ void formed_here(LanePlace& p) { asm volatile("" : "+v"(p.rows), "+v"(p.columns)); }

template <typename T, int D>
__device__ __forceinline__ typename Frag<T>::type tile_rows(lds_u8* X, const LanePlace& at, int r0, int t) {
  if constexpr (sizeof(T) == 4) return lds_rows<T>(X, pitch_of<T, D, true>(), r0, 16 * t);
  else return *(__attribute__((address_space(3))) bf16x8*)(X + r0 * 2 * D + (at.rows ^ (uint32_t)(32 * t)));
}
template <typename T, int D>
__device__ __forceinline__ typename Frag<T>::type tile_columns(lds_u8* X, const LanePlace& at, int r0, int c0) {
  if constexpr (sizeof(T) == 4) {
    return lds_columns<T>(X, pitch_of<T, D, true>(), r0, c0);
  } else {
    lds_u8* p = X + r0 * 2 * D + (at.columns ^ (uint32_t)(2 * c0));
    lds_u8* p8 = X + (r0 + 8) * 2 * D + (at.columns ^ ((uint32_t)(2 * c0) ^ EIGHT_ROWS<D>));
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p8);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
}

// A lane's eight values at p (16-byte aligned), or zeros.
template <typename T>
__device__ __forceinline__ typename Frag<T>::type read_frag(const T* p, bool there) {
  typename Frag<T>::type f;
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = (T)0.0f;
  if (there) f = *(const typename Frag<T>::type*)p;
  return f;
}

typedef __attribute__((address_space(3))) u32x4 lds_u32x4;

// Four values of a row of results, rounded.
template <typename T>
__device__ __forceinline__ void store4(T* p, float a, float b, float c, float d) {
  typedef T t4 __attribute__((ext_vector_type(4)));
  t4 v;
  v[0] = (T)a, v[1] = (T)b, v[2] = (T)c, v[3] = (T)d;
  *(t4*)p = v;
}

// A wave's 32 rows of results (D values each, a lane's column), scaled: to `out`, or in float32 to `part`.
template <typename T, int D>
__device__ __forceinline__ void write_rows(const f32x16* acc, float scale, T* out, float* part, int hd) {
  int tid = (int)threadIdx.x;
  asm volatile("" : "+v"(tid));   // what follows from it is formed here, not kept in registers over the caller's loop
  const int h = (tid & 63) >> 5;
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const int c = 32 * d + 8 * i4 + 4 * h;
      if (c >= hd) continue;
      const float v[4] = {acc[d][4 * i4] * scale, acc[d][4 * i4 + 1] * scale, acc[d][4 * i4 + 2] * scale, acc[d][4 * i4 + 3] * scale};
      if (part) *(float4*)(part + c) = make_float4(v[0], v[1], v[2], v[3]);
      else store4(out + c, v[0], v[1], v[2], v[3]);
    }
}

// ------------------------------------------------------------------ segments
struct Bounds {
  const int32_t* ptr;   // NULL: equal segments of `len` rows
  int64_t n, len;
  __device__ __forceinline__ int64_t at(int s) const {
    if (!ptr) return s * len;
    const int64_t v = ptr[s];
    return v < 0 ? 0 : v > n ? n : v;
  }
};

// The segment of tile t, and that segment's first tile.  A segment whose bounds are b
// and e has the tiles from floor(b M / size) + s on, ceil((e - b) M / size) of them, which ends
// at or ahead of the next one's: nothing has to be counted up.  M rows of work stand
// behind each row; sixty-four bounds are looked at at once.
__device__ __forceinline__ int find_segment(const Bounds& b, int n_seg, int M, int size, int64_t t, int64_t* first) {
  const int l = threadIdx.x & 63;
  int lo = 0, count = n_seg;   // the segment is in [lo, lo + count)
  while (count > 1) {
    const int step = (count + 63) / 64, s = lo + l * step;
    const bool le = l * step < count && b.at(s) * M / size + s <= t;
    const int hit = (int)__popcll(__ballot(le));
    lo += (hit > 0 ? hit - 1 : 0) * step;
    count = min(step, n_seg - lo);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  *first = b.at(lo) * M / size + lo;
  return lo;
}

// The same with the segments of the longest other side first (their workgroups take the longest: begun last
// they would run alone at the end), for up to 64 segments, a lane to each.  The tiles of each are counted
// exactly, and a segment's first follows those of all that come before it.  16 segments of 300 to
// 3,800 nodes, the keys' gradients: 575 us in order, 546 longest first.
__device__ __forceinline__ int find_segment_longest_first(const Bounds& b, const Bounds& other, int n_seg, int M, int size, int64_t t,
                                                          int64_t* first) {
  if (n_seg == 1 || n_seg > 64) return find_segment(b, n_seg, M, size, t, first);
  const int l = (int)threadIdx.x & 63;
  int tiles = 0, work = -1;
  if (l < n_seg) {
    const int64_t rows = (b.at(l + 1) - b.at(l)) * M;
    tiles = rows > 0 ? (int)((rows + size - 1) / size) : 0;
    work = (int)min((int64_t)0x7fffffff, max((int64_t)0, other.at(l + 1) - other.at(l)));
  }
  int before = 0;   // tiles of the segments that come before this lane's
  for (int s = 0; s < n_seg; ++s) {
    const int w = __builtin_amdgcn_readlane(work, s), c = __builtin_amdgcn_readlane(tiles, s);
    before += w > work || (w == work && s < l) ? c : 0;
  }
  const uint64_t hit = __ballot(l < n_seg && t >= before && t < (int64_t)before + tiles);
  if (hit == 0) {   // a workgroup more than there are tiles
    *first = t + 1;
    return 0;
  }
  const int seg = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)hit) - 1);
  *first = __builtin_amdgcn_readlane(before, seg);
  return seg;
}

// ------------------------------------------------------------------ arguments
struct AttnArgs {
  const void *q, *k, *v, *go, *o;
  int64_t ldq, ldk, ldv, ldgo, ldo;
  void *out, *gq, *gk, *gv;
  int64_t ldout, ldgq, ldgk, ldgv;
  const float *pos_q, *pos_k, *slopes;
  const float* lse_in;
  float *lse, *part;   // part: of out, or of dq
  float *shift, *minus_d;   // of each query and head: the exponent of a weight is A u + shift; -D
  Bounds qb, kb;
  int n_seg, H, Hk, G, hd, dim, splits, splits_k;
  int fine;              // FEW tiles in bfloat16: weights and their gradients as sums of two
  unsigned dkv_groups;   // of a launch for both gradients: the first ones are for dk and dv
  float *part_k, *part_v;
  uint32_t g_inv;        // ceil(2^20 / G): x / G = x g_inv >> 20 for x < 512
  float scale, cap;      // of the scores as they are
  int64_t nq, nk;
};

// A lane's row of a workgroup's tile: row = query G + head of the key head's group.
struct RowOf {
  int64_t query;
  int head;
  bool there;
};
__device__ __forceinline__ RowOf row_of(const AttnArgs& a, int64_t q0, int64_t r0, int64_t R, int kvh, bool few, int tid) {
  const int64_t r = r0 + (few ? 0 : 32 * (tid >> 6)) + (tid & 31);
  const bool there = r < R;
  const unsigned q = there ? (unsigned)r / (unsigned)a.G : 0u, g = there ? (unsigned)r - q * a.G : 0u;
  return {q0 + q, kvh * a.G + (int)g, there};
}

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// How a kernel scores: bfloat16 kernels have the cap and the coordinates compiled in,
// float32 ones (CAP < 0), whose products take sixteen times as long, look at the arguments.
template <int CAP_, int DIM_>
struct Mode {
  static constexpr int CAP = CAP_, DIM = DIM_;
  static __device__ __forceinline__ bool cap(const AttnArgs& a) { return CAP < 0 ? a.cap > 0.0f : CAP > 0; }
  static __device__ __forceinline__ int dim(const AttnArgs& a) { return CAP < 0 ? a.dim : DIM; }
};

struct Place {
  float x, y, z;
};

// Coordinates of a row (those that there are).
__device__ __forceinline__ Place place_of(const float* pos, int dim, int64_t row) {
  Place p{0.0f, 0.0f, 0.0f};
  const float* at = pos + row * dim;
  p.x = at[0];
  if (dim > 1) p.y = at[1];
  if (dim > 2) p.z = at[2];
  return p;
}

// Coordinates of BN rows from `row` on (those that there are: `rem`), copied to `to`, one array of BN to each
// coordinate: one wave to each.  Arrays that are not there are cleared once instead.
template <int BN>
__device__ __forceinline__ void copy_places(const float* pos, int dim, int64_t row, int rem, float* to) {
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = (int)threadIdx.x & 63;
  if (wave >= dim) return;
  const auto from = buffer_of(pos + row * dim, (uint32_t)(rem * dim * 4));
#pragma unroll
  for (int i = 0; i < BN / 64; ++i)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(lds_u8*)(to + wave * BN + 64 * i), 4,
                                             ((64 * i + l) * dim + wave) * 4, 0, 0, 0);
}
template <int BN>
__device__ __forceinline__ void clear_places(int there, int dim, float* to) {
  for (int c = there; c < dim; ++c)
    if ((int)threadIdx.x < BN) to[c * BN + threadIdx.x] = 0.0f;
}

__device__ __forceinline__ float distance(int dim, const Place& a, float x, float y, float z) {
  const float dx = a.x - x, dy = a.y - y;
  float d = fmaf(dy, dy, dx * dx);
  if (dim > 2) {
    const float dz = a.z - z;
    d = fmaf(dz, dz, d);
  }
  return __builtin_amdgcn_sqrtf(d);
}

// tanh for float32 scores, within about 3 u of it: 1 - 2 / (1 + e^2x), whose difference costs
// digits near zero, where the series to x^11 takes its place (its next term is 2^-26 of x at 0.35).
__device__ __forceinline__ float tanh_of(float x) {
  const float far = fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + exp2_of(x * (2.0f * LOG2E))), 1.0f), s = x * x;
  float p = fmaf(s, -1382.0f / 155925.0f, 62.0f / 2835.0f);
  p = fmaf(s, p, -17.0f / 315.0f);
  p = fmaf(s, p, 2.0f / 15.0f);
  p = fmaf(s, p, -1.0f / 3.0f);
  return fabsf(x) < 0.35f ? fmaf(x * s, p, x) : far;
}

// A score is formed as u with z log2(e) = A u + C, so that e^(z - b) is one fma and one power:
//   no cap              u = x - (slope / scale) d,      A = scale log2(e),    C = 0
//   cap                 u = -r - (slope / 2 cap) d,     A = 2 cap log2(e),    C = cap log2(e)
//   cap, to its digits  u = tanh - (slope / cap) d,     A = cap log2(e),      C = 0     (float32, and the forward's fine FEW tiles)
// x = q.k, d the distance, r = 1 / (1 + e^(2 scale x / cap)): tanh = 1 - 2 r, whose absolute error of about 2^-23
// bfloat16 operands hide, but not in the lse of few keys, which may be near zero; and 1 - tanh^2 = 4 r (1 - r).
// A is positive: a negative scale goes into the sign of one operand of x, and a scale of 0 makes that operand 0 (`sign`).
template <typename T, bool FEW>
struct Score {
  float A, C, turn, per_slope, sign;
  static constexpr bool EITHER = sizeof(T) == 2 && FEW;
  std::conditional_t<EITHER, int, std::integral_constant<int, sizeof(T) == 4>> digits;
  __device__ __forceinline__ Score(const AttnArgs& a, bool cap) {
    if constexpr (EITHER) digits = a.fine;
    sign = a.scale > 0.0f ? 1.0f : a.scale < 0.0f ? -1.0f : 0.0f;
    const float scale = a.scale == 0.0f ? 1.0f : fabsf(a.scale);
    const float unit = !cap ? scale : digits ? a.cap : 2.0f * a.cap;
    A = unit * LOG2E;
    per_slope = 1.0f / unit;
    C = cap && !digits ? a.cap * LOG2E : 0.0f;
    turn = !cap ? 0.0f : digits ? scale / a.cap : 2.0f * LOG2E * scale / a.cap;
  }
  // u without its bias; `fall` receives 1 - tanh^2
  template <bool SLOPE>
  __device__ __forceinline__ float u(float x, bool cap, float* fall) const {
    if (!cap) return x;
    if (digits) {
      const float t = tanh_of(x * turn);
      if (SLOPE) *fall = 1.0f - t * t;
      return t;
    }
    const float r = __builtin_amdgcn_rcpf(1.0f + exp2_of(x * turn));
    if (SLOPE) *fall = 4.0f * r * (1.0f - r);
    return -r;
  }
};

// N operands of x with the score's sign.
template <int N, typename F>
__device__ __forceinline__ void apply_sign(F* f, float sign) {
  if (sign == 1.0f) return;
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) f[k][e] = sign == 0.0f ? 0.0f : -(float)f[k][e];
}

inline AttnArgs attn_args(const dsmp_attention_desc& d, const dsmp_segments& qs, const dsmp_segments& ks) {
  AttnArgs a{};
  a.qb = {qs.ptr, qs.n, qs.ptr ? 0 : qs.n / qs.n_seg};
  a.kb = {ks.ptr, ks.n, ks.ptr ? 0 : ks.n / ks.n_seg};
  a.n_seg = (int)qs.n_seg;
  a.H = d.heads, a.Hk = d.kv_heads, a.G = d.heads / d.kv_heads, a.hd = d.head_dim, a.dim = d.dim;
  a.g_inv = ((1u << 20) + a.G - 1) / a.G;
  a.scale = d.scale, a.cap = d.cap;
  a.nq = qs.n, a.nk = ks.n;
  a.splits = a.splits_k = 1;
  // Rounded weights put the results, which are rounded too, 1.4 times as far off as float32 products would, and
  // up to 1.6 times with few keys, whose roundings do not average out; as sums of two values no further than those
  // (0.0017 for 0.0023 to 0.0026).  Forward and backward of 300 x 300, 4 heads of 32: 25.9 us without, 26.0 with them;
  // 500 x 500, 8 heads of 128: 52.8 and 56.3; 2,048 x 2,048, 8 heads of 64, which take them no more: 83 and 93.
  a.fine = ks.n <= 512 * ks.n_seg || (double)qs.n * ks.n <= 0x1p18 * qs.n_seg * ks.n_seg;   // 512 keys, or 2^18 scores to a segment
  return a;
}

// Calls f with the element type, the padded head width and the mode of a call.
template <typename F>
void by_attention(const dsmp_attention_desc& d, F f) {
  auto width = [&](auto t, auto mode) {
    if (d.head_dim <= 32) f(t, std::integral_constant<int, 32>{}, mode);
    else if (d.head_dim <= 64) f(t, std::integral_constant<int, 64>{}, mode);
    else f(t, std::integral_constant<int, 128>{}, mode);
  };
  if (d.dtype == DSMP_F32) width(float{}, Mode<-1, 3>{});
  else if (d.dim == 0 && d.cap == 0.0f) width(__bf16{}, Mode<0, 0>{});
  else if (d.dim == 0) width(__bf16{}, Mode<1, 0>{});
  else if (d.cap != 0.0f) width(__bf16{}, Mode<1, 3>{});
  else if (d.dim <= 2) width(__bf16{}, Mode<0, 2>{});
  else width(__bf16{}, Mode<0, 3>{});
}

size_t attention_bwd_bytes(const dsmp_attention_desc& d, const dsmp_segments& qs, const dsmp_segments& ks);
dsmp_status check_attention(dsmp_handle* h, const dsmp_attention_desc* d, const dsmp_segments* qs, const dsmp_segments* ks);
void launch_attention_dq(dsmp_handle* h, const dsmp_attention_desc& d, const AttnArgs& a, int64_t grid);
void launch_attention_dkv(dsmp_handle* h, const dsmp_attention_desc& d, const AttnArgs& a, int64_t grid);

}  // namespace dsmp
