// Group norm with an activation over packed segments (channels last), forward,
// restored and backward, and activation checkpoints in 8 bits.
//
// t = x (+ addend).  Over the rows of a segment and the gs channels of a group:
// mean, var = mean of (t - mean)^2, rstd = 1 / sqrt(var + eps), xn = (t - mean) rstd,
// y = act(gamma xn + beta).  Backward with w = grad_y act'(gamma xn + beta): dbeta and
// dgamma are the sums of w and w xn over all rows; A and B the means of gamma w and
// gamma w xn over a segment's group; grad_x = rstd (gamma w - A - xn B) + grad_addend.
//
// All of it is bound by memory: about 10 operations per value forward and 30
// backward, against 4 to 16 bytes.  A segment's statistics need all its rows
// before any of them can be written, so the long form is two passes: one that
// sums over pieces of the segments (and adds the addend and writes the checkpoint on
// the way), one that joins the sums of the pieces and writes the result.  The second
// reads what the first just touched, as far as that is still in the last-level
// cache (256 MB).  Where each row is a segment, one pass.
//
// A lane holds 4 consecutive channels of a row (8 where a row is not whole aligned
// groups of 4, VEC below), 4 or 8 rows at a time.  A row takes `lpr` lanes, the next
// power of two, so sums over the rows of a wave are exchanges lpr, 2 lpr, ... lanes
// apart, and a checkpoint's block of 64 channels is 16 (8) neighbouring lanes.
//
// Sums run in a fixed order (lane, wave, piece): no atomics, the same bits on
// every run.  A lane sums its rows and a wave its lanes in float32, so a lane's number of
// roundings grows with the rows: it has about rows x lanes of a row / 131,072 of them.  Across
// waves, and across pieces, sums are in float64.
//
// The times below are kernel times on one MI355X, whose large copy runs at 5,144 GB/s
// (read and written bytes together).
#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "common.hpp"

using namespace dsmp;

namespace {

constexpr int MAX_C = 512;      // 64 lanes of 8 channels: a row stays in one wave
constexpr int BLOCK_C = 64;     // channels that share a checkpoint scale
// Threads of the passes over segments: two workgroups to a CU.  256: 53 instead of 47 us
// for the second pass over 285,564 x 128 float32; 1,024: 7.3 instead of 5.3 us for that
// of the backward over 8,192 x 64.
constexpr int NT = 512;
constexpr int NW = NT / 64;
constexpr int SNT = 1024;       // threads where one workgroup takes a whole segment
constexpr int SNW = SNT / 64;
constexpr int RNT = 256;        // threads where each row is a segment, and of the checkpoint passes
// Chunks of rows that sums are split over: one for each CU.  With 512 the second pass
// over 285,564 x 128 takes 54 us instead of 44: every workgroup joins all the sums.
constexpr int MAX_CHUNKS = 256;
constexpr int MAX_PARTS = 512;  // and where there are no sums to join (restore)
constexpr int MAX_GRID = 1024;  // workgroups that pieces are dealt to
constexpr int ROW_PARTS = 512;  // workgroups whose channel sums are kept where each row is a segment
constexpr float TINY = 0x1p-100f;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// the same at any address: one instruction, as for aligned ones
typedef uint32_t any_u32 __attribute__((aligned(1)));
typedef u32x2 any_x2 __attribute__((aligned(1)));
typedef u32x4 any_x4 __attribute__((aligned(1)));

// VEC, in all that follows, a rule on sizes and alignment alone: rows are whole aligned groups of four channels, up to
// 256 of them, and no group of the norm ends inside four.  A lane then holds four
// channels (a load instruction of a wave is one contiguous piece for every type;
// eight channels of float32 take two that each touch every line: 53 us instead of
// 44 for the second pass over 262,144 x 128), with one set of statistics.
// Elsewhere it holds eight, every channel with its own, read in one go from any address,
// past the row's end too where the matrix goes on (WIDE).  Reading a row's end value by
// value instead takes a branch and a wait for each: forward, restore and backward of
// 120,000 x 147 bfloat16 in 7 groups 382 us instead of 200, x 100 in 10 groups 179 / 103,
// x 105 float32 186 / 150.
template <bool VEC>
constexpr int CPL = VEC ? 4 : 8;    // channels per lane
template <bool VEC>
constexpr int UNIT = VEC ? 4 : 1;   // channels with the same statistics

// Steps of rows that a lane has in flight in the forward passes, in the two of the backward,
// and where a whole segment is one tile.  Twice the forward's: 14 instead of 11 us for
// the statistics of 32,768 x 64 bfloat16 in 8 segments (registers: fewer waves); the
// backward's 6 or 8: 56 instead of 33 us for the sums over 285,564 x 128.  Fewer where
// a lane holds eight channels (VEC false), each with statistics of its own: 4 forward
// 53 instead of 51 us for the statistics of 120,000 x 147, 1 for the sums 35 instead of
// 31, 2 in the last pass 25 instead of 22.7 at 120,000 x 77 and 100.
template <bool VEC>
constexpr int FWD_TILE = VEC ? 4 : 2;
template <bool VEC>
constexpr int SUMS_TILE = VEC ? 4 : 2;
template <bool VEC>
constexpr int BWD_TILE = VEC ? 4 : 1;
template <bool VEC>
constexpr int SMALL_TILE = VEC ? 8 : 2;

struct Q8 {};   // tag: a checkpoint as the source of values

struct NormArgs {
  int64_t n;
  int C, G, gs, lg;             // lg: log2 of the lanes of a row
  int n_seg;
  int64_t len;                  // rows of a segment where ptr is null
  const int32_t* ptr;
  int64_t R;                    // rows of a chunk of the summing pass
  const void* x;                // T, or int8 of a checkpoint
  int64_t ldx;
  const float* xscale;
  const void* add;
  int64_t lda;
  void* sum;
  int64_t lds;
  const float *gamma, *beta;
  void* y;
  int64_t ldy;
  float* stats;
  int8_t* q;
  float* scale;
  float2* part;                 // sums of the pieces (chunk x segment), [chunk + segment][G]
  float eps;
  int merge, ck, y_bf16;
  const float* gy;
  int64_t ldgy;
  const float* ga;
  int64_t ldga;
  float* gx;
  int64_t ldgx;
  float* part_c;                // [parts][2][C]: a workgroup's sums of w and w xn
  float *dgamma, *dbeta;
  int accumulate, parts, grid;
  int64_t pieces;
};

// ------------------------------------------------------------ across lanes

// Sums over lanes by data-parallel moves (a shuffle through LDS takes tens of
// cycles more, and these come in chains).
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false);
}
template <int CTRL>
__device__ __forceinline__ float moved(float x) {
  return __builtin_bit_cast(float, moved<CTRL>(__builtin_bit_cast(uint32_t, x)));
}
template <int CTRL>
__device__ __forceinline__ double moved(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, (uint64_t)moved<CTRL>((uint32_t)(u >> 32)) << 32 | moved<CTRL>((uint32_t)u));
}

// A lane's value and that of a lane O away: rotated within 16 lanes, or the two
// sides of an exchange of 16 or 32.  Repeated with O = o, 2 o, ... 32 it meets every
// lane of the same place modulo o once.
template <typename T>
struct Two {
  T a, b;
};
template <int O>
__device__ __forceinline__ Two<uint32_t> across(uint32_t x) {
  if (O == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return {r[0], r[1]};
  }
  if (O == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return {r[0], r[1]};
  }
  return {x, moved<0x120 + (O < 16 ? O : 1)>(x)};
}
template <int O>
__device__ __forceinline__ Two<float> across(float x) {
  const Two<uint32_t> r = across<O>(__builtin_bit_cast(uint32_t, x));
  return {__builtin_bit_cast(float, r.a), __builtin_bit_cast(float, r.b)};
}
template <int O>
__device__ __forceinline__ Two<double> across(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const Two<uint32_t> l = across<O>((uint32_t)u), h = across<O>((uint32_t)(u >> 32));
  return {__builtin_bit_cast(double, (uint64_t)h.a << 32 | l.a), __builtin_bit_cast(double, (uint64_t)h.b << 32 | l.b)};
}

// f(O) for O = first, 2 first, ... 32
template <typename F>
__device__ __forceinline__ void levels(int first, F f) {
  if (first <= 1) f(std::integral_constant<int, 1>{});
  if (first <= 2) f(std::integral_constant<int, 2>{});
  if (first <= 4) f(std::integral_constant<int, 4>{});
  if (first <= 8) f(std::integral_constant<int, 8>{});
  if (first <= 16) f(std::integral_constant<int, 16>{});
  if (first <= 32) f(std::integral_constant<int, 32>{});
}
template <int O, typename T>
__device__ __forceinline__ void add_across(T& x) {
  const Two<T> r = across<O>(x);
  x = r.a + r.b;
}

// op over `width` neighbouring lanes (a power of two), in all of them: pairs, fours,
// then mirrored halves of eight and sixteen, then exchanges.
template <typename T, typename OP>
__device__ __forceinline__ T over_lanes(T x, int width, OP op) {
  if (width > 1) x = op(x, moved<0xb1>(x));
  if (width > 2) x = op(x, moved<0x4e>(x));
  if (width > 4) x = op(x, moved<0x141>(x));
  if (width > 8) x = op(x, moved<0x140>(x));
  if (width > 16) {
    const Two<T> r = across<16>(x);
    x = op(r.a, r.b);
  }
  if (width > 32) {
    const Two<T> r = across<32>(x);
    x = op(r.a, r.b);
  }
  return x;
}
template <typename T>
__device__ __forceinline__ T sum_lanes(T x, int width) {
  return over_lanes(x, width, [](T a, T b) { return a + b; });
}

// to[t] = x of lane t of the 16 lanes (`wide`) or 8 lanes that a lane is one of
template <int T>
__device__ __forceinline__ float from_lane(float x, bool wide) {
  const float low = moved<0x150 + T>(x);
  if (wide) return low;
  const float high = moved<0x158 + T>(x);
  return threadIdx.x & 8 ? high : low;
}
template <int N>
__device__ __forceinline__ void from_lanes(float x, float (&to)[N], bool wide) {
  static_assert(N == 4 || N == 8, "");
  to[0] = from_lane<0>(x, wide), to[1] = from_lane<1>(x, wide), to[2] = from_lane<2>(x, wide);
  to[3] = from_lane<3>(x, wide);
  if constexpr (N == 8) {
    to[4] = from_lane<4>(x, wide), to[5] = from_lane<5>(x, wide), to[6] = from_lane<6>(x, wide);
    to[7] = from_lane<7>(x, wide);
  }
}

// ------------------------------------------------------------ rows and lanes

// The place of a lane: CPL channels from c0 (cnt of them exist) in row rl of the
// RL rows that a workgroup steps over.
template <bool VEC>
struct Lanes {
  int lpr, lr, rl, RL, c0, cnt;
  __device__ __forceinline__ Lanes(int lg, int C, int threads) {
    lpr = 1 << lg;
    lr = threadIdx.x & (lpr - 1);
    rl = threadIdx.x >> lg;
    RL = threads >> lg;
    c0 = lr * CPL<VEC>;
    cnt = std::min(CPL<VEC>, C - c0);
  }
  // Where the lane reads.  With whole groups a lane past the row takes the row's
  // last channels once more (no sum counts them, and a block's largest is the
  // same): a condition would become a branch around the load, and a wait.
  __device__ __forceinline__ int at(int C) const { return std::min(c0, VEC ? C - CPL<VEC> : C - 1); }
};

// Rows of a matrix.  Row i + at, where i is the same for all lanes (scalar
// registers) and `at` the lane's own, small enough for 24-bit products and
// 32-bit offsets.
template <typename T>
struct Mat {
  const char* p;
  int64_t pitch;
  uint32_t off;
  __device__ __forceinline__ Mat(const void* base, int64_t ld, int c)
      : p(static_cast<const char*>(base)), pitch(ld * (int64_t)sizeof(T)), off((uint32_t)c * (uint32_t)sizeof(T)) {}
  __device__ __forceinline__ T* row(int64_t i, int at) const {
    return reinterpret_cast<T*>(const_cast<char*>(p + i * pitch) + (__umul24((uint32_t)at, (uint32_t)pitch) + off));
  }
};

// The rows of a tile: N steps of RL rows, all of which exist (FULL) or the first
// `left`.  Reads then take the last row again past it, and what they bring is not
// used: all loads of a tile go out together, whatever exists.  Where rows are not whole
// groups, the matrix has 7 more rows after a FULL tile: its lanes may read 8 channels
// from any of a row's, whatever the row distance.
template <int N_, bool FULL_>
struct Tile {
  static constexpr int N = N_;
  static constexpr bool FULL = FULL_;
  int rl, RL, left;
  template <typename LANES>
  __device__ __forceinline__ Tile(const LANES& L, int left_) : rl(L.rl), RL(L.RL), left(left_) {}
  // step t's rows: the lane's is at(t) past first(i, t)
  __device__ __forceinline__ int64_t first(int64_t i, int t) const { return FULL ? i + t * RL : i; }
  __device__ __forceinline__ int at(int t) const { return FULL ? rl : std::min(rl + t * RL, left - 1); }
  __device__ __forceinline__ bool ok(int t) const { return FULL || rl + t * RL < left; }
  __device__ __forceinline__ bool end(int t) const { return !FULL && t * RL >= left; }   // no lane has it
};

// Keeps loads ahead of the conditions that their values are used under: sunk into
// them, each would be waited for by itself.
template <int N, int M>
__device__ __forceinline__ void arrived(float (&v)[N][M]) {
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int k = 0; k < M; ++k) asm volatile("" : "+v"(v[t][k]));
}

// tile(i, rows of it) over the rows [r, e): whole tiles of N steps, the rest in
// tiles of half as many.  n: the matrix's rows.
template <bool VEC>
__device__ __forceinline__ int64_t full_end(int64_t e, int64_t n) {
  return VEC ? e : std::min<int64_t>(e, n - (CPL<VEC> - 1));
}
template <int N, bool VEC, typename F>
__device__ __forceinline__ void over_rows(const Lanes<VEC>& L, int64_t r, int64_t e, int64_t n, F tile) {
  constexpr int H = N > 1 ? N / 2 : 1;
  const int64_t f = full_end<VEC>(e, n);
  int64_t i = r;
  for (; i + N * L.RL <= f; i += N * L.RL) tile(i, Tile<N, true>(L, N * L.RL));
  for (; i < e; i += H * L.RL) tile(i, Tile<H, false>(L, (int)std::min<int64_t>(e - i, H * L.RL)));
}

// row(i, whole) where a workgroup's rows are i + rl, all workgroups together go over all
// rows, and only the row's own lanes work together.  whole: as a FULL tile, or only
// the lanes whose row exists.
template <bool VEC, typename F>
__device__ __forceinline__ void each_row(const Lanes<VEC>& L, int64_t n, F row) {
  const int64_t f = full_end<VEC>(n, n), step = (int64_t)gridDim.x * L.RL;
  int64_t i = (int64_t)blockIdx.x * L.RL;
  for (; i + L.RL <= f; i += step) row(i, std::true_type{});
  for (; i < n; i += step)
    if (i + L.rl < n) row(i, std::false_type{});
}

// over_rows in two steps: take(i, rows, v) loads a tile into v, give(i, rows, v) uses
// it.  The next whole tile is on its way while one is used (stores count among the
// memory operations that a load's wait looks at: a tile loaded after them would
// wait for them).
template <int N, bool VEC, typename TAKE, typename GIVE>
__device__ __forceinline__ void pass_rows(const Lanes<VEC>& L, int64_t r, int64_t e, int64_t n, TAKE take, GIVE give) {
  constexpr int H = N > 1 ? N / 2 : 1, M = CPL<VEC>;
  const int64_t S = N * L.RL, f = full_end<VEC>(e, n);
  int64_t i = r;
  if (i + S <= f) {
    const Tile<N, true> rows(L, N * L.RL);
    float v[N][M], w[N][M];
    take(i, rows, v);
    for (; i + 2 * S <= f; i += S) {
      take(i + S, rows, w);
      give(i, rows, v);
#pragma unroll
      for (int t = 0; t < N; ++t)
#pragma unroll
        for (int k = 0; k < M; ++k) v[t][k] = w[t][k];
    }
    give(i, rows, v);
    i += S;
  }
  for (; i < e; i += H * L.RL) {
    const Tile<H, false> rows(L, (int)std::min<int64_t>(e - i, H * L.RL));
    float v[H][M];
    take(i, rows, v);
    arrived(v);
    give(i, rows, v);
  }
}

// N four-byte words from or to any address, or whole aligned ones (VEC).  STREAM:
// with the non-temporal hint, for what is not used again soon.  It keeps what the
// second pass reads again in the last-level cache:
// - results (y, q, grad_x): forward, restore and backward of 285,564 x 128 float32 with
//   addend and checkpoint 306 us without the hint, 290 with.  A kernel that reads the
//   result next, timed with it, gains or loses little: 161.5 / 149.5 after the
//   backward, 112.2 / 109.9 after the forward, 54.4 / 55.6 after restore; 52.9 / 54.4,
//   42.8 / 42.8, 22.1 / 22.4 at 100,000 x 128.
// - inputs where they are used for the last time: 290 / 271 us; forward of
//   262,144 x 128 with an addend 121 / 107.
// Not where it costs: the sum (read again at once: the second pass 54 us with the hint,
// 44 without) and a checkpoint in restore (26 with, 20 without: the backward reads it).
// Not where rows are not whole aligned groups (VEC false): pieces of cache lines past the
// caches cost more than they save.  120,000 rows, forward, restore and backward with it /
// without: 105 channels of float32 155 / 149 us, 147 of bfloat16 204 / 200, 100 in ten groups
// 99 / 103; a checkpoint of 60,000 x 226 stored and loaded 27 / 25.
// One rule for all sizes: chosen when compiled (of two stores in one kernel the
// compiler keeps one, without the hint), and at small sizes the two differ by 0.3 us.
template <bool STREAM, typename W>
__device__ __forceinline__ W get(const void* p) {
  if constexpr (STREAM)
    return __builtin_nontemporal_load(static_cast<const W*>(p));
  else
    return *static_cast<const W*>(p);
}
template <bool STREAM, typename W>
__device__ __forceinline__ void put(void* p, W w) {
  if constexpr (STREAM)
    __builtin_nontemporal_store(w, static_cast<W*>(p));
  else
    *static_cast<W*>(p) = w;
}
template <bool VEC, bool STREAM, int N>
__device__ __forceinline__ void get_words(const void* p, uint32_t (&w)[N]) {
  if constexpr (N == 4) {
    const u32x4 u = get<STREAM && VEC, std::conditional_t<VEC, u32x4, any_x4>>(p);
    w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
  } else if constexpr (N == 2) {
    const u32x2 u = get<STREAM && VEC, std::conditional_t<VEC, u32x2, any_x2>>(p);
    w[0] = u.x, w[1] = u.y;
  } else {
    w[0] = get<STREAM && VEC, std::conditional_t<VEC, uint32_t, any_u32>>(p);
  }
}
template <bool VEC, bool STREAM, int N>
__device__ __forceinline__ void put_words(void* p, const uint32_t (&w)[N]) {
  if constexpr (N == 4)
    put<STREAM && VEC, std::conditional_t<VEC, u32x4, any_x4>>(p, (u32x4){w[0], w[1], w[2], w[3]});
  else if constexpr (N == 2)
    put<STREAM && VEC, std::conditional_t<VEC, u32x2, any_x2>>(p, (u32x2){w[0], w[1]});
  else
    put<STREAM && VEC, std::conditional_t<VEC, uint32_t, any_u32>>(p, w[0]);
}

// by value: of two array elements the compiler would choose the address
template <typename T>
__device__ __forceinline__ T either(bool c, T a, T b) {
  return c ? a : b;
}

// cnt: how many of a lane's channels exist (all, fewer in a last lane, none or
// less past it); not looked at in loads where VEC.  WIDE: the lane reads all of its
// places in one go, past the row's end too (see Tile), and puts 0 in the place of what
// isn't the row's.
template <bool VEC>
__device__ __forceinline__ void only(int cnt, float (&v)[CPL<VEC>]) {
  if (VEC) return;
#pragma unroll
  for (int k = 0; k < CPL<VEC>; ++k) v[k] = k < cnt ? v[k] : 0.0f;
}
template <bool VEC, bool STREAM, bool WIDE = false>
__device__ __forceinline__ void load_row(const float* p, int cnt, float (&v)[CPL<VEC>]) {
  if (VEC || WIDE || cnt == CPL<VEC>) {
#pragma unroll
    for (int j = 0; j < CPL<VEC>; j += 4) {
      uint32_t w[4];
      get_words<VEC, STREAM>(p + j, w);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[j + k] = __builtin_bit_cast(float, w[k]);
    }
    if (WIDE) only<VEC>(cnt, v);
  } else {
#pragma unroll
    for (int k = 0; k < CPL<VEC>; ++k) v[k] = k < cnt ? p[k] : 0.0f;
  }
}
template <bool VEC, bool STREAM, bool WIDE = false>
__device__ __forceinline__ void load_row(const __bf16* p, int cnt, float (&v)[CPL<VEC>]) {
  if (VEC || WIDE || cnt == CPL<VEC>) {
    uint32_t w[CPL<VEC> / 2];
    get_words<VEC, STREAM>(p, w);
#pragma unroll
    for (int k = 0; k < CPL<VEC> / 2; ++k) {
      v[2 * k] = __builtin_bit_cast(float, w[k] << 16);
      v[2 * k + 1] = __builtin_bit_cast(float, w[k] & 0xffff0000u);
    }
    if (WIDE) only<VEC>(cnt, v);
  } else {
#pragma unroll
    for (int k = 0; k < CPL<VEC>; ++k) v[k] = k < cnt ? (float)p[k] : 0.0f;
  }
}
// bytes of a checkpoint times their block's scale
template <bool VEC, bool STREAM, bool WIDE = false>
__device__ __forceinline__ void load_row(const int8_t* p, float scale, int cnt, float (&v)[CPL<VEC>]) {
  if (VEC || WIDE || cnt == CPL<VEC>) {
    uint32_t w[CPL<VEC> / 4];
    get_words<VEC, STREAM>(p, w);
#pragma unroll
    for (int k = 0; k < CPL<VEC>; ++k) v[k] = (float)((int32_t)(w[k / 4] << (24 - 8 * (k % 4))) >> 24) * scale;
    if (WIDE) only<VEC>(cnt, v);
  } else {
#pragma unroll
    for (int k = 0; k < CPL<VEC>; ++k) v[k] = k < cnt ? (float)p[k] * scale : 0.0f;
  }
}

template <bool VEC, bool STREAM>
__device__ __forceinline__ void store_row(float* p, int cnt, const float (&v)[CPL<VEC>]) {
  if (cnt == CPL<VEC>) {
#pragma unroll
    for (int j = 0; j < CPL<VEC>; j += 4) {
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = __builtin_bit_cast(uint32_t, v[j + k]);
      put_words<VEC, STREAM>(p + j, w);
    }
  } else if constexpr (!VEC) {   // a row's end in fours, twos and ones
    uint32_t w[4], u[2];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = __builtin_bit_cast(uint32_t, v[k]);
    if (cnt <= 0) return;
    if (cnt & 4) put_words<VEC, STREAM>(p, w);
#pragma unroll
    for (int k = 0; k < 2; ++k) u[k] = __builtin_bit_cast(uint32_t, either(cnt & 4, v[4 + k], v[k]));
    if (cnt & 2) put_words<VEC, STREAM>(p + (cnt & 4), u);
    if (cnt & 1) p[cnt - 1] = either(cnt & 4, either(cnt & 2, v[6], v[4]), either(cnt & 2, v[2], v[0]));
  }
}
template <bool VEC, bool STREAM>
__device__ __forceinline__ void store_row(__bf16* p, int cnt, const float (&v)[CPL<VEC>]) {
  uint32_t w[CPL<VEC> / 2];
#pragma unroll
  for (int k = 0; k < CPL<VEC> / 2; ++k)
    w[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){v[2 * k], v[2 * k + 1]}, bf16x2));
  if (cnt == CPL<VEC>) {
    put_words<VEC, STREAM>(p, w);
  } else if constexpr (!VEC) {
    if (cnt <= 0) return;
    const uint32_t two[2] = {w[0], w[1]}, one[1] = {either(cnt & 4, w[2], w[0])};
    if (cnt & 4) put_words<VEC, STREAM>(p, two);
    if (cnt & 2) put_words<VEC, STREAM>(p + (cnt & 4), one);
    if (cnt & 1) p[cnt - 1] = (__bf16)either(cnt & 4, either(cnt & 2, v[6], v[4]), either(cnt & 2, v[2], v[0]));
  }
}

__host__ __device__ __forceinline__ int blocks_of(int C) { return (C + BLOCK_C - 1) / BLOCK_C; }

// The values that are normalised: rows of T, or of a checkpoint.
template <typename T, bool VEC, bool STREAM = false>
struct Source {
  Mat<T> m;
  int cnt;
  __device__ __forceinline__ Source(const NormArgs& a, const Lanes<VEC>& L) : m(a.x, a.ldx, L.at(a.C)), cnt(L.cnt) {}
  template <bool WIDE>
  __device__ __forceinline__ void load(int64_t i, int at, float (&v)[CPL<VEC>]) const {
    load_row<VEC, STREAM, WIDE>(m.row(i, at), cnt, v);
  }
};
template <bool VEC, bool STREAM>
struct Source<Q8, VEC, STREAM> {
  Mat<int8_t> m;
  Mat<float> s;
  int cnt;
  __device__ __forceinline__ Source(const NormArgs& a, const Lanes<VEC>& L)
      : m(a.x, a.C, L.at(a.C)),
        s(a.xscale, blocks_of(a.C), std::min(L.at(a.C), a.C - 1) / BLOCK_C), cnt(L.cnt) {}
  template <bool WIDE>
  __device__ __forceinline__ void load(int64_t i, int at, float (&v)[CPL<VEC>]) const {
    load_row<VEC, STREAM, WIDE>(m.row(i, at), *s.row(i, at), cnt, v);
  }
};

// t = x, or x + addend rounded to T, which is then written to sum.
template <typename T, bool VEC, bool ADD>
struct Stream {
  Source<T, VEC, ADD> x;   // with an addend it is the sum that is read again
  Mat<T> add, sum;
  int cnt;
  __device__ __forceinline__ Stream(const NormArgs& a, const Lanes<VEC>& L)
      : x(a, L), add(a.add, a.lda, L.at(a.C)), sum(a.sum, a.lds, L.c0), cnt(L.cnt) {}
  template <int N, bool FULL>
  __device__ __forceinline__ void load(int64_t i, const Tile<N, FULL>& rows, float (&v)[N][CPL<VEC>]) const {
    float u[N][CPL<VEC>];
#pragma unroll
    for (int t = 0; t < N; ++t) {
      x.template load<FULL>(rows.first(i, t), rows.at(t), v[t]);
      if (ADD) load_row<VEC, true, FULL>(add.row(rows.first(i, t), rows.at(t)), cnt, u[t]);
    }
    if (!FULL) {
      arrived(v);
      if (ADD) arrived(u);
    }
    if (ADD) {
#pragma unroll
      for (int t = 0; t < N; ++t) {
#pragma unroll
        for (int k = 0; k < CPL<VEC>; ++k) v[t][k] = (float)(T)(v[t][k] + u[t][k]);
        if (rows.ok(t)) store_row<VEC, false>(sum.row(rows.first(i, t), rows.at(t)), cnt, v[t]);   // read again at once
      }
    }
  }
};

// Where y goes, of either type.
template <bool VEC>
struct Result {
  Mat<float> f;
  Mat<__bf16> b;
  int cnt, bf16;
  __device__ __forceinline__ Result(const NormArgs& a, const Lanes<VEC>& L)
      : f(a.y, a.ldy, L.c0), b(a.y, a.ldy, L.c0), cnt(L.cnt), bf16(a.y_bf16) {}
  __device__ __forceinline__ void store(int64_t i, int at, const float (&v)[CPL<VEC>]) const {
    if (bf16)
      store_row<VEC, true>(b.row(i, at), cnt, v);
    else
      store_row<VEC, true>(f.row(i, at), cnt, v);
  }
};

// Writes rows in 8 bits.  64 / CPL lanes (fewer where a row has fewer) hold a block
// of 64 channels.  Its largest magnitude is found on the bits without the sign,
// which order as the values do and put a NaN above everything.  The division of a
// block is done for all rows of a tile at once, each by another lane of the block.
template <bool VEC>
struct Keep {
  Mat<int8_t> q;
  Mat<float> s;
  int cnt, width;
  bool first;
  __device__ __forceinline__ Keep(const NormArgs& a, const Lanes<VEC>& L)
      : q(a.q, a.C, L.c0), s(a.scale, blocks_of(a.C), L.c0 / BLOCK_C), cnt(L.cnt),
        width(std::min(BLOCK_C / CPL<VEC>, L.lpr)), first(L.c0 % BLOCK_C == 0 && L.cnt > 0) {}

  // 127 / big, and the scale, of a block
  static __device__ __forceinline__ void factors(uint32_t m, float& inv, float& scale) {
    const float big = __builtin_bit_cast(float, m);
    const bool some = m >= __builtin_bit_cast(uint32_t, TINY), odd = m >= 0x7f800000u;
    inv = some && !odd ? 127.0f / big : 0.0f;
    scale = odd ? __builtin_bit_cast(float, 0x7fc00000u) : some ? big * (1.0f / 127.0f) : 0.0f;
  }

  template <int N, bool FULL>
  __device__ __forceinline__ void store(int64_t i, const Tile<N, FULL>& rows, const float (&v)[N][CPL<VEC>]) const {
    uint32_t m[N];
#pragma unroll
    for (int t = 0; t < N; ++t) {
      m[t] = 0;
#pragma unroll
      for (int k = 0; k < CPL<VEC>; ++k) m[t] = max(m[t], __builtin_bit_cast(uint32_t, v[t][k]) & 0x7fffffffu);
      m[t] = over_lanes(m[t], width, [](uint32_t a, uint32_t b) { return max(a, b); });
    }
    float inv[N], scale[N];
    bool done = false;
    if constexpr (N == 8 || N == 4) {
      done = width >= 8;
      if (done) {
        const int l = threadIdx.x & (N - 1);
        uint32_t mine = m[0];
#pragma unroll
        for (int t = 1; t < N; ++t) mine = l == t ? m[t] : mine;
        float fi, fs;
        factors(mine, fi, fs);
        from_lanes(fi, inv, width > 8);
        from_lanes(fs, scale, width > 8);
      }
    }
    if (!done) {
#pragma unroll
      for (int t = 0; t < N; ++t) factors(m[t], inv[t], scale[t]);
    }
#pragma unroll
    for (int t = 0; t < N; ++t) {
      if (rows.end(t)) break;
      if (rows.ok(t)) one(rows.first(i, t), rows.at(t), m[t], inv[t], scale[t], v[t]);
    }
  }

  // x inv rounded to whole numbers: 1.5 2^23 is added, and the sum's last byte is the
  // number (a magnitude of at most 127; product and sum are rounded apart)
  static __device__ __forceinline__ uint32_t whole_number(float x, float inv) {
#pragma clang fp contract(off)
    const float p = x * inv;
    return __builtin_bit_cast(uint32_t, p + 12582912.0f) & 255u;
  }

  __device__ __forceinline__ void one(int64_t i, int at, uint32_t m, float inv, float scale,
                                      const float (&v)[CPL<VEC>]) const {
    uint32_t w[CPL<VEC> / 4];
#pragma unroll
    for (int j = 0; j < CPL<VEC> / 4; ++j) {
      w[j] = whole_number(v[4 * j], inv) | whole_number(v[4 * j + 1], inv) << 8 | whole_number(v[4 * j + 2], inv) << 16 |
             whole_number(v[4 * j + 3], inv) << 24;
      w[j] = m >= 0x7f800000u ? 0u : w[j];
    }
    int8_t* p = q.row(i, at);
    if (cnt == CPL<VEC>) {
      put_words<VEC, true>(p, w);
    } else if constexpr (!VEC) {
      if (cnt > 0) {
        const uint32_t four[1] = {w[0]}, u = either(cnt & 4, w[1], w[0]);
        const uint16_t two = (uint16_t)u;
        if (cnt & 4) put_words<VEC, true>(p, four);
        if (cnt & 2) __builtin_memcpy(p + (cnt & 4), &two, 2);
        if (cnt & 1) p[cnt - 1] = (int8_t)(cnt & 2 ? u >> 16 : u);
      }
    }
    if (first) *s.row(i, at) = scale;
  }
};

// ------------------------------------------------------------ activations

// Upper tail Q of the normal distribution at |z|, and e = exp(-z^2/2).  Q / e falls slowly
// from 1/2 as 1 / |z|; in t = 1 / (1 + 0.31 |z|) it is t times a polynomial of degree 7, fitted
// here to the smallest relative error over |z| <= 14.2 (1.7e-7; below that e is too small for float32).
// So Q has a relative error of at most (20 + 1.5 z^2) 2^-24, the second term from the exponent's
// roundings, and the small values of GELU at negative z, which are taken from Q without a
// difference, keep their digits.
__device__ __forceinline__ float normal_tail(float z, float& e) {
  e = __expf(-0.5f * z * z);
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.31f, __builtin_fabsf(z), 1.0f));
  float p = __builtin_fmaf(0.03585438058f, t, -0.1416601091f);
  p = __builtin_fmaf(p, t, 0.1551691145f);
  p = __builtin_fmaf(p, t, -0.01500251796f);
  p = __builtin_fmaf(p, t, 0.1101661921f);
  p = __builtin_fmaf(p, t, 0.1077528521f);
  p = __builtin_fmaf(p, t, 0.1240634918f);
  p = __builtin_fmaf(p, t, 0.1236566901f);
  return p * t * e;
}

template <int ACT>
__device__ __forceinline__ float activate(float z) {
  if (ACT == DSMP_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.0f + __expf(-z));
  if (ACT == DSMP_ACT_GELU) {
    float e;
    const float q = normal_tail(z, e);
    return z * (z < 0.0f ? q : 1.0f - q);
  }
  if (ACT == DSMP_ACT_RELU) return z < 0.0f ? 0.0f : z;   // a NaN passes
  return z;
}

template <int ACT>
__device__ __forceinline__ float slope(float z) {
  if (ACT == DSMP_ACT_SILU) {
    const float p = __builtin_amdgcn_rcpf(1.0f + __expf(-z));
    return p * __builtin_fmaf(z, 1.0f - p, 1.0f);
  }
  if (ACT == DSMP_ACT_GELU) {
    float e;
    const float q = normal_tail(z, e);
    return __builtin_fmaf(z * 0.39894228f, e, z < 0.0f ? q : 1.0f - q);
  }
  if (ACT == DSMP_ACT_RELU) return z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z;   // a NaN passes
  return 1.0f;
}

// ------------------------------------------------------------ segments

// Begin and end of segment s; values of ptr are limited to [0, n], and the last
// segment ends at n, so that every row has a segment whatever ptr holds.
__device__ __forceinline__ int64_t seg_begin(const NormArgs& a, int s) {
  if (!a.ptr) return s * a.len;
  return s == 0 ? 0 : std::min<int64_t>(std::max<int64_t>(a.ptr[s], 0), a.n);
}
__device__ __forceinline__ int64_t seg_end(const NormArgs& a, int s) {
  return s + 1 >= a.n_seg ? a.n : seg_begin(a, s + 1);
}
// The passes' units of work are pieces: the rows that a segment s has in a chunk j of R
// rows.  Piece j + s: as rows go on, either the chunk or the segment is the next one,
// so the numbers of a segment's pieces follow each other, and every number up to
// chunks + segments is one piece or none.  A piece takes a workgroup through all
// barriers of the joining, however few rows it has: 65,536 x 64 bfloat16 in 4,096 segments
// of 16 rows takes 33 + 28 us forward and 32 + 30 backward, in one segment 5.6 + 7.4 and
// 8.5 + 7.9.
struct Piece {
  int s;
  int64_t b, e;    // the segment's rows
  int64_t r, end;  // the piece's
  bool first;      // the segment begins with it
  __device__ __forceinline__ Piece(const NormArgs& a, int64_t p) {
    s = 0, b = 0, e = a.n;
    if (a.n_seg > 1) find(a, p);
    const int64_t j = p - s;
    r = std::max<int64_t>(b, j * a.R);
    end = std::min<int64_t>(e, (j + 1) * a.R);
    first = r == b;
  }
  // Of the segments whose first number, b / R + s, is at most p, the last: 64 at a time,
  // one to a lane of each wave (every wave finds the same).
  __device__ __forceinline__ void find(const NormArgs& a, int64_t p) {
    const int lane = threadIdx.x & 63;
    int lo = 0, count = a.n_seg, k, mine;   // it is one of lo .. lo + count - 1
    for (;;) {
      const int step = (int)(((int64_t)count + 63) / 64);
      const int64_t off = (int64_t)lane * step, i = lo + off;
      mine = (int)seg_begin(a, (int)std::min<int64_t>(i, a.n_seg - 1));
      const bool at = off < count && (int64_t)((uint32_t)mine / (uint32_t)a.R) + i <= p;
      // bounds that do not ascend still leave the first lane's true
      k = 63 - __builtin_clzll(__ballot(at) | 1ull);
      lo += k * step;
      if (step == 1) break;
      count = std::min(step, count - k * step);
    }
    s = __builtin_amdgcn_readfirstlane(lo);
    k = __builtin_amdgcn_readfirstlane(k);
    b = __builtin_amdgcn_readlane(mine, k);
    // the last round's next lane has the next segment's begin, if it is not the last lane
    e = s + 1 >= a.n_seg ? a.n : k < 63 ? (int64_t)__builtin_amdgcn_readlane(mine, k + 1) : seg_begin(a, s + 1);
  }
};

// s1, s2: the workgroup's sums per channel (or unit of channels), float64 in LDS.
// Gives the sums over each group's gs of them to out(g, sum1, sum2), by one lane each.
template <int W, typename F>
__device__ __forceinline__ void group_sums(const double* s1, const double* s2, int G, int gs, F out) {
  int tg = 1;   // lanes of a group
  while (tg < 64 && tg * 2 * G <= W * 64 && tg < gs) tg <<= 1;
  const int per = W * 64 / tg;
  for (int gb = 0; gb < G; gb += per) {
    const int g = gb + (int)threadIdx.x / tg, l = threadIdx.x % tg;
    double u = 0.0, v = 0.0;
    if (g < G)
      for (int i = l; i < gs; i += tg) u += s1[g * gs + i], v += s2[g * gs + i];
    u = sum_lanes(u, tg);
    v = sum_lanes(v, tg);
    if (g < G && l == 0) out(g, u, v);
  }
}

// ------------------------------------------------------------ per lane

// A value for each of a lane's channels that is the same within a unit.
template <bool VEC>
struct PerUnit {
  static constexpr int N = CPL<VEC> / UNIT<VEC>;
  float v[N];
  __device__ __forceinline__ float operator[](int k) const { return v[k / UNIT<VEC>]; }
};

// The groups of a lane's units.
template <bool VEC>
struct Groups {
  int g[PerUnit<VEC>::N];
  __device__ __forceinline__ Groups(const NormArgs& a, int c0) {
#pragma unroll
    for (int j = 0; j < PerUnit<VEC>::N; ++j) g[j] = std::min(c0 + j * UNIT<VEC>, a.C - 1) / a.gs;
  }
  // pairs of a segment's groups: (mean, rstd), or the two sums of the backward pass
  __device__ __forceinline__ void read(const float2* st, PerUnit<VEC>& x, PerUnit<VEC>& y) const {
#pragma unroll
    for (int j = 0; j < PerUnit<VEC>::N; ++j) {
      const float2 t = st[g[j]];
      x.v[j] = t.x, y.v[j] = t.y;
    }
  }
};

template <bool VEC>
__device__ __forceinline__ void params(const NormArgs& a, const Lanes<VEC>& L, float (&gamma)[CPL<VEC>], float (&beta)[CPL<VEC>]) {
  if (a.gamma) {
    load_row<VEC, false>(a.gamma + L.at(a.C), L.cnt, gamma);
    load_row<VEC, false>(a.beta + L.at(a.C), L.cnt, beta);
  } else {
#pragma unroll
    for (int k = 0; k < CPL<VEC>; ++k) gamma[k] = 1.0f, beta[k] = 0.0f;
  }
}

__device__ __forceinline__ float2* stats_of(const NormArgs& a, int s) {
  return reinterpret_cast<float2*>(a.stats) + (int64_t)s * a.G;
}

// ------------------------------------------------------------ forward, statistics

// Rows, and for each unit the mean and the sum of squares about it.  Rows join
// a few at a time (mean of the tile, then deviations from it, then the pair rule
// of Chan, Golub and LeVeque), so a large mean or a far-out row costs the variance no
// digits.  The means themselves are float32 values, of a lane, a piece and in stats: off by
// a few units in the last place at most, which xn has times rstd (at a mean of 10^4
// deviations half a unit is 5e-4 of one).
template <bool VEC>
struct Moments {
  static constexpr int U = UNIT<VEC>, N = CPL<VEC> / U;
  float n = 0.0f, mean[N] = {}, m2[N] = {};

  template <int T>
  __device__ __forceinline__ void add(const float (&v)[T][CPL<VEC>]) {
    const float nn = n + T, w = T / nn, f = n * w * U;
    n = nn;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      float s = 0.0f, q = 0.0f;
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int k = 0; k < U; ++k) s += v[t][j * U + k];
      const float m = s * (1.0f / (T * U));
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int k = 0; k < U; ++k) q = __builtin_fmaf(v[t][j * U + k] - m, v[t][j * U + k] - m, q);
      const float d = m - mean[j];
      mean[j] = __builtin_fmaf(d, w, mean[j]);
      m2[j] += __builtin_fmaf(d * d, f, q);
    }
  }
  template <int T, bool FULL>
  __device__ __forceinline__ void add(const float (&v)[T][CPL<VEC>], const Tile<T, FULL>& rows) {
    if (FULL)
      add(v);
    else
      add_some(v, rows);
  }
  // where a lane has fewer than T rows
  template <int T, bool FULL>
  __device__ __forceinline__ void add_some(const float (&v)[T][CPL<VEC>], const Tile<T, FULL>& rows) {
    bool ok[T];
    float c = 0.0f;
#pragma unroll
    for (int t = 0; t < T; ++t) ok[t] = rows.ok(t), c += ok[t] ? 1.0f : 0.0f;
    if (c == 0.0f) return;
    const float nn = n + c, w = c / nn, f = n * w * U, inv = 1.0f / (c * U);
    n = nn;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      float s = 0.0f, q = 0.0f;
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int k = 0; k < U; ++k) s += ok[t] ? v[t][j * U + k] : 0.0f;
      const float m = s * inv;
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int k = 0; k < U; ++k) {
          const float d = ok[t] ? v[t][j * U + k] - m : 0.0f;
          q = __builtin_fmaf(d, d, q);
        }
      const float d = m - mean[j];
      mean[j] = __builtin_fmaf(d, w, mean[j]);
      m2[j] += __builtin_fmaf(d * d, f, q);
    }
  }
  // joins the lane O away
  template <int O>
  __device__ __forceinline__ void join() {
    const Two<float> c = across<O>(n);
    const float nn = c.a + c.b, w = nn > 0.0f ? c.b / nn : 0.0f, f = c.a * w * U;
    n = nn;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const Two<float> m = across<O>(mean[j]), q = across<O>(m2[j]);
      const float d = m.b - m.a;
      mean[j] = __builtin_fmaf(d, w, m.a);
      m2[j] = q.a + __builtin_fmaf(d * d, f, q.b);
    }
  }
};

// LDS of the summing passes on W waves: two float64 per channel, two floats per
// wave and channel, a count per wave.  Sixteen waves take rows of at most 256
// channels.  (Row distances known to the compiler: as variables they cost 16
// addresses, kept in registers throughout.)
template <int W>
struct SumsLds {
  static constexpr int C = W == NW ? MAX_C : MAX_C / 2;
  double s1[C], s2[C];
  float u[W * C], v[W * C], n[W];
};

// The workgroup's moments joined: for every group the sum of all values and of
// their squares about zero, in float64, to out(g, u, v).
template <int W, bool VEC, typename OUT>
__device__ __forceinline__ void join_moments(const NormArgs& a, const Lanes<VEC>& L, Moments<VEC>& m, SumsLds<W>& sh,
                                             OUT out) {
  constexpr int U = UNIT<VEC>, N = CPL<VEC> / U, wu = SumsLds<W>::C / U;
  const int wid = threadIdx.x >> 6, lane = threadIdx.x & 63, c = threadIdx.x, units = a.C / U;
  levels(L.lpr, [&](auto o) { m.template join<decltype(o)::value>(); });
  if (lane < L.lpr) {
#pragma unroll
    for (int j = 0; j < N; ++j) sh.u[wid * wu + L.lr * N + j] = m.mean[j], sh.v[wid * wu + L.lr * N + j] = m.m2[j];
    if (lane == 0) sh.n[wid] = m.n;
  }
  __syncthreads();
  if (c < units) {
    double u = 0.0, v = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const double mw = sh.u[w * wu + c], nw = (double)(sh.n[w] * U), t = nw * mw;
      u += t;
      v += __builtin_fma(t, mw, (double)sh.v[w * wu + c]);
    }
    sh.s1[c] = u;
    sh.s2[c] = v;
  }
  __syncthreads();
  group_sums<W>(sh.s1, sh.s2, a.G, a.gs / U, out);
}

// A sum of squares about the mean that rounding has left below zero.  A NaN stays: an
// infinity among the values makes one of it while the mean may be infinite, and a finite
// rstd would then turn the group's other values into infinities, which ReLU hides.
__device__ __forceinline__ double not_negative(double x) { return x < 0.0 ? 0.0 : x; }

// First pass.  Per piece and group the mean and the sum of squares about it; adds and
// writes checkpoints on the way.  Bound by memory: 262,144 x 128 float32 with addend
// and sum 67 us (403 MB, 6.0 TB/s; the second pass's 37 us then reads from the cache in
// part); 285,564 x 128 with a checkpoint too 85 us (477 MB, 5.6 TB/s).  At 99,991 x 64
// bfloat16 in 37 segments 8.6 us for 12.8 MB: its chunks are 15 steps of rows, three whole
// tiles and then two halves, each waited for by itself, so that its launch, these loads'
// way and the joining over lanes and waves are what it takes.
template <typename T, bool VEC, bool ADD>
__global__ __launch_bounds__(NT, VEC ? 4 : 2) void k_norm_stats(NormArgs a) {
  __shared__ SumsLds<NW> sh;
  const Lanes<VEC> L(a.lg, a.C, NT);
  const Stream<T, VEC, ADD> in(a, L);
  const Keep<VEC> keep(a, L);
  for (int64_t p = blockIdx.x; p < a.pieces; p += gridDim.x) {
    const Piece pc(a, p);
    if (pc.end <= pc.r) continue;
    const double inv = 1.0 / ((double)(pc.end - pc.r) * a.gs);
    float2* part = a.part + p * a.G;
    Moments<VEC> m;
    over_rows<FWD_TILE<VEC>>(L, pc.r, pc.end, a.n, [&](int64_t i, const auto& rows) {
      float v[std::decay_t<decltype(rows)>::N][CPL<VEC>];
      in.load(i, rows, v);
      if (a.ck) keep.store(i, rows, v);
      m.add(v, rows);
    });
    join_moments(a, L, m, sh, [&](int g, double u, double v) {
      const double mean = u * inv;
      part[g] = make_float2((float)mean, (float)not_negative(v - u * mean));
    });
    __syncthreads();
  }
}

// mean and rstd of a group from its sums about zero
__device__ __forceinline__ float2 finish(double u, double v, double inv, float eps) {
  const double m = u * inv;
  return make_float2((float)m, 1.0f / sqrtf((float)not_negative(v * inv - m * m) + eps));
}

// ------------------------------------------------------------ joining the pieces

// Sums over the pieces of a segment for every group: term(piece's value, its rows,
// u, v) adds to two float64 sums; done(g, u, v) is called by one lane of each group.
// Consecutive lanes take consecutive groups.
template <int W, typename TERM, typename DONE>
__device__ __forceinline__ void join_pieces(const NormArgs& a, const Piece& pc, double* sh, TERM term,
                                            DONE done) {
  int lgp = 0;
  while ((1 << lgp) < a.G) ++lgp;
  const int gp = 1 << lgp, g = threadIdx.x & (gp - 1), p = threadIdx.x >> lgp, P = (W * 64) >> lgp;
  const int64_t b = pc.b, e = pc.e, j0 = (uint32_t)b / (uint32_t)a.R, j1 = (uint32_t)(e - 1) / (uint32_t)a.R;
  double u = 0.0, v = 0.0;
  if (g < a.G) {
    const float2* part = a.part + pc.s * (int64_t)a.G + g;
#pragma unroll 4
    for (int64_t j = j0 + p; j <= j1; j += P) {
      const int64_t rows = std::min<int64_t>(e, (j + 1) * a.R) - std::max<int64_t>(b, j * a.R);
      term(part[j * a.G], (double)(int32_t)rows, u, v);
    }
  }
  levels(gp, [&](auto o) {
    add_across<decltype(o)::value>(u);
    add_across<decltype(o)::value>(v);
  });
  if (gp >= 64) {
    // P sums of each group, gp apart
    sh[threadIdx.x] = u;
    sh[W * 64 + threadIdx.x] = v;
    __syncthreads();
    if (p == 0 && g < a.G) {
      for (int i = 1; i < P; ++i) u += sh[i * gp + g], v += sh[W * 64 + i * gp + g];
      done(g, u, v);
    }
  } else {
    const int wid = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (lane < gp) sh[wid * 64 + lane] = u, sh[W * 64 + wid * 64 + lane] = v;
    __syncthreads();
    if (threadIdx.x < (unsigned)a.G) {
#pragma unroll
      for (int w = 1; w < W; ++w) u += sh[w * 64 + g], v += sh[W * 64 + w * 64 + g];
      done(g, u, v);
    }
  }
  __syncthreads();
}

// ------------------------------------------------------------ forward, result

// y of rows [r, end) from their groups' mean and rstd.
template <typename T, bool VEC, int ACT>
__device__ __forceinline__ void apply_rows(const NormArgs& a, const Lanes<VEC>& L, int64_t r, int64_t end,
                                           const PerUnit<VEC>& mean, const PerUnit<VEC>& rstd, const float (&gamma)[CPL<VEC>],
                                           const float (&beta)[CPL<VEC>]) {
  const Source<T, VEC, !std::is_same<T, Q8>::value> in(a, L);   // their last use, but for a checkpoint
  const Result<VEC> out(a, L);
  float scale[CPL<VEC>];
#pragma unroll
  for (int k = 0; k < CPL<VEC>; ++k) scale[k] = rstd[k] * gamma[k];
  pass_rows<FWD_TILE<VEC>>(
      L, r, end, a.n,
      [&](int64_t i, const auto& rows, auto& v) {
#pragma unroll
        for (int t = 0; t < std::decay_t<decltype(rows)>::N; ++t)
          in.template load<std::decay_t<decltype(rows)>::FULL>(rows.first(i, t), rows.at(t), v[t]);
      },
      [&](int64_t i, const auto& rows, auto& v) {
#pragma unroll
        for (int t = 0; t < std::decay_t<decltype(rows)>::N; ++t) {
          if (rows.end(t)) break;
#pragma unroll
          for (int k = 0; k < CPL<VEC>; ++k)
            v[t][k] = activate<ACT>(__builtin_fmaf(v[t][k] - mean[k], scale[k], beta[k]));
          if (rows.ok(t)) out.store(rows.first(i, t), rows.at(t), v[t]);
        }
      });
}

// y = act((t - mean) * (rstd gamma) + beta), piece by piece.  a.merge: the statistics
// come from the first pass's pieces (and are written with the segment's first one),
// else from a.stats.  Every workgroup joins the sums of its segment's pieces itself, which
// costs it 2 to 3 us and saves a launch between the passes.  The next tile is loaded while
// one is written (pass_rows); the first one ahead of the joining too gave 1 to 2 us at
// 99,991 x 64 and took 4 at 285,564 x 128.  262,144 x 128 float32 to bfloat16 37 us
// (201 MB, 5.5 TB/s, part of it from the cache), restored from a checkpoint 19 us
// (103 MB, 5.4 TB/s); 99,991 x 64 bfloat16 in 37 segments 11 us (25.6 MB).
template <typename T, bool VEC, int ACT>
__global__ __launch_bounds__(NT, VEC ? 4 : 2) void k_norm_apply(NormArgs a) {
  __shared__ double sh[2 * NT];
  __shared__ float2 st[MAX_C];
  const Lanes<VEC> L(a.lg, a.C, NT);
  const Groups<VEC> groups(a, L.c0);
  float gamma[CPL<VEC>], beta[CPL<VEC>];
  params<VEC>(a, L, gamma, beta);
  for (int64_t p = blockIdx.x; p < a.pieces; p += gridDim.x) {
    const Piece pc(a, p);
    if (pc.end <= pc.r) {
      if (a.merge && pc.e <= pc.b)   // a segment of no rows has one number
        for (int g = threadIdx.x; g < a.G; g += NT) stats_of(a, pc.s)[g] = make_float2(0.0f, 0.0f);
      continue;
    }
    PerUnit<VEC> mean, rstd;
    if (a.merge) {
      const double inv = 1.0 / ((double)(pc.e - pc.b) * a.gs);
      join_pieces<NW>(
          a, pc, sh,
          [&](float2 t, double rows, double& u, double& v) {
            const double m = t.x, k = rows * a.gs;
            u += k * m;
            v += (double)t.y + k * m * m;
          },
          [&](int g, double u, double v) {
            st[g] = finish(u, v, inv, a.eps);
            if (pc.first) stats_of(a, pc.s)[g] = st[g];
          });
      groups.read(st, mean, rstd);
    } else {
      groups.read(stats_of(a, pc.s), mean, rstd);
    }
    apply_rows<T, VEC, ACT>(a, L, pc.r, pc.end, mean, rstd, gamma, beta);
  }
}

// One workgroup to a segment whose rows are one tile: they stay in registers
// between the statistics and the result.  1,024 x 32 float32 7.6 us, all of it latency
// (launch, one load's way, joining over lanes and waves, the store).
template <typename T, bool VEC, bool ADD, int ACT>
__global__ __launch_bounds__(SNT) void k_norm_small(NormArgs a) {
  constexpr int TILE = SMALL_TILE<VEC>;
  __shared__ SumsLds<SNW> sh;
  __shared__ float2 st[MAX_C];
  const Lanes<VEC> L(a.lg, a.C, SNT);
  const int s = blockIdx.x;
  const int64_t b = seg_begin(a, s), e = seg_end(a, s);
  if (e <= b) {
    for (int g = threadIdx.x; g < a.G; g += SNT) stats_of(a, s)[g] = make_float2(0.0f, 0.0f);
    return;
  }
  const Tile<TILE, false> rows(L, (int)(e - b));
  float v[TILE][CPL<VEC>], gamma[CPL<VEC>], beta[CPL<VEC>];
  Stream<T, VEC, ADD>(a, L).load(b, rows, v);
  params<VEC>(a, L, gamma, beta);
  const Groups<VEC> groups(a, L.c0);
  const double inv = 1.0 / ((double)(e - b) * a.gs);
  Moments<VEC> m;
  m.add(v, rows);
  if (a.ck) Keep<VEC>(a, L).store(b, rows, v);
  join_moments(a, L, m, sh, [&](int g, double u, double q) {
    st[g] = finish(u, q, inv, a.eps);
    stats_of(a, s)[g] = st[g];
  });
  __syncthreads();
  PerUnit<VEC> mean, rstd;
  groups.read(st, mean, rstd);
  const Result<VEC> out(a, L);
#pragma unroll
  for (int t = 0; t < TILE; ++t) {
    if (rows.end(t)) break;
#pragma unroll
    for (int k = 0; k < CPL<VEC>; ++k)
      v[t][k] = activate<ACT>(__builtin_fmaf(v[t][k] - mean[k], rstd[k] * gamma[k], beta[k]));
    if (rows.ok(t)) out.store(b, rows.at(t), v[t]);
  }
}

// ------------------------------------------------------------ backward

// What the backward passes know of a segment.
template <bool VEC>
struct Norm {
  PerUnit<VEC> mean, rstd;
  float gamma[CPL<VEC>], beta[CPL<VEC>];
  // of one row: w = grad_y act'(z) in place of grad_y, xn in place of t
  template <int ACT>
  __device__ __forceinline__ void weigh(float (&t)[CPL<VEC>], float (&w)[CPL<VEC>]) const {
#pragma unroll
    for (int k = 0; k < CPL<VEC>; ++k) {
      t[k] = (t[k] - mean[k]) * rstd[k];
      w[k] *= slope<ACT>(__builtin_fmaf(t[k], gamma[k], beta[k]));
    }
  }
};

// The lanes' sums u of w and v of w xn joined over the workgroup: per channel to
// chan(c, u, v), by the thread that has the number c; per group, times gamma, to
// out(g, u, v).
template <int W, bool VEC, typename CHAN, typename OUT>
__device__ __forceinline__ void join_sums(const NormArgs& a, const Lanes<VEC>& L, float (&u)[CPL<VEC>],
                                          float (&v)[CPL<VEC>], SumsLds<W>& sh, CHAN chan, OUT out) {
  constexpr int w8 = SumsLds<W>::C;
  const int wid = threadIdx.x >> 6, lane = threadIdx.x & 63, c = threadIdx.x;
  levels(L.lpr, [&](auto o) {
#pragma unroll
    for (int k = 0; k < CPL<VEC>; ++k) add_across<decltype(o)::value>(u[k]), add_across<decltype(o)::value>(v[k]);
  });
  const double gc = c < a.C && a.gamma ? a.gamma[c] : 1.0f;
  if (lane < L.lpr) {
#pragma unroll
    for (int k = 0; k < CPL<VEC>; ++k) sh.u[wid * w8 + L.c0 + k] = u[k], sh.v[wid * w8 + L.c0 + k] = v[k];
  }
  __syncthreads();
  if (c < a.C) {
    double x = 0.0, y = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) x += sh.u[w * w8 + c], y += sh.v[w * w8 + c];
    chan(c, x, y);
    sh.s1[c] = gc * x;
    sh.s2[c] = gc * y;
  }
  __syncthreads();
  group_sums<W>(sh.s1, sh.s2, a.G, a.gs, out);
}

// w and xn of a tile in place of grad_y and t, added to the lane's sums
template <int ACT, bool VEC, int N, bool FULL>
__device__ __forceinline__ void weigh_tile(const Norm<VEC>& nm, const Tile<N, FULL>& rows, float (&t)[N][CPL<VEC>],
                                           float (&w)[N][CPL<VEC>], float (&u)[CPL<VEC>], float (&v)[CPL<VEC>]) {
  if (!FULL) {
    arrived(t);
    arrived(w);
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if (rows.end(j)) break;
    nm.template weigh<ACT>(t[j], w[j]);
    if (rows.ok(j)) {
#pragma unroll
      for (int k = 0; k < CPL<VEC>; ++k) u[k] += w[j][k], v[k] = __builtin_fmaf(w[j][k], t[j][k], v[k]);
    }
  }
}

// First pass: per piece the groups' sums, per workgroup the channels'.  285,564 x 128
// from a checkpoint 34 us (185 MB, 5.4 TB/s); 262,144 x 128 from float32 values 47 us
// (268 MB, 5.7 TB/s); 8,192 x 64 bfloat16 5.4 us (3.1 MB, latency).
template <typename T, bool VEC, int ACT>
__global__ __launch_bounds__(NT, VEC ? 4 : 2) void k_norm_bwd_sums(NormArgs a) {
  __shared__ SumsLds<NW> sh;
  const Lanes<VEC> L(a.lg, a.C, NT);
  const Groups<VEC> groups(a, L.c0);
  Norm<VEC> nm;
  params<VEC>(a, L, nm.gamma, nm.beta);
  const Source<T, VEC> in(a, L);
  const Mat<float> gy(a.gy, a.ldgy, L.at(a.C));
  double cu = 0.0, cv = 0.0;
  for (int64_t p = blockIdx.x; p < a.pieces; p += gridDim.x) {
    const Piece pc(a, p);
    if (pc.end <= pc.r) continue;
    groups.read(stats_of(a, pc.s), nm.mean, nm.rstd);
    float2* part = a.part + p * a.G;
    float u[CPL<VEC>] = {}, v[CPL<VEC>] = {};
    over_rows<SUMS_TILE<VEC>>(L, pc.r, pc.end, a.n, [&](int64_t i, const auto& rows) {
      constexpr int N = std::decay_t<decltype(rows)>::N;
      constexpr bool FULL = std::decay_t<decltype(rows)>::FULL;
      float t[N][CPL<VEC>], w[N][CPL<VEC>];
#pragma unroll
      for (int j = 0; j < N; ++j) {
        in.template load<FULL>(rows.first(i, j), rows.at(j), t[j]);
        load_row<VEC, false, FULL>(gy.row(rows.first(i, j), rows.at(j)), L.cnt, w[j]);
      }
      weigh_tile<ACT>(nm, rows, t, w, u, v);
    });
    join_sums(
        a, L, u, v, sh, [&](int, double x, double y) { cu += x, cv += y; },
        [&](int g, double x, double y) { part[g] = make_float2((float)x, (float)y); });
    __syncthreads();
  }
  const int c = threadIdx.x;
  if (a.part_c && c < a.C) {
    a.part_c[(int64_t)blockIdx.x * 2 * a.C + c] = (float)cu;
    a.part_c[(int64_t)blockIdx.x * 2 * a.C + a.C + c] = (float)cv;
  }
}

// dbeta and dgamma from the workgroups' sums: 64 columns of part_c to a workgroup,
// the sums dealt to its waves, joined in wave order.
template <int W>
__device__ __forceinline__ void columns(const NormArgs& a, int block, double* sh) {
  const int col = block * 64 + (threadIdx.x & 63), wid = threadIdx.x >> 6;
  double v = 0.0;
  if (col < 2 * a.C) {
#pragma unroll 8
    for (int j = wid; j < a.parts; j += W) v += a.part_c[(int64_t)j * 2 * a.C + col];
  }
  sh[threadIdx.x] = v;
  __syncthreads();
  if (wid == 0 && col < 2 * a.C) {
    for (int w = 1; w < W; ++w) v += sh[w * 64 + threadIdx.x];
    float* p = col < a.C ? a.dbeta + col : a.dgamma + (col - a.C);
    *p = a.accumulate ? *p + (float)v : (float)v;
  }
}

// grad_x of one row from its groups' sums A and B, added to g
template <bool VEC>
__device__ __forceinline__ void grad_row(const Norm<VEC>& nm, const PerUnit<VEC>& A, const PerUnit<VEC>& B,
                                      const float (&w)[CPL<VEC>], const float (&xn)[CPL<VEC>], float (&g)[CPL<VEC>]) {
#pragma unroll
  for (int k = 0; k < CPL<VEC>; ++k)
    g[k] = __builtin_fmaf(nm.rstd[k], __builtin_fmaf(-xn[k], B[k], __builtin_fmaf(nm.gamma[k], w[k], -A[k])), g[k]);
}

template <typename T, bool VEC, int ACT>
__device__ __forceinline__ void grad_rows(const NormArgs& a, const Lanes<VEC>& L, const Norm<VEC>& nm, const PerUnit<VEC>& A,
                                          const PerUnit<VEC>& B, int64_t r, int64_t end) {
  const Source<T, VEC, true> in(a, L);
  const Mat<float> gy(a.gy, a.ldgy, L.at(a.C)), ga(a.ga, a.ldga, L.at(a.C)), gx(a.gx, a.ldgx, L.c0);
  over_rows<BWD_TILE<VEC>>(L, r, end, a.n, [&](int64_t i, const auto& rows) {
    using TL = std::decay_t<decltype(rows)>;
    float t[TL::N][CPL<VEC>], w[TL::N][CPL<VEC>], g[TL::N][CPL<VEC>] = {};
#pragma unroll
    for (int j = 0; j < TL::N; ++j) {
      in.template load<TL::FULL>(rows.first(i, j), rows.at(j), t[j]);
      load_row<VEC, true, TL::FULL>(gy.row(rows.first(i, j), rows.at(j)), L.cnt, w[j]);
      if (a.ga) load_row<VEC, true, TL::FULL>(ga.row(rows.first(i, j), rows.at(j)), L.cnt, g[j]);
    }
    if (!TL::FULL) {
      arrived(t);
      arrived(w);
      arrived(g);
    }
#pragma unroll
    for (int j = 0; j < TL::N; ++j) {
      if (rows.end(j)) break;
      nm.template weigh<ACT>(t[j], w[j]);
      grad_row(nm, A, B, w[j], t[j], g[j]);
      if (rows.ok(j)) store_row<VEC, true>(gx.row(rows.first(i, j), rows.at(j)), L.cnt, g[j]);
    }
  });
}

// Second pass.  The last workgroups, past a.grid, form dbeta and dgamma (4 us as a launch
// of their own).  285,564 x 128 from a checkpoint with grad_addend 77 us (477 MB,
// 6.2 TB/s, part of it from the cache); 262,144 x 128 from float32 values 82 us (537 MB,
// 6.5 TB/s); 8,192 x 64 bfloat16 5.4 us (5.2 MB, latency).
// Pieces in the opposite order (last read, first used) made no difference.
template <typename T, bool VEC, int ACT>
__global__ __launch_bounds__(NT, VEC ? 4 : 2) void k_norm_bwd_dx(NormArgs a) {
  __shared__ double sh[2 * NT];
  __shared__ float2 st[MAX_C];
  if ((int)blockIdx.x >= a.grid) {
    columns<NW>(a, blockIdx.x - a.grid, sh);
    return;
  }
  const Lanes<VEC> L(a.lg, a.C, NT);
  const Groups<VEC> groups(a, L.c0);
  Norm<VEC> nm;
  params<VEC>(a, L, nm.gamma, nm.beta);
  for (int64_t p = blockIdx.x; p < a.pieces; p += a.grid) {
    const Piece pc(a, p);
    if (pc.end <= pc.r) continue;
    groups.read(stats_of(a, pc.s), nm.mean, nm.rstd);
    const double inv = 1.0 / ((double)(pc.e - pc.b) * a.gs);
    join_pieces<NW>(
        a, pc, sh, [&](float2 t, double, double& u, double& v) { u += t.x, v += t.y; },
        [&](int g, double u, double v) { st[g] = make_float2((float)(u * inv), (float)(v * inv)); });
    PerUnit<VEC> A, B;
    groups.read(st, A, B);
    grad_rows<T, VEC, ACT>(a, L, nm, A, B, pc.r, pc.end);
  }
}

// One segment of one tile of rows, one workgroup: w and xn stay in registers.
// 1,000 x 32 from a checkpoint 9.8 us.
template <typename T, bool VEC, int ACT>
__global__ __launch_bounds__(SNT) void k_norm_bwd_small(NormArgs a) {
  constexpr int TILE = SMALL_TILE<VEC>;
  __shared__ SumsLds<SNW> sh;
  __shared__ float2 st[MAX_C];
  const Lanes<VEC> L(a.lg, a.C, SNT);
  const Tile<TILE, false> rows(L, (int)a.n);
  const Source<T, VEC> in(a, L);
  const Mat<float> gy(a.gy, a.ldgy, L.at(a.C)), ga(a.ga, a.ldga, L.at(a.C)), gx(a.gx, a.ldgx, L.c0);
  float t[TILE][CPL<VEC>], w[TILE][CPL<VEC>], u[CPL<VEC>] = {}, v[CPL<VEC>] = {};
#pragma unroll
  for (int j = 0; j < TILE; ++j) {
    in.template load<false>(0, rows.at(j), t[j]);
    load_row<VEC, false>(gy.row(0, rows.at(j)), L.cnt, w[j]);
  }
  const Groups<VEC> groups(a, L.c0);
  Norm<VEC> nm;
  params<VEC>(a, L, nm.gamma, nm.beta);
  groups.read(stats_of(a, 0), nm.mean, nm.rstd);
  weigh_tile<ACT>(nm, rows, t, w, u, v);
  const double inv = 1.0 / ((double)a.n * a.gs);
  join_sums(
      a, L, u, v, sh,
      [&](int c, double x, double y) {
        if (!a.dbeta) return;
        a.dbeta[c] = a.accumulate ? a.dbeta[c] + (float)x : (float)x;
        a.dgamma[c] = a.accumulate ? a.dgamma[c] + (float)y : (float)y;
      },
      [&](int g, double x, double y) { st[g] = make_float2((float)(x * inv), (float)(y * inv)); });
  __syncthreads();
  PerUnit<VEC> A, B;
  groups.read(st, A, B);
#pragma unroll
  for (int j = 0; j < TILE; ++j) {
    if (rows.end(j)) break;
    float g[CPL<VEC>] = {};
    if (a.ga) load_row<VEC, false>(ga.row(0, rows.at(j)), L.cnt, g);
    grad_row(nm, A, B, w[j], t[j], g);
    if (rows.ok(j)) store_row<VEC, true>(gx.row(0, rows.at(j)), L.cnt, g);
  }
}

// dbeta and dgamma alone (rows as segments, no rows at all)
__global__ __launch_bounds__(SNT) void k_norm_columns(NormArgs a) {
  __shared__ double sh[SNT];
  columns<SNW>(a, blockIdx.x, sh);
}

// ------------------------------------------------------------ each row a segment

// Sums over the groups of a row.  How depends on the group: a unit by itself;
// whole lanes, a power of two of them (or the whole row), by shuffles; any
// other through the wave's LDS.
template <bool VEC>
struct RowGroups {
  static constexpr int U = UNIT<VEC>, N = CPL<VEC> / U;
  int width;     // lanes of a group; 0: a unit; -1: through LDS
  int at[N];     // first unit of each unit's group
  float* lds;    // the wave's 64 N floats

  __device__ __forceinline__ RowGroups(const NormArgs& a, const Lanes<VEC>& L, float* wave_lds) : lds(wave_lds) {
    const int lanes = a.gs / CPL<VEC>, gu = a.gs / U;
    width = gu == 1 ? 0 : a.G == 1 ? L.lpr : (a.gs % CPL<VEC> == 0 && (lanes & (lanes - 1)) == 0) ? lanes : -1;
#pragma unroll
    for (int j = 0; j < N; ++j) at[j] = std::min(L.lr * N + j, a.C / U - 1) / gu * gu;
  }
  // p: this lane's values; the sum over its group for each unit
  __device__ __forceinline__ PerUnit<VEC> sum(const NormArgs& a, const Lanes<VEC>& L, const float (&p)[CPL<VEC>]) const {
    PerUnit<VEC> s;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      s.v[j] = p[j * U];
#pragma unroll
      for (int k = 1; k < U; ++k) s.v[j] += p[j * U + k];
    }
    if (width > 0) {
      float t = s.v[0];
#pragma unroll
      for (int j = 1; j < N; ++j) t += s.v[j];
      t = L.cnt > 0 ? t : 0.0f;
      t = sum_lanes(t, width);
#pragma unroll
      for (int j = 0; j < N; ++j) s.v[j] = t;
    } else if (width < 0) {
      float* row = lds + ((threadIdx.x & 63) - L.lr) * N;
#pragma unroll
      for (int j = 0; j < N; ++j) row[L.lr * N + j] = s.v[j];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int j = 0; j < N; ++j) {
        float t = 0.0f;
        for (int i = 0; i < a.gs / U; ++i) t += row[at[j] + i];
        s.v[j] = t;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    return s;
  }
};

// A row's statistics need only its own lanes: one pass, mean and then deviations from
// it in registers.  No tiles: many small workgroups (16 to a CU) hide the loads.
// 8,192 x 64 bfloat16 3.6 us (2.1 MB); 262,144 x 128 float32 to bfloat16 41 us (218 MB,
// 5.3 TB/s).
template <typename T, bool VEC, bool ADD, int ACT>
__global__ __launch_bounds__(RNT) void k_norm_rows(NormArgs a) {
  constexpr int U = UNIT<VEC>, N = CPL<VEC> / U;
  __shared__ float lds[RNT * N];
  const Lanes<VEC> L(a.lg, a.C, RNT);
  const RowGroups<VEC> R(a, L, lds + (threadIdx.x >> 6) * 64 * N);
  const Groups<VEC> groups(a, L.c0);
  float gamma[CPL<VEC>], beta[CPL<VEC>];
  params<VEC>(a, L, gamma, beta);
  const float f = 1.0f / a.gs;
  const Stream<T, VEC, ADD> in(a, L);
  const Keep<VEC> keep(a, L);
  const Result<VEC> out(a, L);
  const Mat<float2> st(a.stats, a.G, 0);
  each_row(L, a.n, [&](int64_t i, auto whole) {
    constexpr bool WIDE = decltype(whole)::value;
    float t[1][CPL<VEC>], q[CPL<VEC>];
    const Tile<1, WIDE> row(L, L.RL);
    in.load(i, row, t);
    float(&v)[CPL<VEC>] = t[0];
    if (a.ck) keep.store(i, row, t);
    PerUnit<VEC> mean = R.sum(a, L, v), rstd;
#pragma unroll
    for (int j = 0; j < N; ++j) mean.v[j] *= f;
#pragma unroll
    for (int k = 0; k < CPL<VEC>; ++k) {
      const float d = k < L.cnt ? v[k] - mean[k] : 0.0f;
      q[k] = d * d;
    }
    rstd = R.sum(a, L, q);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      rstd.v[j] = 1.0f / sqrtf(__builtin_fmaf(rstd.v[j], f, a.eps));
      // a group's first unit writes for it
      if (j * U < L.cnt && L.lr * N + j == R.at[j])
        st.row(i, L.rl)[groups.g[j]] = make_float2(mean.v[j], rstd.v[j]);
    }
#pragma unroll
    for (int k = 0; k < CPL<VEC>; ++k)
      v[k] = activate<ACT>(__builtin_fmaf((v[k] - mean[k]) * rstd[k], gamma[k], beta[k]));
    out.store(i, L.rl, v);
  });
}

// 262,144 x 128 to bfloat16 21 us (119 MB, 5.6 TB/s).
template <bool VEC, int ACT>
__global__ __launch_bounds__(RNT) void k_norm_rows_restore(NormArgs a) {
  const Lanes<VEC> L(a.lg, a.C, RNT);
  const Groups<VEC> groups(a, L.c0);
  float gamma[CPL<VEC>], beta[CPL<VEC>];
  params<VEC>(a, L, gamma, beta);
  const Source<Q8, VEC> in(a, L);
  const Result<VEC> out(a, L);
  const Mat<float2> st(a.stats, a.G, 0);
  each_row(L, a.n, [&](int64_t i, auto whole) {
    constexpr bool WIDE = decltype(whole)::value;
    float v[CPL<VEC>];
    PerUnit<VEC> mean, rstd;
    in.template load<WIDE>(i, L.rl, v);
    groups.read(st.row(i, L.rl), mean, rstd);
#pragma unroll
    for (int k = 0; k < CPL<VEC>; ++k)
      v[k] = activate<ACT>(__builtin_fmaf((v[k] - mean[k]) * rstd[k], gamma[k], beta[k]));
    out.store(i, L.rl, v);
  });
}

// The channels' sums stay in registers over all rows of a workgroup (4 to a CU, at most
// ROW_PARTS: so many sums are joined by k_norm_columns).  100,000 x 128 float32 with
// grad_addend 39 us (211 MB, 5.4 TB/s) and 4.6 us for the columns.
template <typename T, bool VEC, int ACT>
__global__ __launch_bounds__(RNT) void k_norm_rows_bwd(NormArgs a) {
  constexpr int N = CPL<VEC> / UNIT<VEC>;
  __shared__ float lds[RNT * 16];
  const Lanes<VEC> L(a.lg, a.C, RNT);
  const RowGroups<VEC> R(a, L, lds + (threadIdx.x >> 6) * 64 * N);
  const Groups<VEC> groups(a, L.c0);
  Norm<VEC> nm;
  float u[CPL<VEC>] = {}, v[CPL<VEC>] = {};
  params<VEC>(a, L, nm.gamma, nm.beta);
  const float f = 1.0f / a.gs;
  const Source<T, VEC> in(a, L);
  const Mat<float> gy(a.gy, a.ldgy, L.at(a.C)), ga(a.ga, a.ldga, L.at(a.C)), gx(a.gx, a.ldgx, L.c0);
  const Mat<float2> st(a.stats, a.G, 0);
  each_row(L, a.n, [&](int64_t i, auto whole) {
    constexpr bool WIDE = decltype(whole)::value;
    float t[CPL<VEC>], w[CPL<VEC>], g[CPL<VEC>] = {}, x[CPL<VEC>], y[CPL<VEC>];
    in.template load<WIDE>(i, L.rl, t);
    load_row<VEC, false, WIDE>(gy.row(i, L.rl), L.cnt, w);
    if (a.ga) load_row<VEC, false, WIDE>(ga.row(i, L.rl), L.cnt, g);
    groups.read(st.row(i, L.rl), nm.mean, nm.rstd);
    nm.template weigh<ACT>(t, w);
#pragma unroll
    for (int k = 0; k < CPL<VEC>; ++k) {
      if (k >= L.cnt) w[k] = 0.0f;
      u[k] += w[k];
      v[k] = __builtin_fmaf(w[k], t[k], v[k]);
      x[k] = k < L.cnt ? nm.gamma[k] * w[k] : 0.0f;
      y[k] = k < L.cnt ? x[k] * t[k] : 0.0f;
    }
    PerUnit<VEC> A = R.sum(a, L, x), B = R.sum(a, L, y);
#pragma unroll
    for (int j = 0; j < N; ++j) A.v[j] *= f, B.v[j] *= f;
    grad_row(nm, A, B, w, t, g);
    store_row<VEC, true>(gx.row(i, L.rl), L.cnt, g);
  });
  if (!a.part_c) return;
  levels(L.lpr, [&](auto o) {
#pragma unroll
    for (int k = 0; k < CPL<VEC>; ++k) add_across<decltype(o)::value>(u[k]), add_across<decltype(o)::value>(v[k]);
  });
  __syncthreads();
  const int w8 = L.lpr * CPL<VEC>, wid = threadIdx.x >> 6;
  if ((threadIdx.x & 63) < (unsigned)L.lpr) {
#pragma unroll
    for (int k = 0; k < CPL<VEC>; ++k) lds[wid * 2 * w8 + L.c0 + k] = u[k], lds[wid * 2 * w8 + w8 + L.c0 + k] = v[k];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < a.C; c += RNT) {
    double x = 0.0, y = 0.0;
    for (int w = 0; w < RNT / 64; ++w) x += lds[w * 2 * w8 + c], y += lds[w * 2 * w8 + w8 + c];
    a.part_c[(int64_t)blockIdx.x * 2 * a.C + c] = (float)x;
    a.part_c[(int64_t)blockIdx.x * 2 * a.C + a.C + c] = (float)y;
  }
}

// ------------------------------------------------------------ checkpoints alone

// One read, one write; as in the norm's passes, with no statistics to wait for.  A
// bfloat16 or float32 value is kept as an 8-bit multiple of its block's scale,
// rounded to nearest: off by at most half a scale, 1 / 254 of the block's largest.
// 100,000 x 256 float32 stored and loaded as bfloat16: 42 us for both (208 MB,
// 4.9 TB/s); 8,191 x 96 bfloat16 7 us for both.
template <typename T, bool VEC>
__global__ __launch_bounds__(RNT) void k_ckpt_store(NormArgs a) {
  const Lanes<VEC> L(a.lg, a.C, RNT);
  const Source<T, VEC> in(a, L);
  const Keep<VEC> keep(a, L);
  each_row(L, a.n, [&](int64_t i, auto whole) {
    constexpr bool WIDE = decltype(whole)::value;
    float v[1][CPL<VEC>];
    in.template load<WIDE>(i, L.rl, v[0]);
    keep.store(i, Tile<1, WIDE>(L, L.RL), v);
  });
}

template <bool VEC>
__global__ __launch_bounds__(RNT) void k_ckpt_load(NormArgs a) {
  const Lanes<VEC> L(a.lg, a.C, RNT);
  const Source<Q8, VEC> in(a, L);
  const Result<VEC> out(a, L);
  each_row(L, a.n, [&](int64_t i, auto whole) {
    constexpr bool WIDE = decltype(whole)::value;
    float v[CPL<VEC>];
    in.template load<WIDE>(i, L.rl, v);
    out.store(i, L.rl, v);
  });
}

// ------------------------------------------------------------ host side

int lanes_log2(int C, bool vec) {
  int lg = 0;
  while (((vec ? CPL<true> : CPL<false>) << lg) < C) ++lg;
  return lg;
}

// Chunks of rows: whole steps of a workgroup, at most `most` of them.  most_chunks:
// so many that the pieces are not more than the CUs (a few more would leave most
// CUs idle while some have two: 37 segments on 256 chunks 14.5 us instead of 11.5 for
// the second pass over 99,991 x 64), unless the segments alone are half as many.
int most_chunks(int64_t n_seg, int most) { return (int)std::max<int64_t>(most / 2, most + 1 - n_seg); }

void chunking(int64_t n, int lg, int64_t& rows, int64_t& chunks, int most) {
  const int64_t step = NT >> lg;
  const int64_t steps = (n + step - 1) / step;
  rows = std::max<int64_t>(1, (steps + most - 1) / most) * step;
  chunks = (n + rows - 1) / rows;
}

// whole aligned groups of four values in every row
bool aligned(const void* p, int64_t ld, int size) {
  return !p || (reinterpret_cast<uintptr_t>(p) % (4 * size) == 0 && ld % 4 == 0);
}

// (mean, rstd) are read and written in one
bool pairs(const float* stats) { return (reinterpret_cast<uintptr_t>(stats) & 7) == 0; }

int size_of(int dtype) { return dtype == DSMP_BF16 ? 2 : 4; }

// Row distances: at least the channels, and small enough that the rows of a tile
// of a workgroup (8 steps of at most 1,024 rows) lie within 32 bits.
constexpr int64_t MAX_LD = (int64_t)1 << 16;
dsmp_status check_ld(dsmp_handle* h, int C, std::initializer_list<int64_t> lds) {
  for (const int64_t ld : lds) {
    DSMP_CHECK(h, ld >= C, DSMP_INVALID_ARG, "rows are closer than their channels");
    DSMP_CHECK(h, ld <= MAX_LD, DSMP_UNSUPPORTED, "rows more than %lld elements apart", (long long)MAX_LD);
  }
  return DSMP_OK;
}

bool rows_are_segments(const dsmp_segments& s) { return !s.ptr && s.n_seg == s.n; }

dsmp_status check_norm(dsmp_handle* h, const dsmp_norm_desc* d, const dsmp_segments* s) {
  DSMP_CHECK(h, d && s, DSMP_INVALID_ARG, "the descriptor or the segments are NULL");
  DSMP_CHECK(h, d->channels >= 1 && d->groups >= 1 && d->channels % d->groups == 0, DSMP_INVALID_ARG,
             "groups must divide channels");
  DSMP_CHECK(h, d->channels <= MAX_C, DSMP_UNSUPPORTED, "more than %d channels", MAX_C);
  DSMP_CHECK(h, (d->x_dtype == DSMP_F32 || d->x_dtype == DSMP_BF16) && (d->y_dtype == DSMP_F32 || d->y_dtype == DSMP_BF16),
             DSMP_INVALID_ARG, "unknown dtype");
  DSMP_CHECK(h, d->act >= DSMP_ACT_IDENTITY && d->act <= DSMP_ACT_GELU, DSMP_INVALID_ARG, "unknown activation");
  DSMP_CHECK(h, d->eps >= 0.0f && std::isfinite(d->eps), DSMP_INVALID_ARG, "eps must be finite and not negative");
  DSMP_CHECK(h, s->n >= 0 && s->n_seg >= 1, DSMP_INVALID_ARG, "negative rows or no segment");
  DSMP_CHECK(h, s->n < (int64_t)1 << 31 && s->n_seg < (int64_t)1 << 31, DSMP_UNSUPPORTED, "2^31 rows or segments and more");
  DSMP_CHECK(h, s->ptr || s->n % s->n_seg == 0, DSMP_INVALID_ARG, "segments without ptr must divide the rows");
  return DSMP_OK;
}

struct NormWs {
  float2* part;
  float* part_c;
  size_t total;
};

NormWs norm_ws(const dsmp_norm_desc& d, const dsmp_segments& s, bool backward, void* ws) {
  int64_t rows, chunks, wide;
  const int most = most_chunks(s.n_seg, MAX_CHUNKS);
  chunking(s.n, lanes_log2(d.channels, false), rows, chunks, most);
  chunking(s.n, lanes_log2(d.channels, true), rows, wide, most);
  chunks = std::max(chunks, wide);
  Carve cv(ws);
  NormWs w{};
  w.part = cv.take<float2>(rows_are_segments(s) ? 0 : (size_t)(chunks + s.n_seg) * d.groups);
  if (backward) w.part_c = cv.take<float>((size_t)(rows_are_segments(s) ? ROW_PARTS : std::min<int64_t>(chunks + s.n_seg, MAX_GRID)) * 2 * d.channels);
  w.total = cv.used();
  return w;
}

NormArgs norm_args(const dsmp_norm_desc& d, const dsmp_segments& s) {
  NormArgs a{};
  a.n = s.n;
  a.C = d.channels;
  a.G = d.groups;
  a.gs = d.channels / d.groups;
  a.n_seg = (int)s.n_seg;
  a.ptr = s.ptr;
  a.len = s.ptr ? 0 : s.n / s.n_seg;
  a.eps = d.eps;
  return a;
}

// Lanes and chunks.
void place(NormArgs& a, bool vec, int most = MAX_CHUNKS) {
  int64_t chunks;
  a.lg = lanes_log2(a.C, vec);
  chunking(a.n, a.lg, a.R, chunks, most_chunks(a.n_seg, most));
  a.pieces = chunks + a.n_seg;
  a.grid = (int)std::min<int64_t>(a.pieces, MAX_GRID);
}

unsigned row_grid(const dsmp_handle* h, const NormArgs& a, int per_cu) {
  const int64_t step = RNT >> a.lg;
  return (unsigned)std::min<int64_t>((a.n + step - 1) / step, (int64_t)h->n_cu * per_cu);
}

// the channels, groups and parameters that VEC asks for
bool whole(const NormArgs& a) {
  return a.C <= MAX_C / 2 && a.gs % 4 == 0 && aligned(a.gamma, 0, 4) && aligned(a.beta, 0, 4);
}

// One launch with a workgroup to a segment: where all the rows are at most one
// tile of a workgroup, however they are dealt to the segments (and its LDS
// stays within 64 KB).  1,000 x 32 float32 on the GPU, one launch against two:
// forward 7.6 / 4.7 + 4.2 us, backward 9.6 / 4.7 + 5.2.  With an addend and a
// checkpoint 13.9 / 6.2 + 3.6, where one CU does all the work, but the calls are
// bound by the host: forward, restore and backward in a row take 29.1 us with one
// launch for it, 31.0 with two.  Not for more segments than the pieces are dealt to
// (most are empty then): a launch has fewer than 2^32 threads.
bool small(const NormArgs& a, bool vec) {
  return a.C <= MAX_C / 2 && a.n_seg <= MAX_GRID &&
         a.n <= (int64_t)(vec ? SMALL_TILE<true> : SMALL_TILE<false>) * (SNT >> a.lg);
}

template <typename F>
void by_bool(bool b, F f) {
  if (b)
    f(std::true_type{});
  else
    f(std::false_type{});
}
template <typename F>
void by_type(int dtype, F f) {
  if (dtype == DSMP_BF16)
    f(__bf16{});
  else
    f(float{});
}

template <typename F>
void by_act(int act, F f) {
  switch (act) {
    case DSMP_ACT_RELU: return f(std::integral_constant<int, DSMP_ACT_RELU>{});
    case DSMP_ACT_SILU: return f(std::integral_constant<int, DSMP_ACT_SILU>{});
    case DSMP_ACT_GELU: return f(std::integral_constant<int, DSMP_ACT_GELU>{});
    default: return f(std::integral_constant<int, DSMP_ACT_IDENTITY>{});
  }
}

}  // namespace

#define DSMP_GO(kernel, grid, threads, lds) hipLaunchKernelGGL((kernel), dim3(grid), dim3(threads), lds, h->stream, a)

extern "C" dsmp_status dsmp_group_norm_workspace(const dsmp_norm_desc* desc, const dsmp_segments* seg,
                                                 size_t* fwd_ws_bytes, size_t* bwd_ws_bytes) {
  const dsmp_status st = check_norm(nullptr, desc, seg);
  if (st != DSMP_OK) return st;
  if (!fwd_ws_bytes || !bwd_ws_bytes) return DSMP_INVALID_ARG;
  *fwd_ws_bytes = norm_ws(*desc, *seg, false, nullptr).total;
  *bwd_ws_bytes = norm_ws(*desc, *seg, true, nullptr).total;
  return DSMP_OK;
}

extern "C" dsmp_status dsmp_group_norm_forward(dsmp_handle* h, const dsmp_norm_desc* desc, const dsmp_segments* seg,
                                               const void* x, int64_t ldx, const void* addend, int64_t lda, void* sum,
                                               int64_t lds, const float* gamma, const float* beta, void* y,
                                               int64_t ldy, float* stats, const dsmp_checkpoint* ck, void* ws,
                                               size_t ws_bytes) {
  if (!h) return DSMP_INVALID_ARG;
  dsmp_status st = check_norm(h, desc, seg);
  if (st != DSMP_OK) return st;
  const int64_t n = seg->n;
  const int C = desc->channels;
  DSMP_CHECK(h, stats && (n == 0 || (x && y)), DSMP_INVALID_ARG, "a data pointer is NULL");
  DSMP_CHECK(h, pairs(stats), DSMP_INVALID_ARG, "stats must be 8-byte aligned");
  DSMP_CHECK(h, !gamma == !beta, DSMP_INVALID_ARG, "gamma and beta go together");
  DSMP_CHECK(h, !addend == !sum, DSMP_INVALID_ARG, "an addend and the sum go together");
  DSMP_CHECK(h, !ck || n == 0 || (ck->q && ck->scale), DSMP_INVALID_ARG, "a checkpoint pointer is NULL");
  st = check_ld(h, C, {ldx, ldy, addend ? lda : C, addend ? lds : C});
  if (st != DSMP_OK) return st;
  const NormWs w = norm_ws(*desc, *seg, false, ws);
  DSMP_CHECK(h, ws_bytes >= w.total && (ws || w.total == 0), DSMP_WORKSPACE_TOO_SMALL, "workspace needs %zu bytes", w.total);
  NormArgs a = norm_args(*desc, *seg);
  a.x = x, a.ldx = ldx, a.add = addend, a.lda = lda, a.sum = sum, a.lds = lds;
  a.gamma = gamma, a.beta = beta, a.y = y, a.ldy = ldy, a.stats = stats;
  if (ck) a.q = ck->q, a.scale = ck->scale;
  a.part = w.part;
  a.merge = 1;
  a.ck = ck != nullptr;
  a.y_bf16 = desc->y_dtype == DSMP_BF16;
  const int xs = size_of(desc->x_dtype);
  const bool vec = whole(a) && aligned(x, ldx, xs) && aligned(addend, lda, xs) && aligned(sum, lds, xs) &&
                   aligned(y, ldy, size_of(desc->y_dtype)) && (!ck || aligned(ck->q, C, 1));
  place(a, vec);
  ProfScope prof(h, DSMP_K_NORM);
  by_type(desc->x_dtype, [&](auto xt) {
    by_bool(vec, [&](auto v) {
      by_act(desc->act, [&](auto act) {
        using T = decltype(xt);
        constexpr bool V = decltype(v)::value;
        constexpr int ACT = decltype(act)::value;
        if (rows_are_segments(*seg)) {
          by_bool(addend, [&](auto ad) {
            DSMP_GO((k_norm_rows<T, V, decltype(ad)::value, ACT>), row_grid(h, a, 16), RNT, 0);
          });
        } else if (small(a, vec)) {
          by_bool(addend, [&](auto ad) {
            DSMP_GO((k_norm_small<T, V, decltype(ad)::value, ACT>), a.n_seg, SNT, 0);
          });
        } else {
          by_bool(addend, [&](auto ad) {
            DSMP_GO((k_norm_stats<T, V, decltype(ad)::value>), a.grid, NT, 0);
          });
          if (addend) a.x = sum, a.ldx = lds;
          DSMP_GO((k_norm_apply<T, V, ACT>), a.grid, NT, 0);
        }
      });
    });
  });
  DSMP_LAUNCHED(h, "group norm forward");
  return DSMP_OK;
}

extern "C" dsmp_status dsmp_group_norm_restore(dsmp_handle* h, const dsmp_norm_desc* desc, const dsmp_segments* seg,
                                               const dsmp_checkpoint* ck, const float* stats, const float* gamma,
                                               const float* beta, void* y, int64_t ldy) {
  if (!h) return DSMP_INVALID_ARG;
  dsmp_status st = check_norm(h, desc, seg);
  if (st != DSMP_OK) return st;
  const int C = desc->channels;
  DSMP_CHECK(h, seg->n == 0 || (ck && ck->q && ck->scale && stats && y), DSMP_INVALID_ARG, "a data pointer is NULL");
  DSMP_CHECK(h, pairs(stats), DSMP_INVALID_ARG, "stats must be 8-byte aligned");
  DSMP_CHECK(h, !gamma == !beta, DSMP_INVALID_ARG, "gamma and beta go together");
  st = check_ld(h, C, {ldy});
  if (st != DSMP_OK || seg->n == 0) return st;
  NormArgs a = norm_args(*desc, *seg);
  a.x = ck->q, a.xscale = ck->scale;
  a.gamma = gamma, a.beta = beta, a.y = y, a.ldy = ldy, a.stats = const_cast<float*>(stats);
  a.y_bf16 = desc->y_dtype == DSMP_BF16;
  const bool vec = whole(a) && aligned(y, ldy, size_of(desc->y_dtype)) && aligned(ck->q, C, 1);
  place(a, vec, MAX_PARTS);
  ProfScope prof(h, DSMP_K_NORM);
  by_bool(vec, [&](auto v) {
    by_act(desc->act, [&](auto act) {
      constexpr bool V = decltype(v)::value;
      constexpr int ACT = decltype(act)::value;
      if (rows_are_segments(*seg)) {
        DSMP_GO((k_norm_rows_restore<V, ACT>), row_grid(h, a, 16), RNT, 0);
      } else {
        DSMP_GO((k_norm_apply<Q8, V, ACT>), a.grid, NT, 0);
      }
    });
  });
  DSMP_LAUNCHED(h, "group norm restore");
  return DSMP_OK;
}

extern "C" dsmp_status dsmp_group_norm_backward(dsmp_handle* h, const dsmp_norm_desc* desc, const dsmp_segments* seg,
                                                const void* x, int64_t ldx, const dsmp_checkpoint* ck,
                                                const float* stats, const float* gamma, const float* beta,
                                                const float* grad_y, int64_t ldgy, const float* grad_addend,
                                                int64_t ldga, float* grad_x, int64_t ldgx, float* dgamma, float* dbeta,
                                                int32_t flags, void* ws, size_t ws_bytes) {
  if (!h) return DSMP_INVALID_ARG;
  dsmp_status st = check_norm(h, desc, seg);
  if (st != DSMP_OK) return st;
  const int64_t n = seg->n;
  const int C = desc->channels;
  DSMP_CHECK(h, (flags & ~DSMP_GRAD_ACCUMULATE) == 0, DSMP_INVALID_ARG, "unknown flags");
  DSMP_CHECK(h, !x || !ck, DSMP_INVALID_ARG, "x or its checkpoint, not both");
  DSMP_CHECK(h, n == 0 || ((x || (ck && ck->q && ck->scale)) && stats && grad_y && grad_x), DSMP_INVALID_ARG,
             "a data pointer is NULL");
  DSMP_CHECK(h, pairs(stats), DSMP_INVALID_ARG, "stats must be 8-byte aligned");
  DSMP_CHECK(h, !gamma == !beta && !gamma == !dgamma && !gamma == !dbeta, DSMP_INVALID_ARG,
             "gamma, beta and their gradients go together");
  st = check_ld(h, C, {x ? ldx : C, ldgy, ldgx, grad_addend ? ldga : C});
  if (st != DSMP_OK) return st;
  const NormWs w = norm_ws(*desc, *seg, true, ws);
  DSMP_CHECK(h, ws && ws_bytes >= w.total, DSMP_WORKSPACE_TOO_SMALL, "workspace needs %zu bytes", w.total);
  NormArgs a = norm_args(*desc, *seg);
  a.x = ck ? ck->q : x, a.ldx = ldx;
  if (ck) a.xscale = ck->scale;
  a.gamma = gamma, a.beta = beta, a.stats = const_cast<float*>(stats);
  a.gy = grad_y, a.ldgy = ldgy, a.ga = grad_addend, a.ldga = ldga, a.gx = grad_x, a.ldgx = ldgx;
  a.dgamma = dgamma, a.dbeta = dbeta, a.accumulate = flags & DSMP_GRAD_ACCUMULATE;
  a.part = w.part, a.part_c = gamma ? w.part_c : nullptr;
  const unsigned nred = gamma ? ceil_div(2 * C, 64) : 0;
  const bool vec = whole(a) && aligned(x, ldx, size_of(desc->x_dtype)) && aligned(grad_y, ldgy, 4) &&
                   aligned(grad_addend, ldga, 4) && aligned(grad_x, ldgx, 4) && (!ck || aligned(ck->q, C, 1));
  place(a, vec);
  ProfScope prof(h, DSMP_K_NORM);
  if (n == 0) {
    if (nred) DSMP_GO(k_norm_columns, nred, SNT, 0);   // sums of no chunk
    DSMP_LAUNCHED(h, "group norm backward");
    return DSMP_OK;
  }
  auto go = [&](auto xt) {
    by_bool(vec, [&](auto v) {
      by_act(desc->act, [&](auto act) {
        using T = decltype(xt);
        constexpr bool V = decltype(v)::value;
        constexpr int ACT = decltype(act)::value;
        if (rows_are_segments(*seg)) {
          const unsigned grid = std::min<unsigned>(row_grid(h, a, 4), ROW_PARTS);
          a.parts = (int)grid;
          DSMP_GO((k_norm_rows_bwd<T, V, ACT>), grid, RNT, 0);
          if (nred) DSMP_GO(k_norm_columns, nred, SNT, 0);
        } else if (small(a, vec) && a.n_seg == 1) {
          DSMP_GO((k_norm_bwd_small<T, V, ACT>), 1, SNT, 0);
        } else {
          a.parts = a.grid;
          DSMP_GO((k_norm_bwd_sums<T, V, ACT>), a.grid, NT, 0);
          DSMP_GO((k_norm_bwd_dx<T, V, ACT>), a.grid + nred, NT, 0);
        }
      });
    });
  };
  if (ck)
    go(Q8{});
  else
    by_type(desc->x_dtype, go);
  DSMP_LAUNCHED(h, "group norm backward");
  return DSMP_OK;
}

namespace {

dsmp_status check_ckpt(dsmp_handle* h, const dsmp_checkpoint* ck, const void* p, int32_t dtype, int64_t ld, int64_t n,
                       int32_t C) {
  DSMP_CHECK(h, dtype == DSMP_F32 || dtype == DSMP_BF16, DSMP_INVALID_ARG, "unknown dtype");
  DSMP_CHECK(h, n >= 0 && C >= 1, DSMP_INVALID_ARG, "negative rows or no channel");
  DSMP_CHECK(h, n < (int64_t)1 << 31, DSMP_UNSUPPORTED, "2^31 rows and more");
  DSMP_CHECK(h, C <= MAX_C, DSMP_UNSUPPORTED, "more than %d channels", MAX_C);
  DSMP_CHECK(h, n == 0 || (ck && ck->q && ck->scale && p), DSMP_INVALID_ARG, "a data pointer is NULL");
  return check_ld(h, C, {ld});
}

}  // namespace

extern "C" dsmp_status dsmp_checkpoint_store(dsmp_handle* h, const void* x, int32_t dtype, int64_t ldx, int64_t n,
                                             int32_t channels, const dsmp_checkpoint* ck) {
  if (!h) return DSMP_INVALID_ARG;
  const dsmp_status st = check_ckpt(h, ck, x, dtype, ldx, n, channels);
  if (st != DSMP_OK || n == 0) return st;
  NormArgs a{};
  a.n = n, a.C = channels;
  a.x = x, a.ldx = ldx, a.q = ck->q, a.scale = ck->scale;
  const bool vec = channels % 4 == 0 && channels <= MAX_C / 2 && aligned(x, ldx, size_of(dtype)) && aligned(ck->q, channels, 1);
  place(a, vec);
  ProfScope prof(h, DSMP_K_CKPT);
  by_type(dtype, [&](auto t) {
    by_bool(vec, [&](auto v) { DSMP_GO((k_ckpt_store<decltype(t), decltype(v)::value>), row_grid(h, a, 16), RNT, 0); });
  });
  DSMP_LAUNCHED(h, "checkpoint store");
  return DSMP_OK;
}

extern "C" dsmp_status dsmp_checkpoint_load(dsmp_handle* h, const dsmp_checkpoint* ck, int64_t n, int32_t channels,
                                            void* y, int32_t dtype, int64_t ldy) {
  if (!h) return DSMP_INVALID_ARG;
  const dsmp_status st = check_ckpt(h, ck, y, dtype, ldy, n, channels);
  if (st != DSMP_OK || n == 0) return st;
  NormArgs a{};
  a.n = n, a.C = channels;
  a.x = ck->q, a.xscale = ck->scale, a.y = y, a.ldy = ldy, a.y_bf16 = dtype == DSMP_BF16;
  const bool vec = channels % 4 == 0 && channels <= MAX_C / 2 && aligned(y, ldy, size_of(dtype)) && aligned(ck->q, channels, 1);
  place(a, vec);
  ProfScope prof(h, DSMP_K_CKPT);
  by_bool(vec, [&](auto v) { DSMP_GO((k_ckpt_load<decltype(v)::value>), row_grid(h, a, 16), RNT, 0); });
  DSMP_LAUNCHED(h, "checkpoint load");
  return DSMP_OK;
}
