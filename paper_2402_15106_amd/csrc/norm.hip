// Group norm with an activation over packed segments (channels last), forward,
// restored and backward, and activation checkpoints in 8 bits.
//
// All of it is bound by memory: about 10 operations per value forward and 30
// backward, against 4 to 16 bytes.  A segment's statistics need all its rows
// before any of them can be written, so the long form is two passes: one that
// sums over chunks of rows (and adds the addend and writes the checkpoint on
// the way), one that joins the chunks' sums and writes the result.  The second
// reads what the first just touched.  Where each row is a segment, one pass.
//
// Every lane holds 8 consecutive channels of a row: 16 bytes of bfloat16, 32 of
// float32, 8 of a checkpoint.  A row takes `lpr` lanes, the next power of two,
// so sums over the rows of a wave are shuffles by lpr, 2 lpr, ..., and a
// checkpoint's block of 64 channels is 8 neighbouring lanes.
//
// Sums run in a fixed order (lane, wave, chunk): no atomics, the same bits on
// every run.  What crosses a chunk is joined in float64.
#include <algorithm>
#include <cmath>

#include "common.hpp"

using namespace dsmp;

namespace {

constexpr int MAX_C = 512;      // 64 lanes of 8 channels: a row stays in one wave
constexpr int BLOCK_C = 64;     // channels that share a checkpoint scale
constexpr int NT = 512;         // threads of the passes over segments
constexpr int NW = NT / 64;
constexpr int RNT = 256;        // threads where each row is a segment, and of the checkpoint passes
constexpr int MAX_CHUNKS = 512; // chunks of rows that sums are split over
constexpr float TINY = 0x1p-100f;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Rows a lane has in flight in the forward passes, and in the backward ones,
// which hold twice the values of each (rows that are not whole aligned groups:
// one and the same, their loads have branches).
template <bool VEC>
constexpr int FWD_TILE = VEC ? 4 : 2;
template <bool VEC>
constexpr int BWD_TILE = VEC ? 2 : 1;

struct Q8 {};   // tag: a checkpoint as the source of values

struct NormArgs {
  int64_t n;
  int C, G, gs, lg;             // lg: log2 of the lanes of a row
  int n_seg;
  int64_t len;                  // rows of a segment where ptr is null
  const int32_t* ptr;
  int64_t R;                    // rows of a chunk of the summing pass
  int64_t RA;                   // rows of a workgroup of the second pass
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
  int act, merge;
  const float* gy;
  int64_t ldgy;
  const float* ga;
  int64_t ldga;
  float* gx;
  int64_t ldgx;
  float* part_c;                // [chunk][2][C]: chunk sums of w and w xn
  float *dgamma, *dbeta;
  int accumulate, nchunks, nred;
};

// ------------------------------------------------------------ eight channels

// cnt: channels of this lane that exist (8, fewer in a last lane, none past it).
// VEC: rows are whole aligned groups of 8; a lane past the row reads the
// row's first group and drops it (a load under a condition would make the
// compiler wait for everything in flight).
template <bool VEC>
__device__ __forceinline__ void words4(const void* p, uint32_t (&w)[4]) {
  if (VEC) {
    const uint4 u = *static_cast<const uint4*>(p);
    w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
  } else {
    __builtin_memcpy(w, p, 16);   // one load of any alignment
  }
}

template <typename T, bool VEC>
struct Row;

template <bool VEC>
struct Row<float, VEC> {
  static __device__ __forceinline__ void load(const float* row, int c0, int cnt, float (&v)[8]) {
    if (VEC || cnt == 8) {
      const float* p = row + (cnt > 0 ? c0 : 0);
      uint32_t w[4], u[4];
      words4<VEC>(p, w);
      words4<VEC>(p + 4, u);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[k] = cnt > 0 ? __builtin_bit_cast(float, w[k]) : 0.0f;
        v[4 + k] = cnt > 0 ? __builtin_bit_cast(float, u[k]) : 0.0f;
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = k < cnt ? row[c0 + k] : 0.0f;
    }
  }
  static __device__ __forceinline__ void store(float* row, int c0, int cnt, const float (&v)[8]) {
    if (VEC || cnt == 8) {
      if (cnt <= 0) return;
      float* p = row + c0;
      if (VEC) {
        reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
      } else {
        __builtin_memcpy(p, &v[0], 16);
        __builtin_memcpy(p + 4, &v[4], 16);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < cnt) row[c0 + k] = v[k];
    }
  }
};

template <bool VEC>
struct Row<__bf16, VEC> {
  static __device__ __forceinline__ void load(const __bf16* row, int c0, int cnt, float (&v)[8]) {
    if (VEC || cnt == 8) {
      uint32_t w[4];
      const __bf16* p = row + (cnt > 0 ? c0 : 0);
      words4<VEC>(p, w);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[2 * k] = cnt > 0 ? __builtin_bit_cast(float, w[k] << 16) : 0.0f;
        v[2 * k + 1] = cnt > 0 ? __builtin_bit_cast(float, w[k] & 0xffff0000u) : 0.0f;
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = k < cnt ? (float)row[c0 + k] : 0.0f;
    }
  }
  static __device__ __forceinline__ void store(__bf16* row, int c0, int cnt, const float (&v)[8]) {
    if (VEC || cnt == 8) {
      if (cnt <= 0) return;
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        w[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){v[2 * k], v[2 * k + 1]}, bf16x2));
      __bf16* p = row + c0;
      if (VEC)
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
      else
        __builtin_memcpy(p, w, 16);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < cnt) row[c0 + k] = (__bf16)v[k];
    }
  }
};

// The eight bytes of a checkpoint row, times their block's scale.
template <bool VEC>
__device__ __forceinline__ void load_q8(const int8_t* row, const float* scale_row, int c0, int cnt, float (&v)[8]) {
  const int at = cnt > 0 ? c0 : 0;
  const float s = scale_row[at / BLOCK_C];
  if (VEC || cnt == 8) {
    uint32_t w[2];
    if (VEC) {
      const uint2 u = *reinterpret_cast<const uint2*>(row + at);
      w[0] = u.x, w[1] = u.y;
    } else {
      __builtin_memcpy(w, row + at, 8);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int32_t b = (int32_t)(w[k / 4] << (24 - 8 * (k % 4))) >> 24;
      v[k] = cnt > 0 ? (float)b * s : 0.0f;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < cnt ? (float)row[c0 + k] * s : 0.0f;
  }
}

// Row r of the source, whatever it is.
template <typename T, bool VEC>
struct Source {
  static __device__ __forceinline__ void load(const NormArgs& a, int64_t r, int c0, int cnt, float (&v)[8]) {
    Row<T, VEC>::load(static_cast<const T*>(a.x) + r * a.ldx, c0, cnt, v);
  }
};
template <bool VEC>
struct Source<Q8, VEC> {
  static __device__ __forceinline__ void load(const NormArgs& a, int64_t r, int c0, int cnt, float (&v)[8]) {
    load_q8<VEC>(static_cast<const int8_t*>(a.x) + r * a.C, a.xscale + r * ((a.C + BLOCK_C - 1) / BLOCK_C), c0, cnt,
                 v);
  }
};

// Quantises a lane's eight values of a block of 64 channels (8 lanes; `width`
// of them where the row has fewer) and writes them and the block's scale.  The
// largest magnitude is found on the bits without the sign, which order as the
// values do and put a NaN above everything.
template <bool VEC>
__device__ __forceinline__ void store_q8(int8_t* q, float* scale, int64_t r, int C, int c0, int cnt, int width,
                                         const float (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) m = max(m, __builtin_bit_cast(uint32_t, v[k]) & 0x7fffffffu);
  for (int o = 1; o < width; o <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
  const float big = __builtin_bit_cast(float, m);
  const bool some = m >= __builtin_bit_cast(uint32_t, TINY), odd = m >= 0x7f800000u;
  const float inv = some && !odd ? 127.0f / big : 0.0f;
  const float s = odd ? __builtin_bit_cast(float, 0x7fc00000u) : some ? big * (1.0f / 127.0f) : 0.0f;
  if (cnt <= 0) return;
  int b[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float t = odd ? 0.0f : __builtin_rintf(v[k] * inv);
    b[k] = (int)fminf(fmaxf(t, -127.0f), 127.0f);
  }
  int8_t* p = q + r * C + c0;
  if (VEC || cnt == 8) {
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      w[i] = (b[4 * i] & 255) | (b[4 * i + 1] & 255) << 8 | (b[4 * i + 2] & 255) << 16 | (uint32_t)b[4 * i + 3] << 24;
    if (VEC)
      *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else
      __builtin_memcpy(p, w, 8);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < cnt) p[k] = (int8_t)b[k];
  }
  if (c0 % BLOCK_C == 0) scale[r * ((C + BLOCK_C - 1) / BLOCK_C) + c0 / BLOCK_C] = s;
}

// t = x (+ addend, rounded to T and written to sum); its checkpoint.
template <typename T, bool VEC, bool ADD>
__device__ __forceinline__ void take_row(const NormArgs& a, int64_t r, int c0, int cnt, float (&v)[8]) {
  Source<T, VEC>::load(a, r, c0, cnt, v);
  if (ADD) {
    float u[8];
    Row<T, VEC>::load(static_cast<const T*>(a.add) + r * a.lda, c0, cnt, u);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = (float)(T)(v[k] + u[k]);
  }
}

// ------------------------------------------------------------ activations

// Upper tail of the normal distribution at |z| and exp(-z^2/2): Abramowitz and
// Stegun 7.1.26 (a polynomial in 1 / (1 + p x) times exp(-x^2), x = |z| / sqrt 2,
// within 1.5e-7 of erf), on the side where nothing cancels, so the small values
// of GELU at negative z keep their digits.
__device__ __forceinline__ float normal_tail(float z, float& e) {
  const float x = __builtin_fabsf(z) * 0.70710678f;
  e = __expf(-0.5f * z * z);
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f, x, 1.0f));
  float p = __builtin_fmaf(1.061405429f, t, -1.453152027f);
  p = __builtin_fmaf(p, t, 1.421413741f);
  p = __builtin_fmaf(p, t, -0.284496736f);
  p = __builtin_fmaf(p, t, 0.254829592f);
  return 0.5f * p * t * e;
}

__device__ __forceinline__ void activate8(int act, float (&z)[8]) {
  if (act == DSMP_ACT_SILU) {
#pragma unroll
    for (int k = 0; k < 8; ++k) z[k] *= __builtin_amdgcn_rcpf(1.0f + __expf(-z[k]));
  } else if (act == DSMP_ACT_GELU) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float e;
      const float q = normal_tail(z[k], e);
      z[k] *= z[k] < 0.0f ? q : 1.0f - q;
    }
  } else if (act == DSMP_ACT_RELU) {
#pragma unroll
    for (int k = 0; k < 8; ++k) z[k] = z[k] < 0.0f ? 0.0f : z[k];   // a NaN passes
  }
}

// w *= act'(z)
__device__ __forceinline__ void slope8(int act, const float (&z)[8], float (&w)[8]) {
  if (act == DSMP_ACT_SILU) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float p = __builtin_amdgcn_rcpf(1.0f + __expf(-z[k]));
      w[k] *= p * __builtin_fmaf(z[k], 1.0f - p, 1.0f);
    }
  } else if (act == DSMP_ACT_GELU) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float e;
      const float q = normal_tail(z[k], e);
      w[k] *= __builtin_fmaf(z[k] * 0.39894228f, e, z[k] < 0.0f ? q : 1.0f - q);
    }
  } else if (act == DSMP_ACT_RELU) {
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = z[k] > 0.0f ? w[k] : z[k] <= 0.0f ? 0.0f : z[k];
  }
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
// The last segment that begins at or before row r.
__device__ __forceinline__ int seg_find(const NormArgs& a, int64_t r) {
  if (!a.ptr) return a.len > 0 ? (int)std::min<int64_t>(r / a.len, a.n_seg - 1) : 0;
  int lo = 0, hi = a.n_seg - 1;
  while (lo < hi) {
    const int mid = lo + (hi - lo + 1) / 2;
    if (seg_begin(a, mid) <= r)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

struct Lanes {
  int lpr, lr, rl, RL, c0, cnt;
  __device__ __forceinline__ Lanes(int lg, int C, int threads) {
    lpr = 1 << lg;
    lr = threadIdx.x & (lpr - 1);
    rl = threadIdx.x >> lg;
    RL = threads >> lg;
    c0 = lr * 8;
    cnt = std::min(8, C - c0);
  }
};

// s1, s2: the workgroup's sums per channel (float64 in LDS).  Writes the sums
// over each group's channels to out(g, sum1, sum2), by one lane each.
template <typename F>
__device__ __forceinline__ void group_sums(const double* s1, const double* s2, int G, int gs, F out) {
  int tg = 1;   // lanes of a group
  while (tg < 64 && tg * 2 * G <= NT && tg < gs) tg <<= 1;
  const int per = NT / tg;
  for (int gb = 0; gb < G; gb += per) {
    const int g = gb + (int)threadIdx.x / tg, l = threadIdx.x % tg;
    double u = 0.0, v = 0.0;
    if (g < G)
      for (int i = l; i < gs; i += tg) u += s1[g * gs + i], v += s2[g * gs + i];
    for (int o = 1; o < tg; o <<= 1) u += __shfl_xor(u, o, 64), v += __shfl_xor(v, o, 64);
    if (g < G && l == 0) out(g, u, v);
  }
}

// ------------------------------------------------------------ forward, first pass

// Count, mean and sum of squares about the mean of eight channels.  Rows join
// TILE at a time (mean of the tile, then deviations from it, then the pair rule
// of Chan, Golub and LeVeque), so a large mean or a far-out row costs no digits.
struct Moments {
  float n = 0.0f, mean[8] = {}, m2[8] = {};

  template <int N>
  __device__ __forceinline__ void add(const float (&v)[N][8]) {
    const float nn = n + N, w = N / nn, f = n * w;
    n = nn;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float s = v[0][k];
#pragma unroll
      for (int t = 1; t < N; ++t) s += v[t][k];
      const float m = s * (1.0f / N);
      float q = 0.0f;
#pragma unroll
      for (int t = 0; t < N; ++t) q = __builtin_fmaf(v[t][k] - m, v[t][k] - m, q);
      const float d = m - mean[k];
      mean[k] = __builtin_fmaf(d, w, mean[k]);
      m2[k] += __builtin_fmaf(d * d, f, q);
    }
  }
  // joins the lane `o` away
  __device__ __forceinline__ void join(int o) {
    const float nb = __shfl_xor(n, o, 64), nn = n + nb, w = nn > 0.0f ? nb / nn : 0.0f, f = n * w;
    n = nn;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float mb = __shfl_xor(mean[k], o, 64), qb = __shfl_xor(m2[k], o, 64), d = mb - mean[k];
      mean[k] = __builtin_fmaf(d, w, mean[k]);
      m2[k] += __builtin_fmaf(d * d, f, qb);
    }
  }
};

size_t stats_lds(int lg, int C) { return (size_t)NW * (16 << lg) * 4 + NW * 4 + 8 + 16 * (size_t)C; }

template <typename T, bool VEC, bool ADD, bool CK>
__global__ __launch_bounds__(NT) void k_norm_stats(NormArgs a) {
  extern __shared__ double sh[];
  const Lanes L(a.lg, a.C, NT);
  const int wid = threadIdx.x >> 6, lane = threadIdx.x & 63, w8 = L.lpr * 8;
  double *s1 = sh, *s2 = sh + a.C;
  float *mm = reinterpret_cast<float*>(s2 + a.C), *qq = mm + NW * w8, *nn = qq + NW * w8;
  const int64_t r0 = (int64_t)blockIdx.x * a.R, r1 = std::min<int64_t>(r0 + a.R, a.n);
  int s = seg_find(a, r0);
  for (int64_t r = r0; r < r1; ++s) {
    const int64_t e = std::min<int64_t>(seg_end(a, s), r1);
    if (e <= r) continue;
    Moments m;
    constexpr int TILE = FWD_TILE<VEC>;
    int64_t i = r + L.rl;
    auto take = [&](int64_t row, float(&v)[8]) {
      take_row<T, VEC, ADD>(a, row, L.c0, L.cnt, v);
    };
    auto keep = [&](int64_t row, const float(&v)[8]) {
      if (ADD) Row<T, VEC>::store(static_cast<T*>(a.sum) + row * a.lds, L.c0, L.cnt, v);
      if (CK) store_q8<VEC>(a.q, a.scale, row, a.C, L.c0, L.cnt, std::min(8, L.lpr), v);
    };
    for (; i + (TILE - 1) * L.RL < e; i += TILE * L.RL) {
      float v[TILE][8];
#pragma unroll
      for (int t = 0; t < TILE; ++t) take(i + t * L.RL, v[t]);
#pragma unroll
      for (int t = 0; t < TILE; ++t) keep(i + t * L.RL, v[t]);
      m.add<TILE>(v);
    }
    for (; i < e; i += L.RL) {
      float v[1][8];
      take(i, v[0]);
      keep(i, v[0]);
      m.add<1>(v);
    }
    for (int o = L.lpr; o < 64; o <<= 1) m.join(o);
    if (lane < L.lpr) {
#pragma unroll
      for (int k = 0; k < 8; ++k) mm[wid * w8 + L.c0 + k] = m.mean[k], qq[wid * w8 + L.c0 + k] = m.m2[k];
      if (lane == 0) nn[wid] = m.n;
    }
    __syncthreads();
    // per channel: sum n_w mean_w, and the squares about zero, in float64
    const int c = threadIdx.x;
    if (c < a.C) {
      double u = 0.0, v = 0.0;
      for (int w = 0; w < NW; ++w) {
        const double mw = mm[w * w8 + c], nw = nn[w];
        u += nw * mw;
        v += (double)qq[w * w8 + c] + nw * mw * mw;
      }
      s1[c] = u;
      s2[c] = v;
    }
    __syncthreads();
    const double count = (double)(e - r) * a.gs;
    float2* part = a.part + ((int64_t)blockIdx.x + s) * a.G;
    group_sums(s1, s2, a.G, a.gs, [&](int g, double u, double v) {
      const double mean = u / count;
      part[g] = make_float2((float)mean, (float)fmax(v - u * mean, 0.0));
    });
    __syncthreads();
    r = e;
  }
}

// ------------------------------------------------------------ joining the pieces

// Sums over the pieces of segment s (rows [b, e)) for every group: term(piece
// value, rows of the piece, u, v) adds to two float64 sums; done(g, u, v) is called
// by one lane of each group.  Consecutive lanes take consecutive groups.
template <typename TERM, typename DONE>
__device__ __forceinline__ void join_pieces(const NormArgs& a, int s, int64_t b, int64_t e, double* sh, TERM term,
                                            DONE done) {
  int gp = 1;
  while (gp < a.G) gp <<= 1;
  const int g = threadIdx.x & (gp - 1), p = threadIdx.x / gp, P = NT / gp;
  const int64_t j0 = b / a.R, j1 = (e - 1) / a.R;
  double u = 0.0, v = 0.0;
  if (g < a.G) {
#pragma unroll 4
    for (int64_t j = j0 + p; j <= j1; j += P) {
      const float2 t = a.part[(j + s) * a.G + g];
      const int64_t rows = std::min<int64_t>(e, (j + 1) * a.R) - std::max<int64_t>(b, j * a.R);
      term(t, (double)rows, u, v);
    }
  }
  for (int o = gp; o < 64; o <<= 1) u += __shfl_xor(u, o, 64), v += __shfl_xor(v, o, 64);
  if (gp >= 64) {
    // one row of P sums per group
    sh[threadIdx.x] = u;
    sh[NT + threadIdx.x] = v;
    __syncthreads();
    if (p == 0 && g < a.G) {
      for (int i = 1; i < P; ++i) u += sh[i * gp + g], v += sh[NT + i * gp + g];
      done(g, u, v);
    }
  } else {
    const int wid = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (lane < gp) sh[wid * 64 + lane] = u, sh[NT + wid * 64 + lane] = v;
    __syncthreads();
    if (threadIdx.x < (unsigned)gp && g < a.G) {
      for (int w = 1; w < NW; ++w) u += sh[w * 64 + g], v += sh[NT + w * 64 + g];
      done(g, u, v);
    }
  }
  __syncthreads();
}

// ------------------------------------------------------------ forward, second pass

// mean and rstd of eight channels' groups
__device__ __forceinline__ void spread(const float* st, const NormArgs& a, int c0, float (&mean)[8], float (&rstd)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int g = std::min(c0 + k, a.C - 1) / a.gs;
    mean[k] = st[2 * g];
    rstd[k] = st[2 * g + 1];
  }
}

__device__ __forceinline__ void params8(const NormArgs& a, int c0, float (&gamma)[8], float (&beta)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int c = std::min(c0 + k, a.C - 1);
    gamma[k] = a.gamma ? a.gamma[c] : 1.0f;
    beta[k] = a.gamma ? a.beta[c] : 0.0f;
  }
}

// y = act((t - mean) * (rstd gamma) + beta) on this workgroup's rows, segment by
// segment.  a.merge: the statistics come from the first pass's pieces (and are
// written, by the workgroup that has the segment's first row), else from a.stats.
template <typename T, typename Y, bool VEC>
__global__ __launch_bounds__(NT) void k_norm_apply(NormArgs a) {
  __shared__ double sh[2 * NT];
  __shared__ float st[2 * MAX_C];
  const Lanes L(a.lg, a.C, NT);
  const int64_t r0 = (int64_t)blockIdx.x * a.RA, r1 = std::min<int64_t>(r0 + a.RA, a.n);
  if (a.merge && blockIdx.x == 0) {
    for (int s = threadIdx.x; s < a.n_seg; s += NT)
      if (seg_end(a, s) <= seg_begin(a, s))
        for (int g = 0; g < 2 * a.G; ++g) a.stats[(int64_t)s * 2 * a.G + g] = 0.0f;
  }
  if (r0 >= r1) return;
  float gamma[8], beta[8];
  params8(a, L.c0, gamma, beta);
  int s = seg_find(a, r0);
  for (int64_t r = r0; r < r1; ++s) {
    const int64_t b = seg_begin(a, s), e = seg_end(a, s), end = std::min<int64_t>(e, r1);
    if (end <= r) continue;
    float mean[8], scale[8];
    if (a.merge) {
      const double count = (double)(e - b) * a.gs;
      join_pieces(
          a, s, b, e, sh,
          [&](float2 t, double rows, double& u, double& v) {
            const double m = t.x, k = rows * a.gs;
            u += k * m;
            v += (double)t.y + k * m * m;
          },
          [&](int g, double u, double v) {
            const double m = u / count;
            st[2 * g] = (float)m;
            st[2 * g + 1] = (float)(1.0 / sqrt(fmax(v / count - m * m, 0.0) + (double)a.eps));
          });
      if (b >= r0)
        for (int g = threadIdx.x; g < 2 * a.G; g += NT) a.stats[(int64_t)s * 2 * a.G + g] = st[g];
      spread(st, a, L.c0, mean, scale);
    } else {
      spread(a.stats + (int64_t)s * 2 * a.G, a, L.c0, mean, scale);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) scale[k] *= gamma[k];
    auto put = [&](int64_t row, float(&v)[8]) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = __builtin_fmaf(v[k] - mean[k], scale[k], beta[k]);
      activate8(a.act, v);
      Row<Y, VEC>::store(static_cast<Y*>(a.y) + row * a.ldy, L.c0, L.cnt, v);
    };
    constexpr int TILE = FWD_TILE<VEC>;
    int64_t i = r + L.rl;
    for (; i + (TILE - 1) * L.RL < end; i += TILE * L.RL) {
      float v[TILE][8];
#pragma unroll
      for (int t = 0; t < TILE; ++t) Source<T, VEC>::load(a, i + t * L.RL, L.c0, L.cnt, v[t]);
#pragma unroll
      for (int t = 0; t < TILE; ++t) put(i + t * L.RL, v[t]);
    }
    for (; i < end; i += L.RL) {
      float v[8];
      Source<T, VEC>::load(a, i, L.c0, L.cnt, v);
      put(i, v);
    }
    r = end;
  }
}

// ------------------------------------------------------------ backward

// Of one row's eight channels: w = grad_y act'(z) and xn.
template <typename T, bool VEC>
__device__ __forceinline__ void weigh(const NormArgs& a, const float (&t)[8], const float (&mean)[8],
                                      const float (&rstd)[8], const float (&gamma)[8], const float (&beta)[8],
                                      float (&w)[8], float (&xn)[8]) {
  float z[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    xn[k] = (t[k] - mean[k]) * rstd[k];
    z[k] = __builtin_fmaf(xn[k], gamma[k], beta[k]);
  }
  slope8(a.act, z, w);
}

// First pass: per chunk and segment the groups' sums of gamma w and gamma w xn,
// per chunk the channels' sums of w and w xn.
template <typename T, bool VEC>
__global__ __launch_bounds__(NT) void k_norm_bwd_sums(NormArgs a) {
  extern __shared__ double sh[];
  const Lanes L(a.lg, a.C, NT);
  const int wid = threadIdx.x >> 6, lane = threadIdx.x & 63, w8 = L.lpr * 8, c = threadIdx.x;
  double *s1 = sh, *s2 = sh + a.C;
  float *uu = reinterpret_cast<float*>(s2 + a.C), *vv = uu + NW * w8;
  const int64_t r0 = (int64_t)blockIdx.x * a.R, r1 = std::min<int64_t>(r0 + a.R, a.n);
  float gamma[8], beta[8];
  params8(a, L.c0, gamma, beta);
  const double gc = c < a.C && a.gamma ? a.gamma[c] : 1.0;
  double cu = 0.0, cv = 0.0;
  int s = seg_find(a, r0);
  for (int64_t r = r0; r < r1; ++s) {
    const int64_t e = std::min<int64_t>(seg_end(a, s), r1);
    if (e <= r) continue;
    float mean[8], rstd[8], u[8] = {}, v[8] = {};
    spread(a.stats + (int64_t)s * 2 * a.G, a, L.c0, mean, rstd);
    auto add = [&](const float(&t)[8], float(&w)[8]) {
      float xn[8];
      weigh<T, VEC>(a, t, mean, rstd, gamma, beta, w, xn);
#pragma unroll
      for (int k = 0; k < 8; ++k) u[k] += w[k], v[k] = __builtin_fmaf(w[k], xn[k], v[k]);
    };
    constexpr int TILE = BWD_TILE<VEC>;
    int64_t i = r + L.rl;
    for (; i + (TILE - 1) * L.RL < e; i += TILE * L.RL) {
      float t[TILE][8], w[TILE][8];
#pragma unroll
      for (int j = 0; j < TILE; ++j) {
        Source<T, VEC>::load(a, i + j * L.RL, L.c0, L.cnt, t[j]);
        Row<float, VEC>::load(a.gy + (i + j * L.RL) * a.ldgy, L.c0, L.cnt, w[j]);
      }
#pragma unroll
      for (int j = 0; j < TILE; ++j) add(t[j], w[j]);
    }
    for (; i < e; i += L.RL) {
      float t[8], w[8];
      Source<T, VEC>::load(a, i, L.c0, L.cnt, t);
      Row<float, VEC>::load(a.gy + i * a.ldgy, L.c0, L.cnt, w);
      add(t, w);
    }
    for (int o = L.lpr; o < 64; o <<= 1) {
#pragma unroll
      for (int k = 0; k < 8; ++k) u[k] += __shfl_xor(u[k], o, 64), v[k] += __shfl_xor(v[k], o, 64);
    }
    if (lane < L.lpr) {
#pragma unroll
      for (int k = 0; k < 8; ++k) uu[wid * w8 + L.c0 + k] = u[k], vv[wid * w8 + L.c0 + k] = v[k];
    }
    __syncthreads();
    if (c < a.C) {
      double x = 0.0, y = 0.0;
      for (int w = 0; w < NW; ++w) x += uu[w * w8 + c], y += vv[w * w8 + c];
      cu += x, cv += y;
      s1[c] = gc * x;
      s2[c] = gc * y;
    }
    __syncthreads();
    float2* part = a.part + ((int64_t)blockIdx.x + s) * a.G;
    group_sums(s1, s2, a.G, a.gs, [&](int g, double x, double y) { part[g] = make_float2((float)x, (float)y); });
    __syncthreads();
    r = e;
  }
  if (a.part_c && c < a.C) {
    a.part_c[(int64_t)blockIdx.x * 2 * a.C + c] = (float)cu;
    a.part_c[(int64_t)blockIdx.x * 2 * a.C + a.C + c] = (float)cv;
  }
}

// dbeta and dgamma from the chunks' sums: 64 columns of part_c to a workgroup of
// `threads`, the chunks dealt to its waves, joined in wave order.
__device__ __forceinline__ void columns(const NormArgs& a, int block, double* sh, int waves) {
  const int col = block * 64 + (threadIdx.x & 63), wid = threadIdx.x >> 6;
  double v = 0.0;
  if (col < 2 * a.C) {
#pragma unroll 8
    for (int j = wid; j < a.nchunks; j += waves) v += a.part_c[(int64_t)j * 2 * a.C + col];
  }
  sh[threadIdx.x] = v;
  __syncthreads();
  if (wid == 0 && col < 2 * a.C) {
    for (int w = 1; w < waves; ++w) v += sh[w * 64 + threadIdx.x];
    float* p = col < a.C ? a.dbeta + col : a.dgamma + (col - a.C);
    *p = a.accumulate ? *p + (float)v : (float)v;
  }
}

// grad_x of one row from its groups' sums
__device__ __forceinline__ void grad8(const float (&rstd)[8], const float (&gamma)[8], const float (&A)[8],
                                      const float (&B)[8], const float (&w)[8], const float (&xn)[8], float (&g)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k)
    g[k] = __builtin_fmaf(rstd[k], __builtin_fmaf(-xn[k], B[k], __builtin_fmaf(gamma[k], w[k], -A[k])), g[k]);
}

// Second pass.  The first a.nred workgroups form dbeta and dgamma.
template <typename T, bool VEC>
__global__ __launch_bounds__(NT) void k_norm_bwd_dx(NormArgs a) {
  __shared__ double sh[2 * NT];
  __shared__ float st[2 * MAX_C];
  if ((int)blockIdx.x < a.nred) {
    columns(a, blockIdx.x, sh, NW);
    return;
  }
  const Lanes L(a.lg, a.C, NT);
  const int64_t r0 = (int64_t)(blockIdx.x - a.nred) * a.RA, r1 = std::min<int64_t>(r0 + a.RA, a.n);
  if (r0 >= r1) return;
  float gamma[8], beta[8];
  params8(a, L.c0, gamma, beta);
  int s = seg_find(a, r0);
  for (int64_t r = r0; r < r1; ++s) {
    const int64_t b = seg_begin(a, s), e = seg_end(a, s), end = std::min<int64_t>(e, r1);
    if (end <= r) continue;
    const double count = (double)(e - b) * a.gs;
    join_pieces(
        a, s, b, e, sh, [&](float2 t, double, double& u, double& v) { u += t.x, v += t.y; },
        [&](int g, double u, double v) { st[2 * g] = (float)(u / count), st[2 * g + 1] = (float)(v / count); });
    float mean[8], rstd[8], A[8], B[8];
    spread(st, a, L.c0, A, B);
    spread(a.stats + (int64_t)s * 2 * a.G, a, L.c0, mean, rstd);
    auto put = [&](int64_t row, const float(&t)[8], float(&w)[8], float(&g)[8]) {
      float xn[8];
      weigh<T, VEC>(a, t, mean, rstd, gamma, beta, w, xn);
      grad8(rstd, gamma, A, B, w, xn, g);
      Row<float, VEC>::store(a.gx + row * a.ldgx, L.c0, L.cnt, g);
    };
    constexpr int TD = BWD_TILE<VEC>;
    int64_t i = r + L.rl;
    for (; i + (TD - 1) * L.RL < end; i += TD * L.RL) {
      float t[TD][8], w[TD][8], g[TD][8] = {};
#pragma unroll
      for (int j = 0; j < TD; ++j) {
        const int64_t row = i + j * L.RL;
        Source<T, VEC>::load(a, row, L.c0, L.cnt, t[j]);
        Row<float, VEC>::load(a.gy + row * a.ldgy, L.c0, L.cnt, w[j]);
        if (a.ga) Row<float, VEC>::load(a.ga + row * a.ldga, L.c0, L.cnt, g[j]);
      }
#pragma unroll
      for (int j = 0; j < TD; ++j) put(i + j * L.RL, t[j], w[j], g[j]);
    }
    for (; i < end; i += L.RL) {
      float t[8], w[8], g[8] = {};
      Source<T, VEC>::load(a, i, L.c0, L.cnt, t);
      Row<float, VEC>::load(a.gy + i * a.ldgy, L.c0, L.cnt, w);
      if (a.ga) Row<float, VEC>::load(a.ga + i * a.ldga, L.c0, L.cnt, g);
      put(i, t, w, g);
    }
    r = end;
  }
}

// dbeta and dgamma alone (rows as segments, no rows at all)
__global__ __launch_bounds__(RNT) void k_norm_columns(NormArgs a) {
  __shared__ double sh[RNT];
  columns(a, blockIdx.x, sh, RNT / 64);
}

// ------------------------------------------------------------ each row a segment

// Sums over the groups of a row: p[k] becomes the sum over the group of channel
// c0 + k.  width: the lanes of a group where it is whole lanes and a power of two
// of them (or the whole row); 0: any other group, through the wave's LDS.
struct RowGroups {
  int width;
  int at[8];     // first channel of each channel's group
  float* lds;    // the wave's 512 floats

  __device__ __forceinline__ RowGroups(const NormArgs& a, const Lanes& L, float* wave_lds) : lds(wave_lds) {
    const int lg = a.gs / 8;
    width = a.G == 1 ? L.lpr : (a.gs % 8 == 0 && (lg & (lg - 1)) == 0) ? lg : 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) at[k] = std::min(L.c0 + k, a.C - 1) / a.gs * a.gs;
  }
  __device__ __forceinline__ void sum(const NormArgs& a, const Lanes& L, float (&p)[8]) const {
    if (width) {
      float s = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      for (int o = 1; o < width; o <<= 1) s += __shfl_xor(s, o, 64);
#pragma unroll
      for (int k = 0; k < 8; ++k) p[k] = s;
      return;
    }
    float* row = lds + ((threadIdx.x & 63) - L.lr) * 8;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int k = 0; k < 8; ++k) row[L.c0 + k] = p[k];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float s = 0.0f;
      for (int i = 0; i < a.gs; ++i) s += row[at[k] + i];
      p[k] = s;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  // mean and rstd of a row's groups
  __device__ __forceinline__ void read(const NormArgs& a, const float* st, float (&mean)[8], float (&rstd)[8]) const {
    if (width) {
      const float2 t = reinterpret_cast<const float2*>(st)[at[0] / a.gs];
#pragma unroll
      for (int k = 0; k < 8; ++k) mean[k] = t.x, rstd[k] = t.y;
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) mean[k] = st[2 * (at[k] / a.gs)], rstd[k] = st[2 * (at[k] / a.gs) + 1];
    }
  }
};

template <typename T, typename Y, bool VEC, bool ADD, bool CK>
__global__ __launch_bounds__(RNT) void k_norm_rows(NormArgs a) {
  __shared__ float lds[RNT * 8];
  const Lanes L(a.lg, a.C, RNT);
  const RowGroups R(a, L, lds + (threadIdx.x >> 6) * 512);
  float gamma[8], beta[8];
  params8(a, L.c0, gamma, beta);
  const float f = 1.0f / a.gs;
  for (int64_t i = (int64_t)blockIdx.x * L.RL + L.rl; i < a.n; i += (int64_t)gridDim.x * L.RL) {
    float v[8], m[8], q[8];
    take_row<T, VEC, ADD>(a, i, L.c0, L.cnt, v);
    if (ADD) Row<T, VEC>::store(static_cast<T*>(a.sum) + i * a.lds, L.c0, L.cnt, v);
    if (CK) store_q8<VEC>(a.q, a.scale, i, a.C, L.c0, L.cnt, std::min(8, L.lpr), v);
#pragma unroll
    for (int k = 0; k < 8; ++k) m[k] = v[k];
    R.sum(a, L, m);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      m[k] *= f;
      const float d = k < L.cnt ? v[k] - m[k] : 0.0f;
      q[k] = d * d;
    }
    R.sum(a, L, q);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      q[k] = 1.0f / sqrtf(__builtin_fmaf(q[k], f, a.eps));
      if (k < L.cnt && L.c0 + k == R.at[k]) {
        const int64_t g = i * a.G + R.at[k] / a.gs;
        reinterpret_cast<float2*>(a.stats)[g] = make_float2(m[k], q[k]);
      }
      v[k] = __builtin_fmaf((v[k] - m[k]) * q[k], gamma[k], beta[k]);
    }
    activate8(a.act, v);
    Row<Y, VEC>::store(static_cast<Y*>(a.y) + i * a.ldy, L.c0, L.cnt, v);
  }
}

template <typename Y, bool VEC>
__global__ __launch_bounds__(RNT) void k_norm_rows_restore(NormArgs a) {
  const Lanes L(a.lg, a.C, RNT);
  const RowGroups R(a, L, nullptr);
  float gamma[8], beta[8];
  params8(a, L.c0, gamma, beta);
  for (int64_t i = (int64_t)blockIdx.x * L.RL + L.rl; i < a.n; i += (int64_t)gridDim.x * L.RL) {
    float v[8], mean[8], rstd[8];
    Source<Q8, VEC>::load(a, i, L.c0, L.cnt, v);
    R.read(a, a.stats + i * 2 * a.G, mean, rstd);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = __builtin_fmaf((v[k] - mean[k]) * rstd[k], gamma[k], beta[k]);
    activate8(a.act, v);
    Row<Y, VEC>::store(static_cast<Y*>(a.y) + i * a.ldy, L.c0, L.cnt, v);
  }
}

template <typename T, bool VEC>
__global__ __launch_bounds__(RNT) void k_norm_rows_bwd(NormArgs a) {
  __shared__ float lds[RNT * 16];
  const Lanes L(a.lg, a.C, RNT);
  const RowGroups R(a, L, lds + (threadIdx.x >> 6) * 512);
  float gamma[8], beta[8], u[8] = {}, v[8] = {};
  params8(a, L.c0, gamma, beta);
  const float f = 1.0f / a.gs;
  for (int64_t i = (int64_t)blockIdx.x * L.RL + L.rl; i < a.n; i += (int64_t)gridDim.x * L.RL) {
    float t[8], w[8], g[8] = {}, mean[8], rstd[8], xn[8], A[8], B[8];
    Source<T, VEC>::load(a, i, L.c0, L.cnt, t);
    Row<float, VEC>::load(a.gy + i * a.ldgy, L.c0, L.cnt, w);
    if (a.ga) Row<float, VEC>::load(a.ga + i * a.ldga, L.c0, L.cnt, g);
    R.read(a, a.stats + i * 2 * a.G, mean, rstd);
    weigh<T, VEC>(a, t, mean, rstd, gamma, beta, w, xn);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (k >= L.cnt) w[k] = 0.0f;
      u[k] += w[k];
      v[k] = __builtin_fmaf(w[k], xn[k], v[k]);
      A[k] = k < L.cnt ? gamma[k] * w[k] : 0.0f;
      B[k] = k < L.cnt ? A[k] * xn[k] : 0.0f;
    }
    R.sum(a, L, A);
    R.sum(a, L, B);
#pragma unroll
    for (int k = 0; k < 8; ++k) A[k] *= f, B[k] *= f;
    grad8(rstd, gamma, A, B, w, xn, g);
    Row<float, VEC>::store(a.gx + i * a.ldgx, L.c0, L.cnt, g);
  }
  if (!a.part_c) return;
  for (int o = L.lpr; o < 64; o <<= 1) {
#pragma unroll
    for (int k = 0; k < 8; ++k) u[k] += __shfl_xor(u[k], o, 64), v[k] += __shfl_xor(v[k], o, 64);
  }
  __syncthreads();
  const int w8 = L.lpr * 8, wid = threadIdx.x >> 6;
  if ((threadIdx.x & 63) < (unsigned)L.lpr) {
#pragma unroll
    for (int k = 0; k < 8; ++k) lds[wid * 2 * w8 + L.c0 + k] = u[k], lds[wid * 2 * w8 + w8 + L.c0 + k] = v[k];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < a.C; c += RNT) {
    float x = 0.0f, y = 0.0f;
    for (int w = 0; w < RNT / 64; ++w) x += lds[w * 2 * w8 + c], y += lds[w * 2 * w8 + w8 + c];
    a.part_c[(int64_t)blockIdx.x * 2 * a.C + c] = x;
    a.part_c[(int64_t)blockIdx.x * 2 * a.C + a.C + c] = y;
  }
}

// ------------------------------------------------------------ checkpoints alone

template <typename T, bool VEC>
__global__ __launch_bounds__(RNT) void k_ckpt_store(NormArgs a) {
  const Lanes L(a.lg, a.C, RNT);
  for (int64_t i = (int64_t)blockIdx.x * L.RL + L.rl; i < a.n; i += (int64_t)gridDim.x * L.RL) {
    float v[8];
    Source<T, VEC>::load(a, i, L.c0, L.cnt, v);
    store_q8<VEC>(a.q, a.scale, i, a.C, L.c0, L.cnt, std::min(8, L.lpr), v);
  }
}

template <typename Y, bool VEC>
__global__ __launch_bounds__(RNT) void k_ckpt_load(NormArgs a) {
  const Lanes L(a.lg, a.C, RNT);
  for (int64_t i = (int64_t)blockIdx.x * L.RL + L.rl; i < a.n; i += (int64_t)gridDim.x * L.RL) {
    float v[8];
    Source<Q8, VEC>::load(a, i, L.c0, L.cnt, v);
    Row<Y, VEC>::store(static_cast<Y*>(a.y) + i * a.ldy, L.c0, L.cnt, v);
  }
}

// ------------------------------------------------------------ host side

int lanes_log2(int C) {
  int lg = 0;
  while ((8 << lg) < C) ++lg;
  return lg;
}

// Chunks of the summing pass: whole steps of the workgroup's rows, at most MAX_CHUNKS.
void chunking(int64_t n, int C, int64_t& rows, int64_t& chunks) {
  const int64_t step = NT >> lanes_log2(C);
  const int64_t steps = (n + step - 1) / step;
  rows = std::max<int64_t>(1, (steps + MAX_CHUNKS - 1) / MAX_CHUNKS) * step;
  chunks = (n + rows - 1) / rows;
}

// whole aligned groups of eight in every row
bool aligned(const void* p, int64_t ld, int size) {
  return !p || ((reinterpret_cast<uintptr_t>(p) & 15) == 0 && (ld * size & 15) == 0);
}

int size_of(int dtype) { return dtype == DSMP_BF16 ? 2 : 4; }

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
  int64_t rows, chunks;
  chunking(s.n, d.channels, rows, chunks);
  Carve cv(ws);
  NormWs w{};
  w.part = cv.take<float2>(rows_are_segments(s) ? 0 : (size_t)(chunks + s.n_seg) * d.groups);
  if (backward) w.part_c = cv.take<float>((size_t)std::max<int64_t>(chunks, MAX_CHUNKS) * 2 * d.channels);
  w.total = cv.used();
  return w;
}

NormArgs norm_args(const dsmp_norm_desc& d, const dsmp_segments& s) {
  NormArgs a{};
  a.n = s.n;
  a.C = d.channels;
  a.G = d.groups;
  a.gs = d.channels / d.groups;
  a.lg = lanes_log2(a.C);
  a.n_seg = (int)s.n_seg;
  a.ptr = s.ptr;
  a.len = s.ptr ? 0 : s.n / s.n_seg;
  a.eps = d.eps;
  a.act = d.act;
  int64_t chunks;
  chunking(s.n, a.C, a.R, chunks);
  a.nchunks = (int)chunks;
  return a;
}

// workgroups of the second pass and their rows
unsigned second_grid(const dsmp_handle* h, NormArgs& a) {
  const int64_t step = NT >> a.lg, steps = (a.n + step - 1) / step;
  const int64_t most = (int64_t)h->n_cu * 4;
  a.RA = std::max<int64_t>(1, (steps + most - 1) / most) * step;
  return (unsigned)std::max<int64_t>(1, (a.n + a.RA - 1) / a.RA);
}

unsigned row_grid(const dsmp_handle* h, const NormArgs& a, int per_cu) {
  const int64_t step = RNT >> a.lg;
  return (unsigned)std::min<int64_t>((a.n + step - 1) / step, (int64_t)h->n_cu * per_cu);
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
  const dsmp_status st = check_norm(h, desc, seg);
  if (st != DSMP_OK) return st;
  const int64_t n = seg->n;
  const int C = desc->channels;
  DSMP_CHECK(h, stats && (n == 0 || (x && y)), DSMP_INVALID_ARG, "a data pointer is NULL");
  DSMP_CHECK(h, !gamma == !beta, DSMP_INVALID_ARG, "gamma and beta go together");
  DSMP_CHECK(h, !addend == !sum, DSMP_INVALID_ARG, "an addend and the sum go together");
  DSMP_CHECK(h, !ck || n == 0 || (ck->q && ck->scale), DSMP_INVALID_ARG, "a checkpoint pointer is NULL");
  DSMP_CHECK(h, ldx >= C && ldy >= C && (!addend || (lda >= C && lds >= C)), DSMP_INVALID_ARG,
             "rows are closer than their channels");
  const NormWs w = norm_ws(*desc, *seg, false, ws);
  DSMP_CHECK(h, ws_bytes >= w.total && (ws || w.total == 0), DSMP_WORKSPACE_TOO_SMALL, "workspace needs %zu bytes", w.total);
  NormArgs a = norm_args(*desc, *seg);
  a.x = x, a.ldx = ldx, a.add = addend, a.lda = lda, a.sum = sum, a.lds = lds;
  a.gamma = gamma, a.beta = beta, a.y = y, a.ldy = ldy, a.stats = stats;
  if (ck) a.q = ck->q, a.scale = ck->scale;
  a.part = w.part;
  a.merge = 1;
  const int xs = size_of(desc->x_dtype), ys = size_of(desc->y_dtype);
  const bool vec = C % 8 == 0 && aligned(x, ldx, xs) && aligned(addend, lda, xs) && aligned(sum, lds, xs) &&
                   aligned(y, ldy, ys) && (!ck || (reinterpret_cast<uintptr_t>(ck->q) & 7) == 0);
  ProfScope prof(h, DSMP_K_NORM);
  by_type(desc->x_dtype, [&](auto xt) {
    by_type(desc->y_dtype, [&](auto yt) {
      by_bool(vec, [&](auto v) {
        using T = decltype(xt);
        using Y = decltype(yt);
        constexpr bool V = decltype(v)::value;
        if (rows_are_segments(*seg)) {
          by_bool(addend != nullptr, [&](auto ad) {
            by_bool(ck != nullptr, [&](auto c) {
              DSMP_GO((k_norm_rows<T, Y, V, decltype(ad)::value, decltype(c)::value>), row_grid(h, a, 16), RNT, 0);
            });
          });
          return;
        }
        if (n > 0)
          by_bool(addend != nullptr, [&](auto ad) {
            by_bool(ck != nullptr, [&](auto c) {
              DSMP_GO((k_norm_stats<T, V, decltype(ad)::value, decltype(c)::value>), a.nchunks, NT, stats_lds(a.lg, C));
            });
          });
        if (addend) a.x = sum, a.ldx = lds;
        const unsigned grid = second_grid(h, a);
        DSMP_GO((k_norm_apply<T, Y, V>), grid, NT, 0);
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
  const dsmp_status st = check_norm(h, desc, seg);
  if (st != DSMP_OK) return st;
  const int C = desc->channels;
  DSMP_CHECK(h, seg->n == 0 || (ck && ck->q && ck->scale && stats && y), DSMP_INVALID_ARG, "a data pointer is NULL");
  DSMP_CHECK(h, !gamma == !beta, DSMP_INVALID_ARG, "gamma and beta go together");
  DSMP_CHECK(h, ldy >= C, DSMP_INVALID_ARG, "rows are closer than their channels");
  if (seg->n == 0) return DSMP_OK;
  NormArgs a = norm_args(*desc, *seg);
  a.x = ck->q, a.xscale = ck->scale;
  a.gamma = gamma, a.beta = beta, a.y = y, a.ldy = ldy, a.stats = const_cast<float*>(stats);
  const bool vec = C % 8 == 0 && aligned(y, ldy, size_of(desc->y_dtype)) && (reinterpret_cast<uintptr_t>(ck->q) & 7) == 0;
  ProfScope prof(h, DSMP_K_NORM);
  by_type(desc->y_dtype, [&](auto yt) {
    by_bool(vec, [&](auto v) {
      using Y = decltype(yt);
      constexpr bool V = decltype(v)::value;
      if (rows_are_segments(*seg)) {
        DSMP_GO((k_norm_rows_restore<Y, V>), row_grid(h, a, 16), RNT, 0);
      } else {
        const unsigned grid = second_grid(h, a);
        DSMP_GO((k_norm_apply<Q8, Y, V>), grid, NT, 0);
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
  const dsmp_status st = check_norm(h, desc, seg);
  if (st != DSMP_OK) return st;
  const int64_t n = seg->n;
  const int C = desc->channels;
  DSMP_CHECK(h, (flags & ~DSMP_GRAD_ACCUMULATE) == 0, DSMP_INVALID_ARG, "unknown flags");
  DSMP_CHECK(h, !x || !ck, DSMP_INVALID_ARG, "x or its checkpoint, not both");
  DSMP_CHECK(h, n == 0 || ((x || (ck && ck->q && ck->scale)) && stats && grad_y && grad_x), DSMP_INVALID_ARG,
             "a data pointer is NULL");
  DSMP_CHECK(h, !gamma == !beta && !gamma == !dgamma && !gamma == !dbeta, DSMP_INVALID_ARG,
             "gamma, beta and their gradients go together");
  DSMP_CHECK(h, (!x || ldx >= C) && ldgy >= C && ldgx >= C && (!grad_addend || ldga >= C), DSMP_INVALID_ARG,
             "rows are closer than their channels");
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
  const bool vec = C % 8 == 0 && aligned(x, ldx, size_of(desc->x_dtype)) && aligned(grad_y, ldgy, 4) &&
                   aligned(grad_addend, ldga, 4) && aligned(grad_x, ldgx, 4) &&
                   (!ck || (reinterpret_cast<uintptr_t>(ck->q) & 7) == 0);
  ProfScope prof(h, DSMP_K_NORM);
  if (n == 0) {
    if (nred) DSMP_GO(k_norm_columns, nred, RNT, 0);   // sums of no chunk
    DSMP_LAUNCHED(h, "group norm backward");
    return DSMP_OK;
  }
  auto go = [&](auto xt) {
    by_bool(vec, [&](auto v) {
      using T = decltype(xt);
      constexpr bool V = decltype(v)::value;
      if (rows_are_segments(*seg)) {
        const unsigned grid = std::min<unsigned>(row_grid(h, a, 4), MAX_CHUNKS);
        a.nchunks = (int)grid;
        DSMP_GO((k_norm_rows_bwd<T, V>), grid, RNT, 0);
        if (nred) DSMP_GO(k_norm_columns, nred, RNT, 0);
        return;
      }
      DSMP_GO((k_norm_bwd_sums<T, V>), a.nchunks, NT, stats_lds(a.lg, C));
      a.nred = (int)nred;
      const unsigned grid = second_grid(h, a);
      DSMP_GO((k_norm_bwd_dx<T, V>), grid + nred, NT, 0);
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
  DSMP_CHECK(h, ld >= C, DSMP_INVALID_ARG, "rows are closer than their channels");
  return DSMP_OK;
}

}  // namespace

extern "C" dsmp_status dsmp_checkpoint_store(dsmp_handle* h, const void* x, int32_t dtype, int64_t ldx, int64_t n,
                                             int32_t channels, const dsmp_checkpoint* ck) {
  if (!h) return DSMP_INVALID_ARG;
  const dsmp_status st = check_ckpt(h, ck, x, dtype, ldx, n, channels);
  if (st != DSMP_OK || n == 0) return st;
  NormArgs a{};
  a.n = n, a.C = channels, a.lg = lanes_log2(channels);
  a.x = x, a.ldx = ldx, a.q = ck->q, a.scale = ck->scale;
  const bool vec = channels % 8 == 0 && aligned(x, ldx, size_of(dtype)) && (reinterpret_cast<uintptr_t>(ck->q) & 7) == 0;
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
  a.n = n, a.C = channels, a.lg = lanes_log2(channels);
  a.x = ck->q, a.xscale = ck->scale, a.y = y, a.ldy = ldy;
  const bool vec = channels % 8 == 0 && aligned(y, ldy, size_of(dtype)) && (reinterpret_cast<uintptr_t>(ck->q) & 7) == 0;
  ProfScope prof(h, DSMP_K_CKPT);
  by_type(dtype, [&](auto t) {
    by_bool(vec, [&](auto v) { DSMP_GO((k_ckpt_load<decltype(t), decltype(v)::value>), row_grid(h, a, 16), RNT, 0); });
  });
  DSMP_LAUNCHED(h, "checkpoint load");
  return DSMP_OK;
}
