// Norms of queries and keys for each head with the position rotation in the same
// pass, forward and backward.
//
//   u = gamma x r, r = 1 / sqrt(mean x^2 + eps);  t = pos[axis(p)] freq[p]
//   y_a = amp (u_a cos t - u_b sin t),  y_b = amp (u_a sin t + u_b cos t)
//   backward: g = amp times the pairs of dy turned by -t,  w = g gamma
//             dx = r (w - x r mean(w x r)),  dgamma = sum g x r
//
// A lane has 16 bytes of a head (VE = 4 or 8 values) and 2^lg lanes a head; a row's sines and
// cosines serve all of its heads.  The other value of a pair is the lane's own neighbour
// (interleaved pairs) or comes through LDS (half layout), so that every access to memory is
// of whole 16-byte pieces in a row.  Bound by memory.
#include "attention.hpp"

#include <cmath>

using namespace dsmp;

namespace {

constexpr int RT = 256;         // threads of a workgroup
// Workgroups of a backward pass (their sums of dgamma are kept): as many as the card holds at
// once; 99,991 x 10 heads of 64: 1,024 of them 103 us, 768 of them 86.
constexpr int MAX_PARTS = 768;

struct RotArgs {
  int64_t n;
  int heads[2], hd, rot, axes, lg, lanes;   // lanes: of a head, that have values
  int per_axis, interleaved;                // per_axis: pairs to a coordinate
  int chunks, per;                          // a row's heads (both sets, one after the other) in chunks of `per`
  float eps, amp;                           // eps < 0: no norm
  const void* x[2];
  const void* dy[2];
  void* y[2];
  int64_t ldx[2], lddy[2], ldy[2];
  const float* gamma[2];
  float* dgamma[2];
  const float *pos, *freq;
  float* part;
  int parts, accumulate;
};

template <typename T>
constexpr int VE = 16 / (int)sizeof(T);

// The other value of element e's pair (e itself where it is not rotated).
__device__ __forceinline__ int partner(const RotArgs& a, int e) {
  if (e >= a.rot) return e;
  if (a.interleaved) return e ^ 1;
  return e < (a.rot >> 1) ? e + (a.rot >> 1) : e - (a.rot >> 1);
}

// The pair's other values of a lane's own (0 for a value that is not rotated).  PIECE > 0 (half layout): through LDS, PIECE values at
// a time, which divides rot / 2 and VE, so that no piece has partners in two places; `sh` is the
// wave's own, 16 bytes to a lane, and a wave's LDS accesses stay in order.
template <typename T, int PIECE>
__device__ __forceinline__ void exchange(const RotArgs& a, const T* own, T* other, T* sh, int lane) {
  constexpr int N = VE<T>;
  if (PIECE == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) other[i] = lane * N + i < a.rot ? own[i ^ 1] : (T)0.0f;
    return;
  }
  typedef T whole __attribute__((ext_vector_type(N)));
  constexpr int P = PIECE ? PIECE : 1;
  const int wl = (int)threadIdx.x & 63, group = (wl >> a.lg) << a.lg;
  whole w;
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = own[i];
  *(whole*)(sh + wl * N) = w;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < N; i += P) {
    const T* from = sh + group * N + partner(a, lane * N + i);
    const bool turns = lane * N + i < a.rot;
    if constexpr (P == 1) {
      other[i] = turns ? from[0] : (T)0.0f;
    } else {
      typedef T piece __attribute__((ext_vector_type(P)));
      const piece p = *(const piece*)from;
#pragma unroll
      for (int k = 0; k < P; ++k) other[i + k] = turns ? p[k] : (T)0.0f;
    }
  }
}

template <typename T>
__device__ __forceinline__ void load_piece(T* v, const T* p) {
  typedef T whole __attribute__((ext_vector_type(VE<T>)));
  const whole w = *(const whole*)p;
#pragma unroll
  for (int i = 0; i < VE<T>; ++i) v[i] = w[i];
}
// past the caches: 100,000 x 16 heads of 64 102 us without the hint, 83 with it
template <typename T>
__device__ __forceinline__ void store_piece(T* p, const float* v) {
  typedef T whole __attribute__((ext_vector_type(VE<T>)));
  whole w;
#pragma unroll
  for (int i = 0; i < VE<T>; ++i) w[i] = (T)v[i];
  __builtin_nontemporal_store(w, (whole*)p);
}

// The row of an item (chunks of a row after one another; more than one only where the items
// are few enough for 32 bits).
__device__ __forceinline__ int64_t row_of_item(const RotArgs& a, int64_t item) {
  return a.chunks == 1 ? item : (int64_t)((unsigned)item / (unsigned)a.chunks);
}

// sum over the lanes of a head (2^lg of them, side by side)
__device__ __forceinline__ float sum_lanes(float v, int lg) {
  for (int o = 1; o < (1 << lg); o <<= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// For each value of a lane: what its own and its partner's count in the turned one
// (amp cos, and amp sin with its sign); 1 and 0 where nothing is turned.
template <typename T, int PIECE>
__device__ __forceinline__ void angles(const RotArgs& a, int64_t row, int lane, float* c, float* s) {
  constexpr int STEP = PIECE == 0 ? 2 : 1;
#pragma unroll
  for (int i = 0; i < VE<T>; i += STEP) {
    const int e = lane * VE<T> + i, half = a.rot >> 1;
    c[i] = 1.0f, s[i] = 0.0f;
    if (STEP == 2) c[i + STEP - 1] = 1.0f, s[i + STEP - 1] = 0.0f;
    if (e < a.rot) {
      const int p = STEP == 2 ? e >> 1 : e < half ? e : e - half;
      const int axis = p >= 2 * a.per_axis ? 2 : p >= a.per_axis ? 1 : 0;
      // turns in float64: the product of two float32 is exact, and what is left of it in one turn is within 2^-52 of it
      const double turns = (double)a.pos[row * a.axes + axis] * (double)a.freq[p] * 0.15915494309189533577;
      // the hardware's sine and cosine take turns; within 1.3e-7 over one turn (all 2^24 multiples of 2^-24 compared)
      const float rest = (float)(turns - __builtin_rint(turns));
      const float sn = __builtin_amdgcn_sinf(rest), cs = __builtin_amdgcn_cosf(rest);
      c[i] = a.amp * cs, s[i] = a.amp * (STEP == 2 || e < half ? -sn : sn);
      if (STEP == 2) c[i + STEP - 1] = c[i], s[i + STEP - 1] = -s[i];
    }
  }
}

// A row's chunk of heads to a group of lanes, RU of them on their way at once (1 where the chunks are of one head).
template <typename T, int PIECE, int RU>
__global__ __launch_bounds__(RT) void k_rotate(RotArgs a) {
  constexpr int N = VE<T>;
  __shared__ __align__(16) T sh[PIECE ? RU * RT * N : N];
  const int group = (int)threadIdx.x >> a.lg, lane = (int)threadIdx.x & ((1 << a.lg) - 1);
  T* mine = sh + (PIECE ? ((int)threadIdx.x & ~63) * N * RU : 0);
  const int64_t items = a.n * a.chunks, item = (int64_t)blockIdx.x * (RT >> a.lg) + group;
  const bool on = item < items && lane < a.lanes;
  const int64_t row = on ? row_of_item(a, item) : 0;
  const int c0 = on ? (int)(item - row * a.chunks) * a.per : 0;
  const int all = a.heads[0] + a.heads[1], c1 = min(c0 + a.per, all);
  T x[RU][N];
  auto fetch = [&](int j0) {
#pragma unroll
    for (int j = 0; j < RU; ++j) {
      const int hh = c0 + j0 + j, t = hh >= a.heads[0];
#pragma unroll
      for (int i = 0; i < N; ++i) x[j][i] = (T)0.0f;
      if (on && hh < c1)
        load_piece(x[j], (const T*)a.x[t] + row * a.ldx[t] + (int64_t)(hh - (t ? a.heads[0] : 0)) * a.hd + lane * N);
    }
  };
  fetch(0);
  // gamma goes into the angles' factors, one set for the queries and one for the keys
  float c[N], s[N], own[2][N], oth[2][N];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = lane * N + i;
      const bool g = on && a.gamma[t];
      own[t][i] = g ? a.gamma[t][e] : 1.0f, oth[t][i] = g ? a.gamma[t][partner(a, e)] : 1.0f;
    }
#pragma unroll
  for (int i = 0; i < N; ++i) c[i] = 1.0f, s[i] = 0.0f;
  if (on) angles<T, PIECE>(a, row, lane, c, s);
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < N; ++i) own[t][i] *= c[i], oth[t][i] *= s[i];
  const float mean = 1.0f / (float)a.hd;
  for (int j0 = 0; j0 < a.per; j0 += RU) {
    T now[RU][N];
#pragma unroll
    for (int j = 0; j < RU; ++j)
#pragma unroll
      for (int i = 0; i < N; ++i) now[j][i] = x[j][i];
    if (j0 + RU < a.per) fetch(j0 + RU);
#pragma unroll
    for (int j = 0; j < RU; ++j) {
      const int hh = c0 + j0 + j, t = hh >= a.heads[0];
      T other[N];
      exchange<T, PIECE>(a, now[j], other, mine + (PIECE ? j * 64 * N : 0), lane);
      float r = 1.0f, v[N];
      if (a.eps >= 0.0f) {
        float q = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) q = fmaf((float)now[j][i], (float)now[j][i], q);
        r = __builtin_amdgcn_rsqf(fmaf(sum_lanes(q, a.lg), mean, a.eps));
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float ow = t ? own[1][i] : own[0][i], ot = t ? oth[1][i] : oth[0][i];
        v[i] = r * fmaf((float)now[j][i], ow, (float)other[i] * ot);
      }
      if (on && hh < c1)
        store_piece((T*)a.y[t] + row * a.ldy[t] + (int64_t)(hh - (t ? a.heads[0] : 0)) * a.hd + lane * N, v);
    }
  }
}

// Backward; workgroups step over the items, so that a lane's sums of dgamma stay in
// its registers; a workgroup's are added up in a fixed order and kept, [part][2][hd].
template <typename T, int PIECE, int RUB>
__global__ __launch_bounds__(RT) void k_rotate_bwd(RotArgs a) {
  constexpr int N = VE<T>;
  constexpr int WORDS = std::max(RT / 64 * 2 * MAX_HEAD_DIM, RUB * RT * N * (int)sizeof(T) / 4);
  __shared__ __align__(16) float shf[WORDS];
  T* mine = (T*)shf + ((int)threadIdx.x & ~63) * N * RUB;
  const int groups = RT >> a.lg, group = (int)threadIdx.x >> a.lg, lane = (int)threadIdx.x & ((1 << a.lg) - 1);
  const int64_t items = a.n * a.chunks;
  const int all = a.heads[0] + a.heads[1];
  float gam[2][N], dg[2][N];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      gam[t][i] = lane < a.lanes && a.gamma[t] ? a.gamma[t][lane * N + i] : 1.0f;
      dg[t][i] = 0.0f;
    }
  const float mean = 1.0f / (float)a.hd;
  for (int64_t i0 = (int64_t)blockIdx.x * groups; i0 < items; i0 += (int64_t)gridDim.x * groups) {
    const int64_t item = i0 + group;
    const bool on = item < items && lane < a.lanes;
    const int64_t row = on ? row_of_item(a, item) : 0;
    const int c0 = on ? (int)(item - row * a.chunks) * a.per : 0, c1 = min(c0 + a.per, all);
    T xs[RUB][N], gs[RUB][N];
    auto fetch = [&](int j0) {
#pragma unroll
      for (int j = 0; j < RUB; ++j) {
        const int hh = c0 + j0 + j, t = hh >= a.heads[0];
        const int64_t at = (int64_t)(hh - (t ? a.heads[0] : 0)) * a.hd + lane * N;
#pragma unroll
        for (int i = 0; i < N; ++i) xs[j][i] = gs[j][i] = (T)0.0f;
        if (on && hh < c1) {
          load_piece(xs[j], (const T*)a.x[t] + row * a.ldx[t] + at);
          load_piece(gs[j], (const T*)a.dy[t] + row * a.lddy[t] + at);
        }
      }
    };
    fetch(0);
    float c[N], s[N];
#pragma unroll
    for (int i = 0; i < N; ++i) c[i] = 1.0f, s[i] = 0.0f;
    if (on) angles<T, PIECE>(a, row, lane, c, s);
    for (int j0 = 0; j0 < a.per; j0 += RUB) {
      T xn[RUB][N], gn[RUB][N];
#pragma unroll
      for (int j = 0; j < RUB; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) xn[j][i] = xs[j][i], gn[j][i] = gs[j][i];
      if (j0 + RUB < a.per) fetch(j0 + RUB);
#pragma unroll
      for (int j = 0; j < RUB; ++j) {
        const int hh = c0 + j0 + j, t = hh >= a.heads[0];
        T other[N];
        exchange<T, PIECE>(a, gn[j], other, mine + j * 64 * N, lane);
        float x[N], g[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          x[i] = (float)xn[j][i];
          g[i] = fmaf((float)gn[j][i], c[i], -(float)other[i] * s[i]);
        }
        if (a.eps >= 0.0f) {
          float q = 0.0f, m = 0.0f;
#pragma unroll
          for (int i = 0; i < N; ++i) q = fmaf(x[i], x[i], q);
          q = sum_lanes(q, a.lg);
          // a slot without a head has nothing to add to the sums: without eps its zeros would have an infinite 1 / rms
          const float r = on && hh < c1 ? __builtin_amdgcn_rsqf(fmaf(q, mean, a.eps)) : 0.0f;
#pragma unroll
          for (int i = 0; i < N; ++i) {
            x[i] *= r;
            const float d = g[i] * x[i];
            dg[0][i] += t ? 0.0f : d, dg[1][i] += t ? d : 0.0f;
            g[i] *= t ? gam[1][i] : gam[0][i];
            m = fmaf(g[i], x[i], m);
          }
          m = sum_lanes(m, a.lg) * mean;
#pragma unroll
          for (int i = 0; i < N; ++i) g[i] = r * (g[i] - x[i] * m);
        }
        if (on && hh < c1)
          store_piece((T*)a.y[t] + row * a.ldy[t] + (int64_t)(hh - (t ? a.heads[0] : 0)) * a.hd + lane * N, g);
      }
    }
  }
  if (!a.part) return;
  // the groups of a wave across its lanes, then the waves
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < N; ++i)
      for (int o = 1 << a.lg; o < 64; o <<= 1) dg[t][i] += __shfl_xor(dg[t][i], o, 64);
  __syncthreads();
  const int wl = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  if (wl < a.lanes) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < N; ++i) shf[(wave * 2 + t) * a.hd + wl * N + i] = dg[t][i];
  }
  __syncthreads();
  if ((int)threadIdx.x < 2 * a.hd) {
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < RT / 64; ++k) sum += shf[k * 2 * a.hd + threadIdx.x];
    a.part[(int64_t)blockIdx.x * 2 * a.hd + threadIdx.x] = sum;
  }
}

// dgamma: sixteen values to a workgroup, each from sixteen slices of the parts, which are
// added up in a fixed order, in float64.
__global__ __launch_bounds__(RT) void k_rotate_columns(RotArgs a) {
  __shared__ double sh[RT];
  const int e = (int)blockIdx.x * 16 + ((int)threadIdx.x & 15), slice = (int)threadIdx.x >> 4, columns = 2 * a.hd;
  double sum = 0.0;
#pragma unroll 8
  for (int p = slice; p < a.parts; p += 16) sum += (double)a.part[(int64_t)p * columns + e];
  sh[threadIdx.x] = sum;
  __syncthreads();
  if (slice) return;
  sum = 0.0;
  for (int k = 0; k < 16; ++k) sum += sh[16 * k + threadIdx.x];
  float* out = a.dgamma[e >= a.hd];
  if (!out) return;
  out += e >= a.hd ? e - a.hd : e;
  *out = (float)(sum + (a.accumulate ? (double)*out : 0.0));
}

dsmp_status check_rotate(dsmp_handle* h, const dsmp_rotate_desc* d, int64_t n) {
  DSMP_CHECK(h, d, DSMP_INVALID_ARG, "the descriptor is NULL");
  DSMP_CHECK(h, d->heads >= 1 && d->kv_heads >= 1 && d->head_dim >= 1, DSMP_INVALID_ARG, "no heads or no values in them");
  DSMP_CHECK(h, d->heads <= MAX_HEADS && d->kv_heads <= MAX_HEADS, DSMP_UNSUPPORTED, "more than %d heads", MAX_HEADS);
  DSMP_CHECK(h, d->head_dim % 8 == 0 && d->head_dim <= MAX_HEAD_DIM, DSMP_UNSUPPORTED,
             "head_dim must be a multiple of 8 up to %d", MAX_HEAD_DIM);
  DSMP_CHECK(h, d->dtype == DSMP_F32 || d->dtype == DSMP_BF16, DSMP_INVALID_ARG, "unknown dtype");
  DSMP_CHECK(h, d->axes >= 1 && d->axes <= 3, DSMP_INVALID_ARG, "1 to 3 coordinates");
  DSMP_CHECK(h, d->rot >= 0 && d->rot <= d->head_dim && d->rot % (2 * d->axes) == 0, DSMP_INVALID_ARG,
             "rot must be a multiple of 2 axes up to head_dim");
  DSMP_CHECK(h, d->layout == DSMP_ROTATE_HALF || d->layout == DSMP_ROTATE_INTERLEAVED, DSMP_INVALID_ARG, "unknown layout");
  DSMP_CHECK(h, d->norm == 0 || d->norm == 1, DSMP_INVALID_ARG, "norm is 0 or 1");
  DSMP_CHECK(h, std::isfinite(d->eps) && d->eps >= 0.0f && std::isfinite(d->amplitude), DSMP_INVALID_ARG,
             "eps must be finite and not negative, the amplitude finite");
  DSMP_CHECK(h, n >= 0, DSMP_INVALID_ARG, "negative rows");
  DSMP_CHECK(h, n < (int64_t)1 << 31, DSMP_UNSUPPORTED, "2^31 rows and more");
  return DSMP_OK;
}

int64_t rot_items_per_wg(const RotArgs& a) { return RT >> a.lg; }

// Lanes, and a row's heads in chunks: all of them to one group of lanes where that
// alone makes 2,048 workgroups, else so many chunks that there are about as many.
void place(RotArgs& a, const dsmp_rotate_desc& d, int64_t n) {
  a.n = n;
  a.hd = d.head_dim, a.rot = d.rot, a.axes = d.axes;
  a.per_axis = d.rot ? d.rot / 2 / d.axes : 1;
  a.lanes = d.head_dim * (d.dtype == DSMP_BF16 ? 2 : 4) / 16;
  a.interleaved = d.layout == DSMP_ROTATE_INTERLEAVED;
  a.lg = 0;
  while ((1 << a.lg) < a.lanes) ++a.lg;
  a.eps = d.norm ? d.eps : -1.0f, a.amp = d.amplitude;
  const int all = a.heads[0] + a.heads[1];
  const int64_t want = 2048 * rot_items_per_wg(a);
  int64_t chunks = std::min<int64_t>(all, std::max<int64_t>(1, want / std::max<int64_t>(1, n)));
  a.per = (int)ceil_div(all, chunks);
  a.chunks = (int)ceil_div(all, a.per);
}

int bwd_parts(const RotArgs& a) {
  return (int)std::min<int64_t>(MAX_PARTS, ceil_div(a.n * a.chunks, rot_items_per_wg(a)));
}

// Calls f with the type and the largest piece whose partners are together.
template <typename F>
void by_form(const dsmp_rotate_desc& d, F f) {
  const int half = d.layout == DSMP_ROTATE_INTERLEAVED || d.rot == 0 ? 0 : d.rot / 2;
  auto go = [&](auto t) {
    if (half == 0) f(t, std::integral_constant<int, 0>{});
    else if (sizeof(t) == 2 && half % 8 == 0) f(t, std::integral_constant<int, sizeof(t) == 2 ? 8 : 4>{});
    else if (half % 4 == 0) f(t, std::integral_constant<int, 4>{});
    else if (half % 2 == 0) f(t, std::integral_constant<int, 2>{});
    else f(t, std::integral_constant<int, 1>{});
  };
  if (d.dtype == DSMP_BF16) go(__bf16{});
  else go(float{});
}

}  // namespace

extern "C" dsmp_status dsmp_qk_rotate_forward(dsmp_handle* h, const dsmp_rotate_desc* desc, int64_t n, const void* q,
                                              int64_t ldq, const void* k, int64_t ldk, const float* gamma_q,
                                              const float* gamma_k, const float* pos, const float* freq, void* q_out,
                                              int64_t ldqo, void* k_out, int64_t ldko) {
  if (!h) return DSMP_INVALID_ARG;
  dsmp_status st = check_rotate(h, desc, n);
  if (st != DSMP_OK) return st;
  if (n == 0) return DSMP_OK;
  DSMP_CHECK(h, (q || k) && !q == !q_out && !k == !k_out, DSMP_INVALID_ARG, "queries or keys, each with its output");
  DSMP_CHECK(h, !desc->rot || (pos && freq), DSMP_INVALID_ARG, "coordinates and frequencies are needed");
  DSMP_CHECK(h, desc->norm || (!gamma_q && !gamma_k), DSMP_INVALID_ARG, "gamma without a norm");
  RotArgs a{};
  a.heads[0] = q ? desc->heads : 0, a.heads[1] = k ? desc->kv_heads : 0;
  const int wq = desc->heads * desc->head_dim, wk = desc->kv_heads * desc->head_dim;
  const int es = desc->dtype == DSMP_BF16 ? 2 : 4;
  st = check_matrices(h, es, {{q, ldq, wq, "q"}, {k, ldk, wk, "k"}, {q_out, ldqo, wq, "q_out"}, {k_out, ldko, wk, "k_out"}});
  if (st != DSMP_OK) return st;
  place(a, *desc, n);
  a.x[0] = q, a.x[1] = k, a.ldx[0] = ldq, a.ldx[1] = ldk;
  a.y[0] = q_out, a.y[1] = k_out, a.ldy[0] = ldqo, a.ldy[1] = ldko;
  a.gamma[0] = gamma_q, a.gamma[1] = gamma_k, a.pos = pos, a.freq = freq;
  const int64_t grid = (n * a.chunks + rot_items_per_wg(a) - 1) / rot_items_per_wg(a);
  DSMP_CHECK(h, grid < (int64_t)1 << 24, DSMP_UNSUPPORTED, "too many rows for one call");
  DeviceScope dev(h);
  ProfScope prof(h, DSMP_K_ROTATE);
  by_form(*desc, [&](auto t, auto form) {
    constexpr int PIECE = decltype(form)::value;
    if (a.per == 1) hipLaunchKernelGGL((k_rotate<decltype(t), PIECE, 1>), dim3((unsigned)grid), dim3(RT), 0, h->stream, a);
    else hipLaunchKernelGGL((k_rotate<decltype(t), PIECE, 4>), dim3((unsigned)grid), dim3(RT), 0, h->stream, a);
  });
  DSMP_LAUNCHED(h, "rotation");
  return DSMP_OK;
}

extern "C" dsmp_status dsmp_qk_rotate_workspace(const dsmp_rotate_desc* desc, int64_t n, size_t* bwd_ws_bytes) {
  const dsmp_status st = check_rotate(nullptr, desc, n);
  if (st != DSMP_OK) return st;
  if (!bwd_ws_bytes) return DSMP_INVALID_ARG;
  *bwd_ws_bytes = desc->norm ? (size_t)MAX_PARTS * 2 * desc->head_dim * sizeof(float) : 0;
  return DSMP_OK;
}

extern "C" dsmp_status dsmp_qk_rotate_backward(dsmp_handle* h, const dsmp_rotate_desc* desc, int64_t n, const void* q,
                                               int64_t ldq, const void* k, int64_t ldk, const float* gamma_q,
                                               const float* gamma_k, const float* pos, const float* freq,
                                               const void* grad_q_out, int64_t ldgqo, const void* grad_k_out,
                                               int64_t ldgko, void* grad_q, int64_t ldgq, void* grad_k, int64_t ldgk,
                                               float* dgamma_q, float* dgamma_k, int32_t flags, void* ws,
                                               size_t ws_bytes) {
  if (!h) return DSMP_INVALID_ARG;
  dsmp_status st = check_rotate(h, desc, n);
  if (st != DSMP_OK) return st;
  DSMP_CHECK(h, (flags & ~DSMP_GRAD_ACCUMULATE) == 0, DSMP_INVALID_ARG, "unknown flags");
  DSMP_CHECK(h, desc->norm || (!gamma_q && !gamma_k), DSMP_INVALID_ARG, "gamma without a norm");
  DSMP_CHECK(h, !gamma_q == !dgamma_q && !gamma_k == !dgamma_k, DSMP_INVALID_ARG, "a gamma and its gradient go together");
  RotArgs a{};
  if (n > 0) {
    DSMP_CHECK(h, (q || k) && !q == !grad_q && !k == !grad_k && !q == !grad_q_out && !k == !grad_k_out, DSMP_INVALID_ARG,
               "queries or keys, each with its gradients");
    DSMP_CHECK(h, (q || !gamma_q) && (k || !gamma_k), DSMP_INVALID_ARG, "a gamma without its values");
    DSMP_CHECK(h, !desc->rot || (pos && freq), DSMP_INVALID_ARG, "coordinates and frequencies are needed");
    const int wq = desc->heads * desc->head_dim, wk = desc->kv_heads * desc->head_dim;
    const int es = desc->dtype == DSMP_BF16 ? 2 : 4;
    st = check_matrices(h, es, {{q, ldq, wq, "q"}, {k, ldk, wk, "k"}, {grad_q_out, ldgqo, wq, "grad_q_out"},
                                {grad_k_out, ldgko, wk, "grad_k_out"}, {grad_q, ldgq, wq, "grad_q"}, {grad_k, ldgk, wk, "grad_k"}});
    if (st != DSMP_OK) return st;
  }
  const bool sums = gamma_q || gamma_k;
  const size_t need = sums ? (size_t)MAX_PARTS * 2 * desc->head_dim * sizeof(float) : 0;
  DSMP_CHECK(h, !need || (ws && ws_bytes >= need), DSMP_WORKSPACE_TOO_SMALL, "workspace needs %zu bytes", need);
  DSMP_CHECK(h, !need || (reinterpret_cast<uintptr_t>(ws) & 3) == 0, DSMP_INVALID_ARG, "the workspace must be 4-byte aligned");
  a.heads[0] = q ? desc->heads : 0, a.heads[1] = k ? desc->kv_heads : 0;
  if (n > 0) place(a, *desc, n);
  a.hd = desc->head_dim;
  a.x[0] = q, a.x[1] = k, a.ldx[0] = ldq, a.ldx[1] = ldk;
  a.dy[0] = grad_q_out, a.dy[1] = grad_k_out, a.lddy[0] = ldgqo, a.lddy[1] = ldgko;
  a.y[0] = grad_q, a.y[1] = grad_k, a.ldy[0] = ldgq, a.ldy[1] = ldgk;
  a.gamma[0] = gamma_q, a.gamma[1] = gamma_k, a.dgamma[0] = dgamma_q, a.dgamma[1] = dgamma_k;
  a.pos = pos, a.freq = freq, a.part = sums ? (float*)ws : nullptr;
  a.accumulate = flags & DSMP_GRAD_ACCUMULATE;
  if (n == 0 && !sums) return DSMP_OK;
  DeviceScope dev(h);
  ProfScope prof(h, DSMP_K_ROTATE);
  if (n > 0) {
    a.parts = bwd_parts(a);
    by_form(*desc, [&](auto t, auto form) {
      constexpr int PIECE = decltype(form)::value;
      if (a.per == 1) hipLaunchKernelGGL((k_rotate_bwd<decltype(t), PIECE, 1>), dim3(a.parts), dim3(RT), 0, h->stream, a);
      else hipLaunchKernelGGL((k_rotate_bwd<decltype(t), PIECE, 2>), dim3(a.parts), dim3(RT), 0, h->stream, a);
    });
  }
  if (sums) hipLaunchKernelGGL(k_rotate_columns, dim3(a.hd / 8), dim3(RT), 0, h->stream, a);
  DSMP_LAUNCHED(h, "rotation backward");
  return DSMP_OK;
}
