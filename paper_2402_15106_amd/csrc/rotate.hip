// Norms of queries and keys for each head with the position rotation in the same
// pass, forward and backward.
//
//   u = gamma x r, r = 1 / sqrt(mean x^2 + eps);  t = pos[axis(p)] freq[p]
//   y_a = amp (u_a cos t - u_b sin t),  y_b = amp (u_a sin t + u_b cos t)
//   backward: g = amp times the pairs of dy turned by -t,  w = g gamma
//             dx = r (w - x r mean(w x r)),  dgamma = sum g x r
//
// A head is taken by LP = 2^lg >= head_dim / 8 lanes with eight values each; which
// eight is chosen so that both values of a pair are a lane's own, and a row's sines
// and cosines (four pairs to a lane) serve all of its heads.
#include "attention.hpp"

#include <cmath>

using namespace dsmp;

namespace {

constexpr int RT = 256;        // threads of a workgroup
constexpr int RU = 4;          // heads of a lane's row that are on their way at once
constexpr int MAX_PARTS = 1024; // workgroups of a backward pass (their sums of dgamma are kept)

struct RotArgs {
  int64_t n;
  int heads[2], hd, rot, axes, lg, lanes;   // lanes: head_dim / 8
  int per_axis;                             // pairs to a coordinate
  int chunks, per;                          // a row's heads (both sets, one after the other) in chunks of `per`
  float eps, amp;
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

// Where a lane's eight values are.  EIGHT: eight in a row (interleaved pairs, or no
// pairs).  SPLIT: four and their four partners rot / 2 further on, behind the rotated
// part eight in a row (half layout, rot a multiple of 8).  PAIRS: four pairs, each
// value addressed by itself (half layout, any other rot).
enum { EIGHT = 0, SPLIT = 1, PAIRS = 2 };

template <int FORM>
__device__ __forceinline__ int value_at(const RotArgs& a, int lane, int i) {
  if (FORM == EIGHT) return 8 * lane + i;
  const int half = a.rot >> 1;
  if (FORM == SPLIT) {
    if (8 * lane >= a.rot) return 8 * lane + i;
    return i < 4 ? 4 * lane + i : half + 4 * lane + i - 4;
  }
  const int p = 4 * lane + (i & 3);      // pairs behind rot / 2: values from rot on, two by two
  if (p >= half) return 2 * p + (i >> 2);
  return i < 4 ? p : p + half;
}

template <typename T, int FORM>
__device__ __forceinline__ void load8(float* v, const T* head, const RotArgs& a, int lane) {
  if (FORM == PAIRS) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)head[value_at<FORM>(a, lane, i)];
    return;
  }
  if (FORM == EIGHT && sizeof(T) == 2) {
    typedef T t8 __attribute__((ext_vector_type(8)));
    const t8 w = *(const t8*)(head + 8 * lane);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)w[i];
    return;
  }
  const T* lo = head + value_at<FORM>(a, lane, 0);
  const T* hi = head + value_at<FORM>(a, lane, 4);
  typedef T t4 __attribute__((ext_vector_type(4)));
  const t4 l = *(const t4*)lo, u = *(const t4*)hi;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (float)l[i], v[4 + i] = (float)u[i];
}

template <typename T, int FORM>
__device__ __forceinline__ void store8(const float* v, T* head, const RotArgs& a, int lane) {
  if (FORM == PAIRS) {
#pragma unroll
    for (int i = 0; i < 8; ++i) head[value_at<FORM>(a, lane, i)] = (T)v[i];
    return;
  }
  if (FORM == EIGHT && sizeof(T) == 2) {
    typedef T t8 __attribute__((ext_vector_type(8)));
    t8 w;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = (T)v[i];
    *(t8*)(head + 8 * lane) = w;
    return;
  }
  typedef T t4 __attribute__((ext_vector_type(4)));
  t4 l, u;
#pragma unroll
  for (int i = 0; i < 4; ++i) l[i] = (T)v[i], u[i] = (T)v[4 + i];
  *(t4*)(head + value_at<FORM>(a, lane, 0)) = l;
  *(t4*)(head + value_at<FORM>(a, lane, 4)) = u;
}

// the two registers of a lane's pair k (0..3), the row's pair 4 lane + k
template <int FORM>
__device__ __forceinline__ constexpr int first_of(int k) { return FORM == EIGHT ? 2 * k : k; }
template <int FORM>
__device__ __forceinline__ constexpr int second_of(int k) { return FORM == EIGHT ? 2 * k + 1 : k + 4; }

// sum over the lanes of a head (2^lg of them, side by side)
__device__ __forceinline__ float sum_lanes(float v, int lg) {
  for (int o = 1; o < (1 << lg); o <<= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// amp cos and amp sin of a lane's four pairs; pairs that are not rotated get 1 and 0
__device__ __forceinline__ void angles(const RotArgs& a, int64_t row, int lane, float* c, float* s) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int p = 4 * lane + k;
    c[k] = 1.0f, s[k] = 0.0f;
    if (p < (a.rot >> 1)) {
      const int axis = p >= 2 * a.per_axis ? 2 : p >= a.per_axis ? 1 : 0;
      // turns in float64: the product of two float32 is exact, and so is what is left of it in one turn, but for 2^-53 of it
      const double turns = (double)a.pos[row * a.axes + axis] * (double)a.freq[p] * 0.15915494309189533577;
      float sn, cs;
      sincospif(2.0f * (float)(turns - __builtin_rint(turns)), &sn, &cs);
      c[k] = a.amp * cs, s[k] = a.amp * sn;
    }
  }
}

// One row and chunk of heads to a group of lanes.  Bound by memory: values read and
// written once.
template <typename T, int FORM>
__global__ __launch_bounds__(RT) void k_rotate(RotArgs a) {
  const int group = (int)threadIdx.x >> a.lg, lane = (int)threadIdx.x & ((1 << a.lg) - 1);
  const int64_t items = a.n * a.chunks, item = (int64_t)blockIdx.x * (RT >> a.lg) + group;
  const bool on = item < items && lane < a.lanes;
  const int64_t row = on ? item / a.chunks : 0;
  const int c0 = on ? (int)(item - row * a.chunks) * a.per : 0;
  const int all = a.heads[0] + a.heads[1], c1 = min(c0 + a.per, all);
  float cs[4], sn[4], gam[2][8];
  if (on) angles(a, row, lane, cs, sn);
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 8; ++i) gam[t][i] = on && a.gamma[t] ? a.gamma[t][value_at<FORM>(a, lane, i)] : 1.0f;
  const float mean = 1.0f / (float)a.hd;
  for (int j0 = 0; j0 < a.per; j0 += RU) {
    float v[RU][8];
#pragma unroll
    for (int j = 0; j < RU; ++j) {
      const int hh = c0 + j0 + j, t = hh >= a.heads[0];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] = 0.0f;
      if (on && hh < c1)
        load8<T, FORM>(v[j], (const T*)a.x[t] + row * a.ldx[t] + (int64_t)(hh - (t ? a.heads[0] : 0)) * a.hd, a, lane);
    }
#pragma unroll
    for (int j = 0; j < RU; ++j) {
      const int hh = c0 + j0 + j, t = hh >= a.heads[0];
      float r = 1.0f;
      if (a.eps >= 0.0f) {
        float q = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) q = fmaf(v[j][i], v[j][i], q);
        r = 1.0f / sqrtf(fmaf(sum_lanes(q, a.lg), mean, a.eps));
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] *= r * (t ? gam[1][i] : gam[0][i]);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float p = v[j][first_of<FORM>(k)], q = v[j][second_of<FORM>(k)];
        v[j][first_of<FORM>(k)] = p * cs[k] - q * sn[k];
        v[j][second_of<FORM>(k)] = p * sn[k] + q * cs[k];
      }
      if (on && hh < c1)
        store8<T, FORM>(v[j], (T*)a.y[t] + row * a.ldy[t] + (int64_t)(hh - (t ? a.heads[0] : 0)) * a.hd, a, lane);
    }
  }
}

// Backward; workgroups step over the items, so that a lane's sums of dgamma stay in
// its registers; a workgroup's are added up in a fixed order and kept, [part][2][hd].
template <typename T, int FORM>
__global__ __launch_bounds__(RT) void k_rotate_bwd(RotArgs a) {
  __shared__ float sh[RT * 8];
  const int groups = RT >> a.lg, group = (int)threadIdx.x >> a.lg, lane = (int)threadIdx.x & ((1 << a.lg) - 1);
  const int64_t items = a.n * a.chunks;
  const int all = a.heads[0] + a.heads[1];
  float gam[2][8], dg[2][8];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      gam[t][i] = lane < a.lanes && a.gamma[t] ? a.gamma[t][value_at<FORM>(a, lane, i)] : 1.0f;
      dg[t][i] = 0.0f;
    }
  const float mean = 1.0f / (float)a.hd;
  for (int64_t i0 = (int64_t)blockIdx.x * groups; i0 < items; i0 += (int64_t)gridDim.x * groups) {
    const int64_t item = i0 + group;
    const bool on = item < items && lane < a.lanes;
    const int64_t row = on ? item / a.chunks : 0;
    const int c0 = on ? (int)(item - row * a.chunks) * a.per : 0, c1 = min(c0 + a.per, all);
    float cs[4], sn[4];
    if (on) angles(a, row, lane, cs, sn);
    constexpr int U = 2;
    for (int j0 = 0; j0 < a.per; j0 += U) {
      float x[U][8], g[U][8];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int hh = c0 + j0 + j, t = hh >= a.heads[0];
        const int64_t at = (int64_t)(hh - (t ? a.heads[0] : 0)) * a.hd;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] = g[j][i] = 0.0f;
        if (on && hh < c1) {
          load8<T, FORM>(x[j], (const T*)a.x[t] + row * a.ldx[t] + at, a, lane);
          load8<T, FORM>(g[j], (const T*)a.dy[t] + row * a.lddy[t] + at, a, lane);
        }
      }
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int hh = c0 + j0 + j, t = hh >= a.heads[0];
        const bool here = on && hh < c1;
        const int64_t at = (int64_t)(hh - (t ? a.heads[0] : 0)) * a.hd;
        if (here) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float p = g[j][first_of<FORM>(k)], q = g[j][second_of<FORM>(k)];
            g[j][first_of<FORM>(k)] = p * cs[k] + q * sn[k];
            g[j][second_of<FORM>(k)] = q * cs[k] - p * sn[k];
          }
        }
        if (a.eps >= 0.0f) {
          float q = 0.0f, m = 0.0f;
#pragma unroll
          for (int i = 0; i < 8; ++i) q = fmaf(x[j][i], x[j][i], q);
          const float r = 1.0f / sqrtf(fmaf(sum_lanes(q, a.lg), mean, a.eps));
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x[j][i] *= r;
            const float d = g[j][i] * x[j][i];
            if (here) dg[0][i] += t ? 0.0f : d, dg[1][i] += t ? d : 0.0f;
            g[j][i] *= t ? gam[1][i] : gam[0][i];
            m = fmaf(g[j][i], x[j][i], m);
          }
          m = sum_lanes(m, a.lg) * mean;
#pragma unroll
          for (int i = 0; i < 8; ++i) g[j][i] = r * (g[j][i] - x[j][i] * m);
        }
        if (here) store8<T, FORM>(g[j], (T*)a.y[t] + row * a.ldy[t] + at, a, lane);
      }
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) sh[(int)threadIdx.x * 8 + i] = dg[t][i];
    __syncthreads();
    for (int e = (int)threadIdx.x; e < 8 * a.lanes; e += RT) {
      float sum = 0.0f;
      for (int g = 0; g < groups; ++g) sum += sh[(g << a.lg) * 8 + e];
      a.part[((int64_t)blockIdx.x * 2 + t) * a.hd + value_at<FORM>(a, e >> 3, e & 7)] = sum;
    }
  }
}

// dgamma: a wave to a value; the parts are added up in a fixed order, in float64
__global__ __launch_bounds__(64) void k_rotate_columns(RotArgs a) {
  const int t = (int)blockIdx.x / a.hd, e = (int)blockIdx.x % a.hd;
  if (!a.dgamma[t]) return;
  double sum = 0.0;
  for (int p = (int)threadIdx.x; p < a.parts; p += 64) sum += (double)a.part[((int64_t)p * 2 + t) * a.hd + e];
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if (threadIdx.x == 0) a.dgamma[t][e] = (float)(sum + (a.accumulate ? (double)a.dgamma[t][e] : 0.0));
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
  a.lanes = d.head_dim / 8;
  a.lg = 0;
  while ((1 << a.lg) < a.lanes) ++a.lg;
  a.eps = d.norm ? d.eps : -1.0f, a.amp = d.amplitude;
  const int all = a.heads[0] + a.heads[1];
  const int64_t want = 2048 * rot_items_per_wg(a);
  int64_t chunks = std::min<int64_t>(all, std::max<int64_t>(1, want / std::max<int64_t>(1, n)));
  a.per = (int)ceil_div(all, chunks);
  a.chunks = (int)ceil_div(all, a.per);
}

int form_of(const dsmp_rotate_desc& d) {
  if (d.layout == DSMP_ROTATE_INTERLEAVED || d.rot == 0) return EIGHT;
  return d.rot % 8 == 0 ? SPLIT : PAIRS;
}

int bwd_parts(const RotArgs& a) {
  return (int)std::min<int64_t>(MAX_PARTS, ceil_div(a.n * a.chunks, rot_items_per_wg(a)));
}

template <typename F>
void by_form(int dtype, int form, F f) {
  auto go = [&](auto t) {
    if (form == EIGHT) f(t, std::integral_constant<int, EIGHT>{});
    else if (form == SPLIT) f(t, std::integral_constant<int, SPLIT>{});
    else f(t, std::integral_constant<int, PAIRS>{});
  };
  if (dtype == DSMP_BF16) go(__bf16{});
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
  by_form(desc->dtype, form_of(*desc), [&](auto t, auto form) {
    hipLaunchKernelGGL((k_rotate<decltype(t), decltype(form)::value>), dim3((unsigned)grid), dim3(RT), 0, h->stream, a);
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
    by_form(desc->dtype, form_of(*desc), [&](auto t, auto form) {
      hipLaunchKernelGGL((k_rotate_bwd<decltype(t), decltype(form)::value>), dim3(a.parts), dim3(RT), 0, h->stream, a);
    });
  }
  if (sums) hipLaunchKernelGGL(k_rotate_columns, dim3(2 * a.hd), dim3(64), 0, h->stream, a);
  DSMP_LAUNCHED(h, "rotation backward");
  return DSMP_OK;
}
