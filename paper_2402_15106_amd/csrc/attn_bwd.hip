// Attention backward: the call, and its kernels for few rows and keys.
#include "attn_bwd.hpp"

using namespace dsmp;

namespace {

// Both gradients in one launch, for tiles of 32 rows or keys: the first dkv_groups workgroups
// take those of the keys, which are the longer ones and form D_i of their rows
// themselves and so wait for nobody; the others those of the queries.
// ROLE 1 and 2: the one or the other alone (wide heads in float32: both together leave the scalar
// registers no room).
template <typename T, int D, int ROLE, typename M>
__global__ __launch_bounds__(BT, D == 128 || (D == 64 && sizeof(T) == 4) ? 1 : 2) void k_attn_bwd_few(AttnArgs a) {
  using C = Bwd<T, D, true, true>;   // the larger of both
  DSMP_BWD_LDS(C, lds);
  if (ROLE == 1 || (ROLE == 0 && blockIdx.x < a.dkv_groups)) dkv_tile<T, D, true, false, M>(a, lds, blockIdx.x);
  else dq_tile<T, D, true, M>(a, lds, blockIdx.x - (ROLE == 0 ? a.dkv_groups : 0));
}

// The splits of the gradients added up in their order, four values to a thread: those of dq, then
// of dk, then of dv (where there is more than one of each).
template <typename T>
__global__ __launch_bounds__(BT) void k_attn_bwd_join(AttnArgs a) {
  const int64_t nq = a.splits > 1 ? a.nq * a.H * a.hd / 4 : 0, nk = a.splits_k > 1 ? a.nk * a.Hk * a.hd / 4 : 0;
  int64_t i = (int64_t)blockIdx.x * BT + threadIdx.x;
  const int which = i < nq ? 0 : i < nq + nk ? 1 : 2;
  i -= which == 0 ? 0 : which == 1 ? nq : nq + nk;
  if (which == 2 && i >= nk) return;
  const int width = (which ? a.Hk : a.H) * a.hd, splits = which ? a.splits_k : a.splits;
  const int64_t row = 4 * i / width, step = 4 * (which ? nk : nq);
  const Bounds& b = which ? a.kb : a.qb;
  if (row < b.at(0) || row >= b.at(a.n_seg)) return;
  const float* from = (which == 0 ? a.part : which == 1 ? a.part_k : a.part_v) + 4 * i;
  float4 v = *(const float4*)from;
#pragma unroll 4
  for (int s = 1; s < splits; ++s) {
    const float4 x = *(const float4*)(from + s * step);
    v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
  }
  T* out = (T*)(which == 0 ? a.gq : which == 1 ? a.gk : a.gv) + row * (which == 0 ? a.ldgq : which == 1 ? a.ldgk : a.ldgv);
  store4(out + (4 * i - row * width), v.x, v.y, v.z, v.w);
}

struct BwdWs {
  float *shift, *minus_d, *q, *k, *v;
  size_t total;
};

BwdWs bwd_ws(const dsmp_attention_desc& d, const dsmp_segments& qs, const dsmp_segments& ks, void* ws) {
  const BwdPlan p = bwd_plan(d, qs, ks);
  Carve cv(ws);
  BwdWs w{};
  w.shift = cv.take<float>((size_t)qs.n * d.heads), w.minus_d = cv.take<float>((size_t)qs.n * d.heads);
  const size_t of_q = p.splits_q > 1 ? (size_t)p.splits_q * qs.n * d.heads * d.head_dim : 0;
  const size_t of_k = p.splits_k > 1 ? (size_t)p.splits_k * ks.n * d.kv_heads * d.head_dim : 0;
  w.q = cv.take<float>(of_q), w.k = cv.take<float>(of_k), w.v = cv.take<float>(of_k);
  w.total = cv.used();
  return w;
}

}  // namespace

namespace dsmp {

size_t attention_bwd_bytes(const dsmp_attention_desc& d, const dsmp_segments& qs, const dsmp_segments& ks) {
  return bwd_ws(d, qs, ks, nullptr).total;
}

}  // namespace dsmp

extern "C" dsmp_status dsmp_attention_backward(dsmp_handle* h, const dsmp_attention_desc* desc, const dsmp_segments* qs,
                                               const dsmp_segments* ks, const void* q, int64_t ldq, const void* k,
                                               int64_t ldk, const void* v, int64_t ldv, const float* pos_q,
                                               const float* pos_k, const float* slopes, const void* out, int64_t ldo,
                                               const float* lse, const void* grad_out, int64_t ldgo, void* grad_q,
                                               int64_t ldgq, void* grad_k, int64_t ldgk, void* grad_v, int64_t ldgv,
                                               void* ws, size_t ws_bytes) {
  if (!h) return DSMP_INVALID_ARG;
  dsmp_status st = check_attention(h, desc, qs, ks);
  if (st != DSMP_OK) return st;
  DSMP_CHECK(h, (qs->n == 0 || (q && out && lse && grad_out && grad_q)) && (ks->n == 0 || (k && v && grad_k && grad_v)),
             DSMP_INVALID_ARG, "a data pointer is NULL");
  DSMP_CHECK(h, desc->dim == 0 || (slopes && (qs->n == 0 || pos_q) && (ks->n == 0 || pos_k)), DSMP_INVALID_ARG,
             "coordinates and slopes are needed");
  const int es = desc->dtype == DSMP_BF16 ? 2 : 4, wq = desc->heads * desc->head_dim, wk = desc->kv_heads * desc->head_dim;
  st = check_matrices(h, es, {{q, ldq, wq, "q"}, {k, ldk, wk, "k"}, {v, ldv, wk, "v"}, {out, ldo, wq, "out"},
                              {grad_out, ldgo, wq, "grad_out"}, {grad_q, ldgq, wq, "grad_q"},
                              {grad_k, ldgk, wk, "grad_k"}, {grad_v, ldgv, wk, "grad_v"}});
  if (st != DSMP_OK) return st;
  const BwdWs w = bwd_ws(*desc, *qs, *ks, ws);
  DSMP_CHECK(h, !w.total || (ws && ws_bytes >= w.total), DSMP_WORKSPACE_TOO_SMALL, "workspace needs %zu bytes", w.total);
  DSMP_CHECK(h, reinterpret_cast<uintptr_t>(ws) % 16 == 0, DSMP_INVALID_ARG, "the workspace must be 16-byte aligned");
  const BwdPlan p = bwd_plan(*desc, *qs, *ks);
  AttnArgs a = attn_args(*desc, *qs, *ks);
  // Biases that fall fast leave few keys of many: 2,895 x 2,895, 2 heads of 16, the queries' gradients 0.0026 off, as sums
  // of two 0.0018; 2,048 x 2,048, 4 heads of 64, which pays most, 82 -> 92 us.
  if (desc->dim && ks->n <= 4096 * ks->n_seg) a.fine = 1;
  a.q = q, a.ldq = ldq, a.k = k, a.ldk = ldk, a.v = v, a.ldv = ldv, a.o = out, a.ldo = ldo, a.go = grad_out, a.ldgo = ldgo;
  a.gq = grad_q, a.ldgq = ldgq, a.gk = grad_k, a.ldgk = ldgk, a.gv = grad_v, a.ldgv = ldgv;
  a.lse_in = lse, a.shift = w.shift, a.minus_d = w.minus_d, a.part = w.q, a.part_k = w.k, a.part_v = w.v;
  a.splits = p.splits_q, a.splits_k = p.splits_k;
  a.pos_q = pos_q, a.pos_k = pos_k, a.slopes = slopes;
  DeviceScope dev(h);
  ProfScope prof(h, DSMP_K_ATTN_BWD);
  // a launch for keys in wide tiles reads what the queries' has written
  if (p.wide_q && p.grid_q) launch_attention_dq(h, *desc, a, p.grid_q);
  const int64_t few_q = p.wide_q ? 0 : p.grid_q, few_k = p.wide_k ? 0 : p.grid_k;
  a.dkv_groups = (unsigned)few_k;
  const int64_t joined = ((p.splits_q > 1 ? qs->n * wq : 0) + (p.splits_k > 1 ? 2 * ks->n * wk : 0)) / 4;
  by_attention(*desc, [&](auto t, auto width, auto mode) {
    using T = decltype(t);
    constexpr int D = decltype(width)::value;
    using M = decltype(mode);
    if constexpr (sizeof(T) == 4 && D == 128) {
      if (few_k) hipLaunchKernelGGL((k_attn_bwd_few<T, D, 1, M>), dim3((unsigned)few_k), dim3(BT), 0, h->stream, a);
      if (few_q) hipLaunchKernelGGL((k_attn_bwd_few<T, D, 2, M>), dim3((unsigned)few_q), dim3(BT), 0, h->stream, a);
    } else if (few_q + few_k) {
      const int64_t first = few_q + few_k > MAX_GROUPS ? few_k : few_q + few_k;   // what one launch takes
      hipLaunchKernelGGL((k_attn_bwd_few<T, D, 0, M>), dim3((unsigned)first), dim3(BT), 0, h->stream, a);
      a.dkv_groups = 0;
      if (first < few_q + few_k)
        hipLaunchKernelGGL((k_attn_bwd_few<T, D, 0, M>), dim3((unsigned)few_q), dim3(BT), 0, h->stream, a);
    }
  });
  if (p.wide_k && p.grid_k) launch_attention_dkv(h, *desc, a, p.grid_k);
  if (joined) {
    const dim3 grid(ceil_div(joined, BT));
    if (desc->dtype == DSMP_BF16) hipLaunchKernelGGL((k_attn_bwd_join<__bf16>), grid, dim3(BT), 0, h->stream, a);
    else hipLaunchKernelGGL((k_attn_bwd_join<float>), grid, dim3(BT), 0, h->stream, a);
  }
  DSMP_LAUNCHED(h, "attention backward");
  return DSMP_OK;
}
