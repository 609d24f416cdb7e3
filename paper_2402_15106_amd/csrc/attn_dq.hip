// Attention within packed segments, backward: the gradient of the queries.
//
//   P_ij = e^(z_ij - lse_i),  D_i = dO_i . o_i,  dS_ij = P_ij (dO_i . v_j - D_i) (1 - tanh^2)
//   dq_i = scale sum_j dS_ij k_j
//
// Rows as in the forward pass.  The pass over the keys has no atomics and keeps dq in
// registers; the pass for dk and dv forms P and dS a second time (two of its four
// products), which sums of dq over workgroups in a fixed order would cost in memory instead.
#include "attention.hpp"

using namespace dsmp;

namespace {

constexpr int NT = 256, NW = 4;

template <typename T, int D, bool FEW>
struct Dq {
  static constexpr int ROWS = FEW ? 32 : 32 * NW;
  static constexpr int BN = FEW ? 32 * NW : sizeof(T) == 2 ? 64 : 32;
  static constexpr int SUB = FEW ? 1 : BN / 32;
  static constexpr int PK = pitch_of<T, D, false>(), PV = pitch_of<T, D, true>();   // K is read both ways
  static constexpr int PER = BN * D * (int)sizeof(T) / 16 / NT, STEP = NT * 16 / (D * (int)sizeof(T));
  // the next tile waits in registers, but for FEW's large ones in float32: those come four units at a time
  static constexpr bool AHEAD = !(FEW && sizeof(T) == 4 && D == 128);
  static constexpr int HELD = AHEAD || PER < 4 ? PER : 4;
  static constexpr int TILE = BN * (PK + PV) + 3 * BN * 4;
  static constexpr int JOIN = FEW ? NW * 32 * D * 4 : 0;
  static constexpr int LDS = TILE > JOIN ? TILE : JOIN;
};

template <typename T, int D, bool FEW, typename M>
__global__ __launch_bounds__(NT, (D == 128 && (FEW || sizeof(T) == 4)) || (D == 64 && FEW && sizeof(T) == 4) ? 1 : 2) void k_attn_dq(AttnArgs a) {
  using C = Dq<T, D, FEW>;
  constexpr int ES = sizeof(T), KS = D / 16, DB = D / 32;
  typedef typename Frag<T>::type frag;
  __shared__ __align__(16) unsigned char smem[C::LDS];
  lds_u8* ldsK = (lds_u8*)smem;
  lds_u8* ldsV = ldsK + C::BN * C::PK;
  float* places = (float*)(smem + C::BN * (C::PK + C::PV));

  const int tid = (int)threadIdx.x, l = tid & 63, h = l >> 5, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = (int)(blockIdx.x % (unsigned)a.Hk);
  const int64_t tile = blockIdx.x / (unsigned)a.Hk;
  int64_t first;
  const int seg = find_segment(a.qb, a.n_seg, a.G, C::ROWS, tile, &first);
  const int64_t q0 = a.qb.at(seg), R = (a.qb.at(seg + 1) - q0) * a.G, r0 = (tile - first) * C::ROWS;
  if (tile < first || r0 >= R) return;
  const int64_t k0 = a.kb.at(seg), klen = a.kb.at(seg + 1) - k0;
  const int tiles = klen > 0 ? (int)((klen + C::BN - 1) / C::BN) : 0;

  const bool cap = M::cap(a);
  const int dim = M::dim(a);
  const ScoreConst sc = score_const(a);
  const int64_t r = r0 + (FEW ? 0 : 32 * w) + (l & 31);
  const bool there = r < R;
  const unsigned rq = there ? (unsigned)r / (unsigned)a.G : 0u, rg = there ? (unsigned)r - rq * a.G : 0u;
  const int64_t query = q0 + rq;
  const int head = kvh * a.G + (int)rg;
  const int64_t slot = query * a.H + head;
  frag qf[KS], gf[KS];
  float delta = 0.0f;
#pragma unroll
  for (int t = 0; t < KS; ++t) {
    const int c = 16 * t + 8 * h;
    const bool in = there && c < a.hd;
    qf[t] = read_frag<T>((const T*)a.q + query * a.ldq + head * a.hd + c, in);
    gf[t] = read_frag<T>((const T*)a.go + query * a.ldgo + head * a.hd + c, in);
    const frag of = read_frag<T>((const T*)a.o + query * a.ldo + head * a.hd + c, in);
#pragma unroll
    for (int e = 0; e < 8; ++e) delta = fmaf((float)gf[t][e], (float)of[e], delta);
  }
  delta += other_half(delta);
  if (there && h == 0 && (!FEW || w == 0)) a.delta[slot] = delta;
  const float lse = there ? a.lse_in[slot] : INFINITY, lse2 = lse == -INFINITY ? INFINITY : lse * LOG2E;
  Place me{0.0f, 0.0f, 0.0f};
  float slope2 = 0.0f;
  if (dim && a.dim && there) me = place_of(a.pos_q, a.dim, query), slope2 = a.slopes[head] * LOG2E;

  // a thread's 16-byte units of a tile: one place in every STEP-th row
  const int row0 = tid / (D * ES / 16), c0 = tid % (D * ES / 16) * 16;
  const bool in = c0 < a.hd * ES;
  const uint32_t offK = in ? (uint32_t)(row0 * a.ldk * ES + c0) : NOWHERE, stepK = (uint32_t)(C::STEP * a.ldk * ES);
  const uint32_t offV = in ? (uint32_t)(row0 * a.ldv * ES + c0) : NOWHERE, stepV = (uint32_t)(C::STEP * a.ldv * ES);
  u32x4 regK[C::HELD], regV[C::HELD];
  Place key{0.0f, 0.0f, 0.0f};
  auto fetch = [&](int t, int i0) {
    const int64_t j0 = k0 + (int64_t)t * C::BN;
    const int rem = (int)min((int64_t)C::BN, klen - (int64_t)t * C::BN);
    const auto bk = buffer_of((const T*)a.k + j0 * a.ldk + kvh * a.hd, (uint32_t)(rem * a.ldk * ES));
    const auto bv = buffer_of((const T*)a.v + j0 * a.ldv + kvh * a.hd, (uint32_t)(rem * a.ldv * ES));
#pragma unroll
    for (int i = 0; i < C::HELD; ++i)
      regK[i] = buffer_read(bk, offK + (i0 + i) * stepK), regV[i] = buffer_read(bv, offV + (i0 + i) * stepV);
    if (dim && a.dim && i0 == 0 && tid < rem) key = place_of(a.pos_k, a.dim, j0 + tid);
  };
  auto put = [&](int i0) {
#pragma unroll
    for (int i = 0; i < C::HELD; ++i) {
      const int row = row0 + (i0 + i) * C::STEP;
      *(__attribute__((address_space(3))) u32x4*)(ldsK + row * C::PK + c0) = regK[i];
      *(__attribute__((address_space(3))) u32x4*)(ldsV + row * C::PV + c0) = regV[i];
    }
    if (dim && i0 == 0 && tid < C::BN) places[tid] = key.x, places[C::BN + tid] = key.y, places[2 * C::BN + tid] = key.z;
  };

  f32x16 acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[d][i] = 0.0f;

  if (C::AHEAD && tiles > 0) fetch(0, 0);
  for (int t = 0; t < tiles; ++t) {
    __syncthreads();
    if (C::AHEAD) {
      put(0);
    } else {
#pragma unroll 1
      for (int i0 = 0; i0 < C::PER; i0 += C::HELD) fetch(t, i0), put(i0);
    }
    __syncthreads();
    if (C::AHEAD && t + 1 < tiles) fetch(t + 1, 0);
    const int rem = (int)min((int64_t)C::BN, klen - (int64_t)t * C::BN);
    if (FEW && 32 * w >= rem) continue;
#pragma unroll
    for (int b = 0; b < C::SUB; ++b) {
      const int at = 32 * ((FEW ? w : 0) + b);
      f32x16 x, dp;
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = 0.0f, dp[i] = 0.0f;
#pragma unroll
      for (int t2 = 0; t2 < KS; ++t2) {
        x = mma(lds_rows<T>(ldsK, C::PK, at, 16 * t2), qf[t2], x);
        dp = mma(lds_rows<T>(ldsV, C::PV, at, 16 * t2), gf[t2], dp);
      }
      float ds[16];
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        float4 px{}, py{}, pz{};
        if (dim) {
          const float* p = places + at + 8 * i4 + 4 * h;
          px = *(const float4*)p, py = *(const float4*)(p + C::BN);
          if (dim > 2) pz = *(const float4*)(p + 2 * C::BN);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 4 * i4 + e;
          float fall;
          float z = capped<T, true>(x[i], cap, sc, &fall);
          if (dim) z = fmaf(-slope2, distance(dim, me, (&px.x)[e], (&py.x)[e], (&pz.x)[e]), z);
          ds[i] = exp2_of(z - lse2) * (dp[i] - delta);
          if (cap) ds[i] *= fall;
        }
      }
      if (at + 32 > rem) {   // behind the last key
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (at + result_row(i) >= rem) ds[i] = 0.0f;
      }
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2) {
        const frag f = to_frag<T>(&ds[8 * t2]);
#pragma unroll
        for (int d = 0; d < DB; ++d) acc[d] = mma(lds_columns<T>(ldsK, C::PK, at + 16 * t2, 32 * d), f, acc[d]);
      }
    }
  }

  T* out = (T*)a.gq + query * a.ldgq + head * a.hd;
  if (!FEW) {
    if (!there) return;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const int c = 32 * d + 8 * i4 + 4 * h;
        if (c < a.hd)
          store4(out + c, acc[d][4 * i4] * a.scale, acc[d][4 * i4 + 1] * a.scale, acc[d][4 * i4 + 2] * a.scale,
                 acc[d][4 * i4 + 3] * a.scale);
      }
    return;
  }
  float* join = (float*)smem;   // the waves' parts, [wave][value][row]
  __syncthreads();
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) join[(w * D + 32 * d + result_row(i)) * 32 + (l & 31)] = acc[d][i];
  __syncthreads();
  if (!there) return;
#pragma unroll
  for (int d = 0; d < DB; ++d) {
    const int c = 32 * d + 4 * (tid >> 5);
    if (c >= a.hd) continue;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = 0.0f;
#pragma unroll
      for (int k = 0; k < NW; ++k) v[e] += join[(k * D + c + e) * 32 + (l & 31)];
    }
    store4(out + c, v[0] * a.scale, v[1] * a.scale, v[2] * a.scale, v[3] * a.scale);
  }
}

}  // namespace

namespace dsmp {

// Rows in tiles of 128 where these fill the card, else of 32 (as in the forward pass).
dsmp_status launch_attention_dq(dsmp_handle* h, const dsmp_attention_desc& d, AttnArgs a) {
  const int64_t wide = tiles_of(a.qb.n, a.n_seg, a.G, 32 * NW) * a.Hk, few = tiles_of(a.qb.n, a.n_seg, a.G, 32) * a.Hk;
  by_attention(d, [&](auto t, auto width, auto mode) {
    using T = decltype(t);
    constexpr int D = decltype(width)::value;
    using M = decltype(mode);
    if (wide >= FILL) hipLaunchKernelGGL((k_attn_dq<T, D, false, M>), dim3((unsigned)wide), dim3(NT), 0, h->stream, a);
    else hipLaunchKernelGGL((k_attn_dq<T, D, true, M>), dim3((unsigned)few), dim3(NT), 0, h->stream, a);
  });
  return DSMP_OK;
}

}  // namespace dsmp
