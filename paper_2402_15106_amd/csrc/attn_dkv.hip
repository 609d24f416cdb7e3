// Attention within packed segments, backward: the gradients of the keys and values.
//
//   dv_j = sum_i P_ij dO_i,  dk_j = scale sum_i dS_ij q_i   (P, dS as for the queries)
//
// A workgroup owns keys of one key head, 32 to a wave, and passes over the rows of its
// segment: the queries of all G heads that share the keys, whose gradients so add up in
// the accumulators.  D_i comes from the pass for dq.
#include "attention.hpp"

using namespace dsmp;

namespace {

constexpr int NT = 256, NW = 4;

// WIDE: 128 keys to a workgroup.  FEW: 32, a quarter of a tile's rows to each wave.
template <typename T, int D, bool FEW>
struct Dkv {
  static constexpr int KEYS = FEW ? 32 : 32 * NW;
  static constexpr int BQ = FEW ? 32 * NW : sizeof(T) == 2 ? 64 : 32;
  static constexpr int SUB = FEW ? 1 : BQ / 32;
  static constexpr int P = pitch_of<T, D, false>();   // both matrices are read both ways
  static constexpr int PER = BQ * D * (int)sizeof(T) / 16 / NT, STEP = NT * 16 / (D * (int)sizeof(T));
  static constexpr bool AHEAD = !(FEW && sizeof(T) == 4 && D == 128);
  static constexpr int HELD = AHEAD ? PER : PER < 4 ? PER : 2;
  static constexpr int TILE = 2 * BQ * P + 6 * BQ * 4;
  static constexpr int JOIN = FEW ? NW * 32 * D * 4 : 0;
  static constexpr int LDS = TILE > JOIN ? TILE : JOIN;
};

template <typename T, int D, bool FEW, typename M>
__global__ __launch_bounds__(NT, D == 128 || (D == 64 && sizeof(T) == 4) ? 1 : 2) void k_attn_dkv(AttnArgs a) {
  using C = Dkv<T, D, FEW>;
  constexpr int ES = sizeof(T), KS = D / 16, DB = D / 32;
  typedef typename Frag<T>::type frag;
  __shared__ __align__(16) unsigned char smem[C::LDS];
  lds_u8* ldsQ = (lds_u8*)smem;
  lds_u8* ldsG = ldsQ + C::BQ * C::P;
  float* rows = (float*)(smem + 2 * C::BQ * C::P);   // lse, D, slope, x, y, z of the tile's rows

  const int tid = (int)threadIdx.x, l = tid & 63, h = l >> 5, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = (int)(blockIdx.x % (unsigned)a.Hk);
  const int64_t tile = blockIdx.x / (unsigned)a.Hk;
  int64_t first;
  const int seg = find_segment(a.kb, a.n_seg, 1, C::KEYS, tile, &first);
  const int64_t k0 = a.kb.at(seg), klen = a.kb.at(seg + 1) - k0, j0 = (tile - first) * C::KEYS;
  if (tile < first || j0 >= klen) return;
  const int64_t q0 = a.qb.at(seg), queries = a.qb.at(seg + 1) - q0, R = queries > 0 ? queries * a.G : 0;
  const int tiles = (int)((R + C::BQ - 1) / C::BQ);

  const bool cap = M::cap(a);
  const int dim = M::dim(a);
  const ScoreConst sc = score_const(a);
  const int64_t j = j0 + (FEW ? 0 : 32 * w) + (l & 31);
  const bool there = j < klen;
  const int64_t key = k0 + (there ? j : 0);
  frag kf[KS], vf[KS];
#pragma unroll
  for (int t = 0; t < KS; ++t) {
    const int c = 16 * t + 8 * h;
    kf[t] = read_frag<T>((const T*)a.k + key * a.ldk + kvh * a.hd + c, there && c < a.hd);
    vf[t] = read_frag<T>((const T*)a.v + key * a.ldv + kvh * a.hd + c, there && c < a.hd);
  }
  Place me{0.0f, 0.0f, 0.0f};
  if (dim && a.dim && there) me = place_of(a.pos_k, a.dim, key);

  const int row0 = tid / (D * ES / 16), c0 = tid % (D * ES / 16) * 16;
  const bool in = c0 < a.hd * ES;
  u32x4 regQ[C::HELD], regG[C::HELD];
  float rl = INFINITY, rd = 0.0f, rs = 0.0f;
  Place rp{0.0f, 0.0f, 0.0f};
  auto fetch = [&](int t, int first_unit) {
    const unsigned base = (unsigned)t * C::BQ;   // rows before this tile
    const unsigned i0 = base / (unsigned)a.G, g0 = base - i0 * a.G;
    const int64_t left = queries - i0;
    const int rem = (int)min((int64_t)C::BQ + 1, left);
    const int64_t at = q0 + i0;
    const auto bq = buffer_of((const T*)a.q + at * a.ldq + kvh * a.G * a.hd, (uint32_t)(rem * a.ldq * ES));
    const auto bg = buffer_of((const T*)a.go + at * a.ldgo + kvh * a.G * a.hd, (uint32_t)(rem * a.ldgo * ES));
#pragma unroll
    for (int i = 0; i < C::HELD; ++i) {
      const uint32_t x = g0 + row0 + (first_unit + i) * C::STEP, qi = (x * a.g_inv) >> 20, g = x - qi * a.G;
      const uint32_t off = g * (uint32_t)(a.hd * ES) + c0;
      regQ[i] = buffer_read(bq, in && (int)qi < rem ? qi * (uint32_t)(a.ldq * ES) + off : NOWHERE);
      regG[i] = buffer_read(bg, in && (int)qi < rem ? qi * (uint32_t)(a.ldgo * ES) + off : NOWHERE);
    }
    if (first_unit == 0 && tid < C::BQ) {
      const uint32_t x = g0 + tid, qi = (x * a.g_inv) >> 20, g = x - qi * a.G;
      rl = INFINITY, rd = 0.0f, rs = 0.0f, rp = Place{0.0f, 0.0f, 0.0f};
      if ((int64_t)qi < left) {
        const int64_t query = at + qi, slot = query * a.H + kvh * a.G + g;
        const float lse = a.lse_in[slot];
        rl = lse == -INFINITY ? INFINITY : lse * LOG2E;
        rd = a.delta[slot];
        if (dim && a.dim) rp = place_of(a.pos_q, a.dim, query), rs = a.slopes[kvh * a.G + g] * LOG2E;
      }
    }
  };
  auto put = [&](int first_unit) {
#pragma unroll
    for (int i = 0; i < C::HELD; ++i) {
      const int row = row0 + (first_unit + i) * C::STEP;
      *(__attribute__((address_space(3))) u32x4*)(ldsQ + row * C::P + c0) = regQ[i];
      *(__attribute__((address_space(3))) u32x4*)(ldsG + row * C::P + c0) = regG[i];
    }
    if (first_unit == 0 && tid < C::BQ) {
      rows[tid] = rl, rows[C::BQ + tid] = rd;
      if (dim) rows[2 * C::BQ + tid] = rs, rows[3 * C::BQ + tid] = rp.x, rows[4 * C::BQ + tid] = rp.y, rows[5 * C::BQ + tid] = rp.z;
    }
  };

  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) dk[d][i] = 0.0f, dv[d][i] = 0.0f;

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
    if (FEW && (int64_t)t * C::BQ + 32 * w >= R) continue;
#pragma unroll
    for (int b = 0; b < C::SUB; ++b) {
      const int at = 32 * ((FEW ? w : 0) + b);
      f32x16 x, dp;
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = 0.0f, dp[i] = 0.0f;
#pragma unroll
      for (int t2 = 0; t2 < KS; ++t2) {
        if (ES == 4) __builtin_amdgcn_sched_barrier(0);   // float32 fragments are large: not all of them at once
        x = mma(lds_rows<T>(ldsQ, C::P, at, 16 * t2), kf[t2], x);
        dp = mma(lds_rows<T>(ldsG, C::P, at, 16 * t2), vf[t2], dp);
      }
      float p[16], ds[16];
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const float* row = rows + at + 8 * i4 + 4 * h;
        const float4 lse = *(const float4*)row, delta = *(const float4*)(row + C::BQ);
        float4 sl{}, px{}, py{}, pz{};
        if (dim) {
          sl = *(const float4*)(row + 2 * C::BQ), px = *(const float4*)(row + 3 * C::BQ), py = *(const float4*)(row + 4 * C::BQ);
          if (dim > 2) pz = *(const float4*)(row + 5 * C::BQ);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 4 * i4 + e;
          float fall;
          float z = capped<T, true>(x[i], cap, sc, &fall);
          if (dim) z = fmaf(-(&sl.x)[e], distance(dim, me, (&px.x)[e], (&py.x)[e], (&pz.x)[e]), z);
          p[i] = exp2_of(z - (&lse.x)[e]);
          ds[i] = p[i] * (dp[i] - (&delta.x)[e]);
          if (cap) ds[i] *= fall;
        }
      }
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2) {
        const frag pf = to_frag<T>(&p[8 * t2]), sf = to_frag<T>(&ds[8 * t2]);
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          if (ES == 4) __builtin_amdgcn_sched_barrier(0);
          dv[d] = mma(lds_columns<T>(ldsG, C::P, at + 16 * t2, 32 * d), pf, dv[d]);
          dk[d] = mma(lds_columns<T>(ldsQ, C::P, at + 16 * t2, 32 * d), sf, dk[d]);
        }
      }
    }
  }

  // the lane's key once more: formed here, not kept in registers over the loop
  int lane = (int)threadIdx.x;
  asm volatile("" : "+v"(lane));
  const int64_t mine = j0 + (FEW ? lane & 31 : 32 * (lane >> 6) + (lane & 31));
  const bool mine_there = mine < klen;
  T* gk = (T*)a.gk + (k0 + mine) * a.ldgk + kvh * a.hd;
  T* gv = (T*)a.gv + (k0 + mine) * a.ldgv + kvh * a.hd;
  if (!FEW) {
    if (!mine_there) return;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const int c = 32 * d + 8 * i4 + 4 * h;
        if (c < a.hd) {
          store4(gk + c, dk[d][4 * i4] * a.scale, dk[d][4 * i4 + 1] * a.scale, dk[d][4 * i4 + 2] * a.scale,
                 dk[d][4 * i4 + 3] * a.scale);
          store4(gv + c, dv[d][4 * i4], dv[d][4 * i4 + 1], dv[d][4 * i4 + 2], dv[d][4 * i4 + 3]);
        }
      }
    return;
  }
  float* join = (float*)smem;   // the waves' parts, [wave][value][key], of dk and then of dv
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) join[(w * D + 32 * d + result_row(i)) * 32 + (l & 31)] = which ? dv[d][i] : dk[d][i];
    __syncthreads();
    const float scale = which ? 1.0f : a.scale;
    T* out = which ? gv : gk;
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      const int c = 32 * d + 4 * (tid >> 5);
      if (c >= a.hd || !mine_there) continue;
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = 0.0f;
#pragma unroll
        for (int k = 0; k < NW; ++k) v[e] += join[(k * D + c + e) * 32 + (l & 31)];
      }
      store4(out + c, v[0] * scale, v[1] * scale, v[2] * scale, v[3] * scale);
    }
  }
}

}  // namespace

namespace dsmp {

// Keys in tiles of 128 where these fill the card, else of 32.
dsmp_status launch_attention_dkv(dsmp_handle* h, const dsmp_attention_desc& d, AttnArgs a, int64_t nk) {
  const int64_t wide = tiles_of(nk, a.n_seg, 1, 32 * NW) * a.Hk, few = tiles_of(nk, a.n_seg, 1, 32) * a.Hk;
  by_attention(d, [&](auto t, auto width, auto mode) {
    using T = decltype(t);
    constexpr int D = decltype(width)::value;
    using M = decltype(mode);
    if (wide >= FILL) hipLaunchKernelGGL((k_attn_dkv<T, D, false, M>), dim3((unsigned)wide), dim3(NT), 0, h->stream, a);
    else hipLaunchKernelGGL((k_attn_dkv<T, D, true, M>), dim3((unsigned)few), dim3(NT), 0, h->stream, a);
  });
  return DSMP_OK;
}

}  // namespace dsmp
