// Attention within packed segments, backward: what a workgroup does for the gradients of the
// queries (dq_tile) and for those of the keys and values (dkv_tile).
//
//   P_ij = e^(z_ij - lse_i),  D_i = dO_i . o_i,  dS_ij = P_ij (dO_i . v_j - D_i) (1 - tanh^2)
//   dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i P_ij dO_i
//
// Neither has atomics: a workgroup owns its rows or its keys and keeps their sums in registers.
// P and dS are so formed in both (two products of seven), which sums over workgroups in a
// fixed order would cost in memory instead.  D comes from the rounded out in bfloat16, an error of up to
// 2^-8 |dO| |out| that all keys of a row share: with many keys it is lost in their own
// roundings, with few it is the largest (4 to 12 keys: dq 0.0026 to 0.0032 off).  Where a segment's keys are in one block of 32
// FEW tiles take D from the weights instead, D = sum_j P_ij dP_ij (dq and dk 0.0017 off).  The gradients of shared key heads add up in the
// accumulators: the rows of a key head are the queries times the G heads that share it.
#pragma once

#include "attention.hpp"

namespace dsmp {

constexpr int BT = 256, BW = 4;   // threads and waves of a workgroup

// WIDE: 32 rows (or keys) to a wave, 128 to a workgroup, all keys (rows) of a tile to every wave.
// FEW: 32 to a workgroup, a quarter of a tile's keys (rows) to each wave; joined at the end.
// KEYS_OWNED: dkv_tile.  bfloat16 tiles are copied into two buffers in turn, one barrier to a tile; float32
// ones wait in registers.
template <typename T, int D, bool FEW, bool KEYS_OWNED>
struct Bwd {
  static constexpr bool DMA = sizeof(T) == 2;
  static constexpr int OWN = FEW ? FEW_ROWS : WIDE_ROWS;
  static constexpr int BN = FEW ? 32 * BW : DMA ? 64 : 32;
  static constexpr int SUB = FEW ? 1 : BN / 32;
  static constexpr int PITCH = DMA ? 2 * D : pitch_of<T, D, true>(), MATRIX = BN * PITCH;
  static constexpr int EXTRA = (KEYS_OWNED ? 6 : 3) * BN;   // float32 of the rows that go along
  // float32: 16-byte units to a thread; the next tile waits in registers, but for FEW's large ones: those come one at a time
  static constexpr int PER = BN * D * (int)sizeof(T) / 16 / BT, STEP = BT * 16 / (D * (int)sizeof(T));
  static constexpr bool AHEAD = !(FEW && D == 128);
  static constexpr int HELD = AHEAD ? PER : 1;
  static_assert(FEW_ROWS == 32 && WIDE_ROWS == 32 * BW, "32 rows or keys to a wave");
  static_assert(!FEW || MATRIX >= 2 * 32 * D * 4, "two waves' parts fit into a matrix");
  static_assert(PER >= 1 && PER * BT * 16 == BN * D * (int)sizeof(T), "whole units for every thread");
};

// A workgroup's LDS: two buffers of two matrices and what goes along.  They are arrays of their own
// in the kernels, so that a copy into one buffer is not waited for by reads of the other.
struct BwdLds {
  unsigned char *a0, *b0, *a1, *b1;
  float *extra0, *extra1;
};
#define DSMP_BWD_LDS(C, name)                                                                                     \
  __shared__ __align__(1024) unsigned char name##a0[C::MATRIX], name##b0[C::MATRIX], name##a1[C::DMA ? C::MATRIX : 16], \
      name##b1[C::DMA ? C::MATRIX : 16];                                                                          \
  __shared__ __align__(16) float name##x0[C::EXTRA], name##x1[C::DMA ? C::EXTRA : 4];                             \
  const BwdLds name{name##a0, name##b0, name##a1, name##b1, name##x0, name##x1}

// The four waves' results of the same 32 rows added up in LDS ([value][row], two waves' in each of a buffer's
// matrices) and written: 256 threads with a row and four values in 32 each.
template <typename T, int D>
__device__ __forceinline__ void join_rows(const f32x16* acc, const BwdLds& lds, float scale, T* out, float* part, int hd, bool there) {
  const int tid = (int)threadIdx.x, l = tid & 63, w = tid >> 6;
  auto part_of = [&](int wave) { return (float*)(wave < 2 ? lds.a0 : lds.b0) + (wave & 1) * 32 * D; };
  __syncthreads();
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) part_of(w)[(32 * d + result_row(i)) * 32 + (l & 31)] = acc[d][i];
  __syncthreads();
#pragma unroll
  for (int d = 0; d < D / 32; ++d) {
    const int c = 32 * d + 4 * (tid >> 5);
    if (c >= hd || !there) continue;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = 0.0f;
#pragma unroll
      for (int k = 0; k < BW; ++k) v[e] += part_of(k)[(c + e) * 32 + (l & 31)];
      v[e] *= scale;
    }
    if (part) *(float4*)(part + c) = make_float4(v[0], v[1], v[2], v[3]);
    else store4(out + c, v[0], v[1], v[2], v[3]);
  }
}

// Of a wave's 32 lanes.
__device__ __forceinline__ float sum_of_half(float v) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) v += __shfl_xor(v, o, 64);
  return v;
}

template <typename T, int D, bool FEW, typename M>
__device__ __forceinline__ void dq_tile(const AttnArgs& a, const BwdLds& lds, unsigned group) {
  using C = Bwd<T, D, FEW, false>;
  constexpr int ES = sizeof(T), KS = D / 16, DB = D / 32;
  typedef typename Frag<T>::type frag;

  const int tid = (int)threadIdx.x, l = tid & 63, h = l >> 5, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = (int)(group % (unsigned)a.Hk);
  const unsigned rest = group / (unsigned)a.Hk;
  const int split = (int)(rest % (unsigned)a.splits);
  const int64_t tile = rest / (unsigned)a.splits;
  int64_t first;
  const int seg = FEW ? find_segment(a.qb, a.n_seg, a.G, C::OWN, tile, &first)
                      : find_segment_longest_first(a.qb, a.kb, a.n_seg, a.G, C::OWN, tile, &first);
  const int64_t q0 = a.qb.at(seg), R = (a.qb.at(seg + 1) - q0) * a.G, r0 = (tile - first) * C::OWN;
  if (tile < first || r0 >= R) return;
  const int64_t k0 = a.kb.at(seg), klen = a.kb.at(seg + 1) - k0;
  const int tiles = klen > 0 ? (int)((klen + C::BN - 1) / C::BN) : 0;
  const int per = (tiles + a.splits - 1) / a.splits;
  const int t_begin = min(split * per, tiles), t_end = min(t_begin + per, tiles);

  const bool cap = M::cap(a);
  const int dim = M::dim(a);
  const Score<T, false> sc(a, cap);
  const RowOf row = row_of(a, q0, r0, R, kvh, FEW, tid);
  const int64_t slot = row.query * a.H + row.head;
  frag qf[KS], gf[KS];
  float delta = 0.0f;
#pragma unroll
  for (int t = 0; t < KS; ++t) {
    const int c = 16 * t + 8 * h;
    const bool in = row.there && c < a.hd;
    qf[t] = read_frag<T>((const T*)a.q + row.query * a.ldq + row.head * a.hd + c, in);
    gf[t] = read_frag<T>((const T*)a.go + row.query * a.ldgo + row.head * a.hd + c, in);
    const frag of = read_frag<T>((const T*)a.o + row.query * a.ldo + row.head * a.hd + c, in);
#pragma unroll
    for (int e = 0; e < 8; ++e) delta = fmaf((float)gf[t][e], (float)of[e], delta);
  }
  apply_sign<KS>(qf, sc.sign);
  delta += other_half(delta);
  // the exponent of a weight is A u + shift; a row without keys has the weights 0
  const float lse = row.there ? a.lse_in[slot] : INFINITY, shift = lse == -INFINITY ? -INFINITY : sc.C - lse * LOG2E;
  if (row.there && h == 0 && split == 0 && (!FEW || w == 0)) a.shift[slot] = shift, a.minus_d[slot] = -delta;
  Place me{0.0f, 0.0f, 0.0f};
  float slope = 0.0f;
  if (dim && a.dim && row.there) me = place_of(a.pos_q, a.dim, row.query), slope = a.slopes[row.head] * sc.per_slope;

  f32x16 acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = f32x16{};

  const LanePlace place = lane_place<D>();
  auto step = [&](lds_u8* ldsK, lds_u8* ldsV, const float* places, int t) {
    const int rem = (int)min((int64_t)C::BN, klen - (int64_t)t * C::BN);
    if (FEW && 32 * w >= rem) return;
    LanePlace lane = place;
    formed_here(lane);
#pragma unroll
    for (int b = 0; b < C::SUB; ++b) {
      const int at = 32 * ((FEW ? w : 0) + b);
      // fragments one step ahead of their products, as in the forward pass
      f32x16 x{}, dp;
#pragma unroll
      for (int i = 0; i < 16; ++i) dp[i] = -delta;
      frag kf[2], vf[2];
      kf[0] = tile_rows<T, D>(ldsK, lane, at, 0), vf[0] = tile_rows<T, D>(ldsV, lane, at, 0);
#pragma unroll
      for (int t2 = 0; t2 < KS; ++t2) {
        if (t2 + 1 < KS)
          kf[(t2 + 1) & 1] = tile_rows<T, D>(ldsK, lane, at, t2 + 1), vf[(t2 + 1) & 1] = tile_rows<T, D>(ldsV, lane, at, t2 + 1);
        x = mma(kf[t2 & 1], qf[t2], x);
        dp = mma(vf[t2 & 1], gf[t2], dp);
        __builtin_amdgcn_sched_barrier(0);
      }
      int left = rem - at - 4 * h;
      asm volatile("" : "+v"(left));   // compared with constants, not with sixteen row numbers kept over the loop
      float more = 0.0f;   // sum of P (dP - D) over the keys: what D lacks, where all of them are here
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
          float u = sc.template u<true>(x[i], cap, &fall);
          if (dim) u = fmaf(-slope, distance(dim, me, (&px.x)[e], (&py.x)[e], (&pz.x)[e]), u);
          const float p = exp2_of(fmaf(u, sc.A, shift));
          if constexpr (FEW && C::DMA) {
            x[i] = 8 * i4 + e < left ? p : 0.0f;
            more = fmaf(x[i], dp[i], more);
          } else {
            x[i] = p * dp[i];
          }
          if (cap) x[i] *= fall;
        }
        if (dim) __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (FEW && C::DMA) {
        more = klen <= 32 ? more + other_half(more) : 0.0f;
        if (klen <= 32 && row.there && h == 0) a.minus_d[slot] = -delta - more;   // for a launch for keys in wide tiles
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] *= dp[i] - more;
      } else if (at + 32 > rem) {   // behind the last key
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (8 * (i >> 2) + (i & 3) >= left) x[i] = 0.0f;
      }
      __builtin_amdgcn_sched_barrier(0);
      frag cf[2], f{}, rest[2]{};
      cf[0] = tile_columns<T, D>(ldsK, lane, at, 0);
#pragma unroll
      for (int k = 0; k < 2 * DB; ++k) {
        const int t2 = k / DB, d = k % DB;
        if (d == 0) {
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = x[8 * t2 + i];
          f = to_frag<T>(v);
          if constexpr (FEW && C::DMA) rest[t2] = rest_frag(v, f);
        }
        if (k + 1 < 2 * DB) cf[(k + 1) & 1] = tile_columns<T, D>(ldsK, lane, at + 16 * ((k + 1) / DB), 32 * ((k + 1) % DB));
        acc[d] = mma(cf[k & 1], f, acc[d]);
        if (d & 1 || DB == 1) __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (FEW && C::DMA)
        if (a.fine) {
#pragma unroll
          for (int k = 0; k < 2 * DB; ++k) {
            acc[k % DB] = mma(tile_columns<T, D>(ldsK, lane, at + 16 * (k / DB), 32 * (k % DB)), rest[k / DB], acc[k % DB]);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
    }
#pragma unroll
    for (int d = 0; d < DB; ++d) asm volatile("" : "+v"(acc[d]));   // one place for the sums after either buffer's tile
  };

  const T* keys = (const T*)a.k + k0 * a.ldk + kvh * a.hd;
  const T* values = (const T*)a.v + k0 * a.ldv + kvh * a.hd;
  if constexpr (C::DMA) {
    using TC = TileCopy<D, C::BN>;
    const bool in = TC::unit0() < a.hd * ES;
    const uint32_t offK = in ? (uint32_t)(TC::row0() * a.ldk * ES + TC::unit0()) : NOWHERE, stepK = (uint32_t)(TC::STEP * a.ldk * ES);
    const uint32_t offV = in ? (uint32_t)(TC::row0() * a.ldv * ES + TC::unit0()) : NOWHERE, stepV = (uint32_t)(TC::STEP * a.ldv * ES);
    auto copy = [&](int t, lds_u8* toK, lds_u8* toV, float* places) {
      const int64_t j = (int64_t)t * C::BN;
      const int rem = (int)min((int64_t)C::BN, klen - j);
      const auto bk = buffer_of(keys + j * a.ldk, (uint32_t)(rem * a.ldk * ES));
      const auto bv = buffer_of(values + j * a.ldv, (uint32_t)(rem * a.ldv * ES));
#pragma unroll
      for (int i = 0; i < TC::PER; ++i) TC::copy(bk, toK, i, offK + i * stepK), TC::copy(bv, toV, i, offV + i * stepV);
      if (dim) copy_places<C::BN>(a.pos_k, a.dim, k0 + j, rem, places);
    };
    if (dim) clear_places<C::BN>(a.dim, dim, lds.extra0), clear_places<C::BN>(a.dim, dim, lds.extra1);
    if (t_begin < t_end) copy(t_begin, (lds_u8*)lds.a0, (lds_u8*)lds.b0, lds.extra0);
    for (int t = t_begin; t < t_end; t += 2) {
      stage_wait();
      __syncthreads();   // the tile is there, and all waves have left the other buffer
      if (t + 1 < t_end) copy(t + 1, (lds_u8*)lds.a1, (lds_u8*)lds.b1, lds.extra1);
      step((lds_u8*)lds.a0, (lds_u8*)lds.b0, lds.extra0, t);
      if (t + 1 < t_end) {   // no second way out of the loop: the sums would have a second place for it
        stage_wait();
        __syncthreads();
        if (t + 2 < t_end) copy(t + 2, (lds_u8*)lds.a0, (lds_u8*)lds.b0, lds.extra0);
        step((lds_u8*)lds.a1, (lds_u8*)lds.b1, lds.extra1, t + 1);
      }
    }
  } else {
    const int row0 = tid / (D * ES / 16), c0 = tid % (D * ES / 16) * 16;
    const bool in = c0 < a.hd * ES;
    const uint32_t offK = in ? (uint32_t)(row0 * a.ldk * ES + c0) : NOWHERE, stepK = (uint32_t)(C::STEP * a.ldk * ES);
    const uint32_t offV = in ? (uint32_t)(row0 * a.ldv * ES + c0) : NOWHERE, stepV = (uint32_t)(C::STEP * a.ldv * ES);
    u32x4 regK[C::HELD], regV[C::HELD];
    Place key{0.0f, 0.0f, 0.0f};
    auto fetch = [&](int t, int i0) {
      const int64_t j = (int64_t)t * C::BN;
      const int rem = (int)min((int64_t)C::BN, klen - j);
      const auto bk = buffer_of(keys + j * a.ldk, (uint32_t)(rem * a.ldk * ES));
      const auto bv = buffer_of(values + j * a.ldv, (uint32_t)(rem * a.ldv * ES));
#pragma unroll
      for (int i = 0; i < C::HELD; ++i)
        regK[i] = buffer_read(bk, offK + (i0 + i) * stepK), regV[i] = buffer_read(bv, offV + (i0 + i) * stepV);
      if (dim && a.dim && i0 == 0 && tid < rem) key = place_of(a.pos_k, a.dim, k0 + j + tid);
    };
    auto put = [&](int i0) {
#pragma unroll
      for (int i = 0; i < C::HELD; ++i) {
        const int at = (row0 + (i0 + i) * C::STEP) * C::PITCH + c0;
        *(lds_u32x4*)((lds_u8*)lds.a0 + at) = regK[i];
        *(lds_u32x4*)((lds_u8*)lds.b0 + at) = regV[i];
      }
      float* places = lds.extra0;
      if (dim && i0 == 0 && tid < C::BN) places[tid] = key.x, places[C::BN + tid] = key.y, places[2 * C::BN + tid] = key.z;
    };
    if (C::AHEAD && t_begin < t_end) fetch(t_begin, 0);
    for (int t = t_begin; t < t_end; ++t) {
      __syncthreads();
      if (C::AHEAD) {
        put(0);
      } else {
#pragma unroll 1
        for (int i0 = 0; i0 < C::PER; i0 += C::HELD) fetch(t, i0), put(i0);
      }
      __syncthreads();
      if (C::AHEAD && t + 1 < t_end) fetch(t + 1, 0);
      step((lds_u8*)lds.a0, (lds_u8*)lds.b0, lds.extra0, t);
    }
  }

  int again = tid;   // the row once more: formed here, not kept in registers over the loop
  asm volatile("" : "+v"(again));
  const RowOf mine = row_of(a, q0, r0, R, kvh, FEW, again);
  T* out = (T*)a.gq + mine.query * a.ldgq + mine.head * a.hd;
  float* part = a.splits > 1 ? a.part + ((int64_t)split * a.nq * a.H + mine.query * a.H + mine.head) * a.hd : nullptr;
  if (FEW) join_rows<T, D>(acc, lds, a.scale, out, part, a.hd, mine.there);
  else if (mine.there) write_rows<T, D>(acc, a.scale, out, part, a.hd);
}

// PAIRED: an even number of heads share their keys, so that rows two by two have the same query, and the
// same distance.
template <typename T, int D, bool FEW, bool PAIRED, typename M>
__device__ __forceinline__ void dkv_tile(const AttnArgs& a, const BwdLds& lds, unsigned group) {
  using C = Bwd<T, D, FEW, true>;
  constexpr int ES = sizeof(T), KS = D / 16, DB = D / 32, UNITS = D * ES / 16;
  typedef typename Frag<T>::type frag;

  const int tid = (int)threadIdx.x, l = tid & 63, h = l >> 5, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = (int)(group % (unsigned)a.Hk);
  const unsigned rest = group / (unsigned)a.Hk;
  const int split = (int)(rest % (unsigned)a.splits_k);
  const int64_t tile = rest / (unsigned)a.splits_k;
  int64_t first;
  const int seg = FEW ? find_segment(a.kb, a.n_seg, 1, C::OWN, tile, &first)
                      : find_segment_longest_first(a.kb, a.qb, a.n_seg, 1, C::OWN, tile, &first);
  const int64_t k0 = a.kb.at(seg), klen = a.kb.at(seg + 1) - k0, j0 = (tile - first) * C::OWN;
  if (tile < first || j0 >= klen) return;
  const int64_t q0 = a.qb.at(seg), queries = a.qb.at(seg + 1) - q0, R = queries > 0 ? queries * a.G : 0;
  const int tiles = (int)((R + C::BN - 1) / C::BN);
  const int per = (tiles + a.splits_k - 1) / a.splits_k;
  const int t_begin = min(split * per, tiles), t_end = min(t_begin + per, tiles);

  const bool cap = M::cap(a);
  const int dim = M::dim(a);
  const Score<T, false> sc(a, cap);
  frag kf[KS], vf[KS];
  Place me{0.0f, 0.0f, 0.0f};
  {
    const int64_t j = j0 + (FEW ? 0 : 32 * w) + (l & 31);
    const bool there = j < klen;
    const int64_t key = k0 + (there ? j : 0);
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      const int c = 16 * t + 8 * h;
      kf[t] = read_frag<T>((const T*)a.k + key * a.ldk + kvh * a.hd + c, there && c < a.hd);
      vf[t] = read_frag<T>((const T*)a.v + key * a.ldv + kvh * a.hd + c, there && c < a.hd);
    }
    apply_sign<KS>(kf, sc.sign);
    if (dim && a.dim && there) me = place_of(a.pos_k, a.dim, key);
  }

  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) dk[d] = f32x16{}, dv[d] = f32x16{};

  const LanePlace place = lane_place<D>();
  // rows: shift, -D, slope, x, y, z of the tile's rows
  auto step = [&](lds_u8* ldsQ, lds_u8* ldsG, const float* rows, int t) {
    if (FEW && (int64_t)t * C::BN + 32 * w >= R) return;
    LanePlace lane = place;
    formed_here(lane);
#pragma unroll
    for (int b = 0; b < C::SUB; ++b) {
      const int at = 32 * ((FEW ? w : 0) + b);
      f32x16 x{}, dp;
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const float4 d = *(const float4*)(rows + C::BN + at + 8 * i4 + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) dp[4 * i4 + e] = (&d.x)[e];
      }
      frag rq[2], rg[2];
      rq[0] = tile_rows<T, D>(ldsQ, lane, at, 0), rg[0] = tile_rows<T, D>(ldsG, lane, at, 0);
#pragma unroll
      for (int t2 = 0; t2 < KS; ++t2) {
        if (ES == 4 && D == 128 && t2 > 0) rq[t2 & 1] = tile_rows<T, D>(ldsQ, lane, at, t2), rg[t2 & 1] = tile_rows<T, D>(ldsG, lane, at, t2);
        if (!(ES == 4 && D == 128) && t2 + 1 < KS)
          rq[(t2 + 1) & 1] = tile_rows<T, D>(ldsQ, lane, at, t2 + 1), rg[(t2 + 1) & 1] = tile_rows<T, D>(ldsG, lane, at, t2 + 1);
        x = mma(rq[t2 & 1], kf[t2], x);
        dp = mma(rg[t2 & 1], vf[t2], dp);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const float* row = rows + at + 8 * i4 + 4 * h;
        float4 far{};
        if (dim) {
          const float4 px = *(const float4*)(row + 3 * C::BN), py = *(const float4*)(row + 4 * C::BN);
          float4 pz{};
          if (dim > 2) pz = *(const float4*)(row + 5 * C::BN);
          far.x = distance(dim, me, px.x, py.x, pz.x), far.z = distance(dim, me, px.z, py.z, pz.z);
          far.y = far.x, far.w = far.z;
          if (!PAIRED) far.y = distance(dim, me, px.y, py.y, pz.y), far.w = distance(dim, me, px.w, py.w, pz.w);
          __builtin_amdgcn_sched_barrier(0);   // not all of a row's numbers in registers at once
        }
        const float4 shift = *(const float4*)row;
        float4 sl{};
        if (dim) sl = *(const float4*)(row + 2 * C::BN);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 4 * i4 + e;
          float fall;
          float u = sc.template u<true>(x[i], cap, &fall);
          if (dim) u = fmaf(-(&sl.x)[e], (&far.x)[e], u);
          x[i] = exp2_of(fmaf(u, sc.A, (&shift.x)[e]));
          if constexpr (FEW && C::DMA)
            if (klen <= 32) dp[i] -= sum_of_half((l & 31) < klen ? x[i] * dp[i] : 0.0f);
          dp[i] *= x[i];
          if (cap) dp[i] *= fall;
        }
        if (dim || i4 == 1) __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_sched_barrier(0);
      // the products for dv and dk in turn, fragments one ahead (none in float32, whose are large and products long)
      frag cf[2], pf{}, sf{}, rest[4]{};
      auto columns = [&](int n) {
        return tile_columns<T, D>(n & 1 ? ldsQ : ldsG, lane, at + 16 * (n / 2 / DB), 32 * (n / 2 % DB));
      };
      cf[0] = columns(0);
#pragma unroll
      for (int n = 0; n < 4 * DB; ++n) {
        const int t2 = n / 2 / DB, d = n / 2 % DB;
        if (d == 0 && n % 2 == 0) {
          float p[8], ds[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) p[i] = x[8 * t2 + i], ds[i] = dp[8 * t2 + i];
          pf = to_frag<T>(p), sf = to_frag<T>(ds);
          if constexpr (FEW && C::DMA) rest[2 * t2] = rest_frag(p, pf), rest[2 * t2 + 1] = rest_frag(ds, sf);
        }
        if (ES == 4 && n > 0) cf[n & 1] = columns(n);
        if (ES != 4 && n + 1 < 4 * DB) cf[(n + 1) & 1] = columns(n + 1);
        if (n & 1) dk[d] = mma(cf[n & 1], sf, dk[d]);
        else dv[d] = mma(cf[n & 1], pf, dv[d]);
        if (n & 1) __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (FEW && C::DMA)
        if (a.fine) {
#pragma unroll
          for (int n = 0; n < 4 * DB; ++n) {
            const int d = n / 2 % DB;
            const frag f = columns(n);
            if (n & 1) dk[d] = mma(f, rest[2 * (n / 2 / DB) + 1], dk[d]);
            else dv[d] = mma(f, rest[2 * (n / 2 / DB)], dv[d]);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
    }
#pragma unroll
    for (int d = 0; d < DB; ++d)
      if (D <= 64) asm volatile("" : "+v"(dk[d]), "+v"(dv[d]));   // one place for the sums after either buffer's tile
  };

  // what belongs to a row, one row to a thread: the shift is formed here (FEW) or was by the launch for the
  // queries, and so was -D, but for FEW, which forms it from its rows' units.  A row behind the last has zeros: its
  // weights, whatever they are, meet gradients of 0.
  float rl = 0.0f, rd = 0.0f, rs = 0.0f;
  Place rp{0.0f, 0.0f, 0.0f};
  // a tile's first query, the head that it begins with, and the queries from it on
  struct First {
    int64_t at, left;
    unsigned head;
  };
  auto first_of = [&](int t) {
    const unsigned base = (unsigned)t * C::BN, f = base / (unsigned)a.G;
    return First{q0 + f, queries - f, base - f * (unsigned)a.G};
  };
  auto fetch_row = [&](const First& f) {
    if (tid >= C::BN) return;
    const uint32_t x = f.head + tid, qi = (x * a.g_inv) >> 20, g = x - qi * a.G;
    rl = rd = rs = 0.0f, rp = Place{0.0f, 0.0f, 0.0f};
    if ((int64_t)qi < f.left) {
      const int64_t query = f.at + qi, slot = query * a.H + kvh * a.G + g;
      if (FEW) {
        const float lse = a.lse_in[slot];
        rl = lse == -INFINITY ? -INFINITY : sc.C - lse * LOG2E;
      } else if (!C::DMA) {
        rl = a.shift[slot], rd = a.minus_d[slot];
      }
      if (dim && a.dim) rp = place_of(a.pos_q, a.dim, query), rs = a.slopes[kvh * a.G + g] * sc.per_slope;
    }
  };
  auto put_row = [&](float* rows) {
    if (tid >= C::BN) return;
    if (FEW || !C::DMA) rows[tid] = rl;
    if (!FEW && !C::DMA) rows[C::BN + tid] = rd;
    if (dim) rows[2 * C::BN + tid] = rs, rows[3 * C::BN + tid] = rp.x, rows[4 * C::BN + tid] = rp.y, rows[5 * C::BN + tid] = rp.z;
  };
  // FEW: dO . o of the tile's rows, from the units of a row, which are a row of lanes
  typedef T unit __attribute__((ext_vector_type(16 / ES)));
  auto dot_of = [&](const u32x4& g, const u32x4& o) {
    const unit gv = __builtin_bit_cast(unit, g), ov = __builtin_bit_cast(unit, o);
    float d = 0.0f;
#pragma unroll
    for (int e = 0; e < 16 / ES; ++e) d = fmaf((float)gv[e], (float)ov[e], d);
#pragma unroll
    for (int o2 = 1; o2 < UNITS; o2 <<= 1) d += __shfl_xor(d, o2, 64);
    return d;
  };
  const int64_t side = (int64_t)kvh * a.G * a.hd;
  // where a row's unit is, from the tile's first query on
  auto offset_of = [&](const First& f, int rem, int row, int byte, bool in, int64_t ld) {
    const uint32_t x = f.head + row, qi = (x * a.g_inv) >> 20, g = x - qi * a.G;
    return in && (int)qi < rem ? qi * (uint32_t)(ld * ES) + g * (uint32_t)(a.hd * ES) + byte : NOWHERE;
  };
  if constexpr (C::DMA) {
    using TC = TileCopy<D, C::BN>;
    constexpr int DOTS = FEW ? TC::PER : 1;
    const int row0 = TC::row0(), byte = TC::unit0();
    const bool in = byte < a.hd * ES;
    u32x4 regG[DOTS], regO[DOTS];
    auto copy = [&](int t, lds_u8* toQ, lds_u8* toG, float* rows) {
      const First f = first_of(t);
      const int rem = (int)min((int64_t)C::BN + 1, f.left);
      const auto bq = buffer_of((const T*)a.q + f.at * a.ldq + side, (uint32_t)(rem * a.ldq * ES));
      const auto bg = buffer_of((const T*)a.go + f.at * a.ldgo + side, (uint32_t)(rem * a.ldgo * ES));
#pragma unroll
      for (int i = 0; i < TC::PER; ++i) {
        TC::copy(bq, toQ, i, offset_of(f, rem, row0 + i * TC::STEP, byte, in, a.ldq));
        TC::copy(bg, toG, i, offset_of(f, rem, row0 + i * TC::STEP, byte, in, a.ldgo));
      }
      if (FEW) {
        const auto bo = buffer_of((const T*)a.o + f.at * a.ldo + side, (uint32_t)(rem * a.ldo * ES));
#pragma unroll
        for (int i = 0; i < DOTS; ++i) {
          regG[i] = buffer_read(bg, offset_of(f, rem, row0 + i * TC::STEP, byte, in, a.ldgo));
          regO[i] = buffer_read(bo, offset_of(f, rem, row0 + i * TC::STEP, byte, in, a.ldo));
        }
      }
      if (!FEW && w < 2) {   // a wave for the shifts, one for -D
        static_assert(FEW || C::BN == 64, "a row to a lane");
        const auto from = buffer_of((w ? a.minus_d : a.shift) + f.at * a.H, (uint32_t)(rem * a.H * 4));
        const uint32_t x = f.head + l, qi = (x * a.g_inv) >> 20, g = x - qi * a.G;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(lds_u8*)(rows + w * C::BN), 4,
                                                 (int)((int)qi < rem ? (qi * a.H + kvh * a.G + g) * 4 : NOWHERE), 0, 0, 0);
      }
      if (FEW || dim) fetch_row(f);
    };
    auto put = [&](float* rows) {
      put_row(rows);
      if (FEW) {
#pragma unroll
        for (int i = 0; i < DOTS; ++i) {
          const float d = dot_of(regG[i], regO[i]);
          if (tid % UNITS == 0) rows[C::BN + row0 + i * TC::STEP] = -d;
        }
      }
    };
    if (t_begin < t_end) copy(t_begin, (lds_u8*)lds.a0, (lds_u8*)lds.b0, lds.extra0), put(lds.extra0);
    for (int t = t_begin; t < t_end; t += 2) {
      stage_wait();
      __syncthreads();   // the tile is there, and all waves have left the other buffer
      if (t + 1 < t_end) copy(t + 1, (lds_u8*)lds.a1, (lds_u8*)lds.b1, lds.extra1);
      step((lds_u8*)lds.a0, (lds_u8*)lds.b0, lds.extra0, t);
      if (t + 1 < t_end) {   // no second way out of the loop: the sums would have a second place for it
        put(lds.extra1);
        stage_wait();
        __syncthreads();
        if (t + 2 < t_end) copy(t + 2, (lds_u8*)lds.a0, (lds_u8*)lds.b0, lds.extra0);
        step((lds_u8*)lds.a1, (lds_u8*)lds.b1, lds.extra1, t + 1);
        if (t + 2 < t_end) put(lds.extra0);
      }
    }
  } else {
    const int row0 = tid / UNITS, c0 = tid % UNITS * 16;
    const bool in = c0 < a.hd * ES;
    u32x4 regQ[C::HELD], regG[C::HELD];
    float dots[C::HELD];
    auto fetch = [&](int t, int i0) {
      const First f = first_of(t);
      const int rem = (int)min((int64_t)C::BN + 1, f.left);
      const auto bq = buffer_of((const T*)a.q + f.at * a.ldq + side, (uint32_t)(rem * a.ldq * ES));
      const auto bg = buffer_of((const T*)a.go + f.at * a.ldgo + side, (uint32_t)(rem * a.ldgo * ES));
      const auto bo = buffer_of((const T*)a.o + f.at * a.ldo + side, (uint32_t)(rem * a.ldo * ES));
#pragma unroll
      for (int i = 0; i < C::HELD; ++i) {
        const int row = row0 + (i0 + i) * C::STEP;
        regQ[i] = buffer_read(bq, offset_of(f, rem, row, c0, in, a.ldq));
        regG[i] = buffer_read(bg, offset_of(f, rem, row, c0, in, a.ldgo));
        if (FEW) dots[i] = dot_of(regG[i], buffer_read(bo, offset_of(f, rem, row, c0, in, a.ldo)));
      }
      if (i0 == 0) fetch_row(f);
    };
    auto put = [&](int i0) {
#pragma unroll
      for (int i = 0; i < C::HELD; ++i) {
        const int row = row0 + (i0 + i) * C::STEP;
        *(lds_u32x4*)((lds_u8*)lds.a0 + row * C::PITCH + c0) = regQ[i];
        *(lds_u32x4*)((lds_u8*)lds.b0 + row * C::PITCH + c0) = regG[i];
        if (FEW && c0 == 0) lds.extra0[C::BN + row] = -dots[i];
      }
      if (i0 == 0) put_row(lds.extra0);
    };
    if (C::AHEAD && t_begin < t_end) fetch(t_begin, 0);
    for (int t = t_begin; t < t_end; ++t) {
      __syncthreads();
      if (C::AHEAD) {
        put(0);
      } else {
#pragma unroll 1
        for (int i0 = 0; i0 < C::PER; i0 += C::HELD) fetch(t, i0), put(i0);
      }
      __syncthreads();
      if (C::AHEAD && t + 1 < t_end) fetch(t + 1, 0);
      step((lds_u8*)lds.a0, (lds_u8*)lds.b0, lds.extra0, t);
    }
  }

  int again = tid;   // the lane's key once more: formed here, not kept in registers over the loop
  asm volatile("" : "+v"(again));
  const int64_t j = j0 + (FEW ? again & 31 : 32 * (again >> 6) + (again & 31)), key = k0 + j;
  const bool there = j < klen;
  T* gk = (T*)a.gk + key * a.ldgk + kvh * a.hd;
  T* gv = (T*)a.gv + key * a.ldgv + kvh * a.hd;
  const int64_t at = (((int64_t)split * a.nk + key) * a.Hk + kvh) * a.hd;
  float *pk = a.splits_k > 1 ? a.part_k + at : nullptr, *pv = a.splits_k > 1 ? a.part_v + at : nullptr;
  if (FEW) {
    join_rows<T, D>(dk, lds, a.scale, gk, pk, a.hd, there);
    join_rows<T, D>(dv, lds, 1.0f, gv, pv, a.hd, there);
  } else if (there) {
    write_rows<T, D>(dk, a.scale, gk, pk, a.hd);
    write_rows<T, D>(dv, 1.0f, gv, pv, a.hd);
  }
}

}  // namespace dsmp
