// Attention within packed segments, forward, and the argument checks of both passes.
//
//   z_ij = c(scale q_i.k_j) - slope |p_i - p_j|,  out_i = sum_j e^(z_ij - m_i) v_j / l_i
//   m_i = max_j z_ij, l_i = sum_j e^(z_ij - m_i), lse_i = m_i + log l_i
//
// One pass over the keys with the running maximum m and sum l of each row.  The rows
// of a key head are its segment's queries times the G query heads that share it (row
// = query G + head), so one query with eight heads fills eight rows and reads the keys once.
#include "attention.hpp"

using namespace dsmp;

namespace {

constexpr int NT = 256, NW = 4;   // threads and waves of a workgroup

// WIDE: 32 rows to a wave, 128 to a workgroup, every wave takes every key of a tile.
// FEW: all waves have the same 32 rows and a quarter of a tile's keys each; they are joined at the end.
// bfloat16 tiles are copied into two buffers in turn, one barrier to a tile; float32 ones wait in registers.
template <typename T, int D, bool FEW>
struct Fwd {
  static constexpr bool DMA = sizeof(T) == 2;
  static constexpr int ROWS = FEW ? FEW_ROWS : WIDE_ROWS;
  static constexpr int BN = FEW ? 32 * NW : DMA ? 64 : 32;
  static constexpr int SUB = FEW ? 1 : BN / 32;   // blocks of 32 keys that a wave takes of a tile
  static constexpr int PITCH = DMA ? 2 * D : pitch_of<T, D, true>(), MATRIX = BN * PITCH, PLACES = 3 * BN;
  // float32: 16-byte units to a thread; the next tile waits in registers, but for FEW's large ones: those come four at a time
  static constexpr int PER = BN * D * (int)sizeof(T) / 16 / NT, STEP = NT * 16 / (D * (int)sizeof(T));
  static constexpr bool AHEAD = !(FEW && D == 128);
  static constexpr int HELD = AHEAD || PER < 4 ? PER : 4;
  static_assert(FEW_ROWS == 32 && WIDE_ROWS == 32 * NW, "32 rows to a wave");
  static_assert(!FEW || MATRIX >= 2 * 32 * D * 4, "two waves' parts fit into a matrix");
  static_assert(PER >= 1 && PER * NT * 16 == BN * D * (int)sizeof(T), "whole units for every thread");
  // waves to a SIMD that the registers are cut to
  template <typename M>
  static constexpr int WAVES = D == 128 ? (FEW || !DMA ? 1 : 2) : FEW || !DMA ? 2 : D == 64 && M::DIM > 0 ? 3 : 4;
};

// How far the scores of a tile may pass the maximum that a row's sums refer to, in powers of two,
// before the sums are brought to a new one: weights then reach 2^8, which costs neither
// float32 sums nor the rounded weights a digit.
constexpr float SLACK = 8.0f;

template <typename T, int D, bool FEW, typename M>
__global__ __launch_bounds__(NT, (Fwd<T, D, FEW>::template WAVES<M>)) void k_attn_fwd(AttnArgs a) {
  using C = Fwd<T, D, FEW>;
  constexpr int ES = sizeof(T), KS = D / 16, DB = D / 32;
  typedef typename Frag<T>::type frag;
  // the buffers are arrays of their own, so that a copy into one is not waited for by reads of the other
  __shared__ __align__(1024) unsigned char mK0[C::MATRIX], mV0[C::MATRIX], mK1[C::DMA ? C::MATRIX : 16], mV1[C::DMA ? C::MATRIX : 16];
  __shared__ __align__(16) float mP0[C::PLACES], mP1[C::DMA ? C::PLACES : 4];

  const int tid = (int)threadIdx.x, l = tid & 63, h = l >> 5, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = (int)(blockIdx.x % (unsigned)a.Hk);
  const unsigned rest = blockIdx.x / (unsigned)a.Hk;
  const int split = (int)(rest % (unsigned)a.splits);
  const int64_t tile = rest / (unsigned)a.splits;
  int64_t first;
  const int seg = FEW ? find_segment(a.qb, a.n_seg, a.G, C::ROWS, tile, &first)
                      : find_segment_longest_first(a.qb, a.kb, a.n_seg, a.G, C::ROWS, tile, &first);
  const int64_t q0 = a.qb.at(seg), R = (a.qb.at(seg + 1) - q0) * a.G, r0 = (tile - first) * C::ROWS;
  if (tile < first || r0 >= R) return;
  const int64_t k0 = a.kb.at(seg), klen = a.kb.at(seg + 1) - k0;
  const int tiles = klen > 0 ? (int)((klen + C::BN - 1) / C::BN) : 0;
  const int per = (tiles + a.splits - 1) / a.splits;
  const int t_begin = min(split * per, tiles), t_end = min(t_begin + per, tiles);

  // this lane's row
  const bool cap = M::cap(a);
  const int dim = M::dim(a);
  const Score<T, FEW> sc(a, cap);
  const RowOf row = row_of(a, q0, r0, R, kvh, FEW, tid);
  const bool there = row.there;
  const int64_t query = row.query;
  const int head = row.head;
  frag qf[KS];
#pragma unroll
  for (int t = 0; t < KS; ++t) {
    qf[t] = read_frag<T>((const T*)a.q + query * a.ldq + head * a.hd + 16 * t + 8 * h, there && 16 * t + 8 * h < a.hd);
  }
  apply_sign<KS>(qf, sc.sign);
  Place me{0.0f, 0.0f, 0.0f};
  float slope = 0.0f;
  if (dim && a.dim && there) me = place_of(a.pos_q, a.dim, query), slope = a.slopes[head] * sc.per_slope;

  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
  float m = -INFINITY, sum = 0.0f;   // the u that this lane's row refers to; the sum over this half's keys

  const LanePlace place = lane_place<D>();
  // one tile: scores, then weights and their products with the values
  auto step = [&](lds_u8* ldsK, lds_u8* ldsV, const float* places, int t) {
    const int rem = (int)min((int64_t)C::BN, klen - (int64_t)t * C::BN);
    if (FEW && 32 * w >= rem) return;
    const int sub0 = FEW ? w : 0;
    LanePlace lane = place;
    formed_here(lane);
    // Fragments are read one step ahead of their products and no further (the scheduler would
    // read all of them at once and run out of registers); the products run while the
    // next step's powers are formed.
    f32x16 x[C::SUB];
    frag kf[2][C::SUB];
#pragma unroll
    for (int b = 0; b < C::SUB; ++b) kf[0][b] = tile_rows<T, D>(ldsK, lane, 32 * (sub0 + b), 0), x[b] = f32x16{};
#pragma unroll
    for (int t2 = 0; t2 < KS; ++t2) {
#pragma unroll
      for (int b = 0; b < C::SUB; ++b)
        if (t2 + 1 < KS) kf[(t2 + 1) & 1][b] = tile_rows<T, D>(ldsK, lane, 32 * (sub0 + b), t2 + 1);
#pragma unroll
      for (int b = 0; b < C::SUB; ++b) x[b] = mma(kf[t2 & 1][b], qf[t2], x[b]);
      __builtin_amdgcn_sched_barrier(0);
    }
    float top = -INFINITY;
#pragma unroll
    for (int b = 0; b < C::SUB; ++b) {
      const int at = 32 * (sub0 + b);
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
          float u = sc.template u<false>(x[b][i], cap, nullptr);
          if (dim) u = fmaf(-slope, distance(dim, me, (&px.x)[e], (&py.x)[e], (&pz.x)[e]), u);
          x[b][i] = u;
        }
      }
      if (at + 32 > rem) {   // behind the last key
        int left = rem - at - 4 * h;
        asm volatile("" : "+v"(left));   // compared with constants, not with sixteen row numbers kept over the loop
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (8 * (i >> 2) + (i & 3) >= left) x[b][i] = -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, x[b][i]);
      if (dim) __builtin_amdgcn_sched_barrier(0);
    }
    frag vf[2][DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) vf[0][d] = tile_columns<T, D>(ldsV, lane, 32 * sub0, 32 * d);
    top = fmaxf(top, other_half(top));
    if (__any((top - m) * sc.A > SLACK)) {   // also where m is -infinity
      const float now = fmaxf(m, top), shrink = m == -INFINITY ? 0.0f : exp2_of((m - now) * sc.A);
      m = now;
      sum *= shrink;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= shrink;
    }
    const float base = m == -INFINITY ? 0.0f : -m * sc.A;
    float add = 0.0f;
#pragma unroll
    for (int k = 0; k < 2 * C::SUB; ++k) {
      const int b = k >> 1, t2 = k & 1;
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = exp2_of(fmaf(x[b][8 * t2 + i], sc.A, base)), add += p[i];
      const frag pf = to_frag<T>(p);
#pragma unroll
      for (int d = 0; d < DB; ++d)
        if (k + 1 < 2 * C::SUB) vf[(k + 1) & 1][d] = tile_columns<T, D>(ldsV, lane, 32 * sub0 + 16 * (k + 1), 32 * d);
#pragma unroll
      for (int d = 0; d < DB; ++d) o[d] = mma(vf[k & 1][d], pf, o[d]);
      if constexpr (FEW && C::DMA)
        if (a.fine) {
          const frag rest = rest_frag(p, pf);
#pragma unroll
          for (int d = 0; d < DB; ++d) o[d] = mma(vf[k & 1][d], rest, o[d]);
        }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int d = 0; d < DB; ++d)
      if (C::template WAVES<M> > 1) asm volatile("" : "+v"(o[d]));   // one place for the sums after either buffer's tile
    sum += add;
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
    if (dim) clear_places<C::BN>(a.dim, dim, mP0), clear_places<C::BN>(a.dim, dim, mP1);
    if (t_begin < t_end) copy(t_begin, (lds_u8*)mK0, (lds_u8*)mV0, mP0);
    for (int t = t_begin; t < t_end; t += 2) {
      stage_wait();
      __syncthreads();   // the tile is there, and all waves have left the other buffer
      if (t + 1 < t_end) copy(t + 1, (lds_u8*)mK1, (lds_u8*)mV1, mP1);
      step((lds_u8*)mK0, (lds_u8*)mV0, mP0, t);
      if (t + 1 < t_end) {   // no second way out of the loop: the sums would have a second place for it
        stage_wait();
        __syncthreads();
        if (t + 2 < t_end) copy(t + 2, (lds_u8*)mK0, (lds_u8*)mV0, mP0);
        step((lds_u8*)mK1, (lds_u8*)mV1, mP1, t + 1);
      }
    }
  } else {
    // a thread's 16-byte units of a tile: one place in every STEP-th row
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
        *(lds_u32x4*)((lds_u8*)mK0 + at) = regK[i];
        *(lds_u32x4*)((lds_u8*)mV0 + at) = regV[i];
      }
      if (dim && i0 == 0 && tid < C::BN) mP0[tid] = key.x, mP0[C::BN + tid] = key.y, mP0[2 * C::BN + tid] = key.z;
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
      step((lds_u8*)mK0, (lds_u8*)mV0, mP0, t);
    }
  }
  sum += other_half(sum);

  int again = tid;   // the row once more: formed here, not kept in registers over the loop
  asm volatile("" : "+v"(again));
  const RowOf mine = row_of(a, q0, r0, R, kvh, FEW, again);
  const int64_t slot = mine.query * a.H + mine.head;   // this row's among all queries and heads
  const int64_t part = (int64_t)split * a.nq * a.H + slot;
  float* const ml = a.part + (int64_t)a.splits * a.nq * a.H * a.hd + 2 * part;
  if (!FEW) {
    if (!mine.there) return;
    if (a.splits > 1) {
      if (h == 0) ml[0] = fmaf(m, sc.A, sc.C), ml[1] = sum;
      write_rows<T, D>(o, 1.0f, (T*)nullptr, a.part + part * a.hd, a.hd);
      return;
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    if (a.lse && h == 0) a.lse[slot] = (fmaf(m, sc.A, sc.C) + __log2f(sum)) * LN2;
    write_rows<T, D>(o, inv, (T*)a.out + mine.query * a.ldout + mine.head * a.hd, nullptr, a.hd);
    return;
  }
  // the waves' parts, [value][row], two in each of a buffer's matrices, joined by 256 threads: a row and
  // four values in 32 each
  m = fmaf(m, sc.A, sc.C);   // in powers of two from here on
  float *jm = mP0, *js = mP0 + NW * 32;
  auto part_of = [&](int wave) { return (float*)(wave < 2 ? mK0 : mV0) + (wave & 1) * 32 * D; };
  __syncthreads();
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) part_of(w)[(32 * d + result_row(i)) * 32 + (l & 31)] = o[d][i];
  if (h == 0) jm[w * 32 + l] = m, js[w * 32 + l] = sum;
  __syncthreads();
  if (!mine.there) return;
  float top = -INFINITY, weight[NW], total = 0.0f;
#pragma unroll
  for (int k = 0; k < NW; ++k) top = fmaxf(top, jm[k * 32 + (l & 31)]);
#pragma unroll
  for (int k = 0; k < NW; ++k) {
    weight[k] = exp2_of(jm[k * 32 + (l & 31)] - (top == -INFINITY ? 0.0f : top));
    total = fmaf(weight[k], js[k * 32 + (l & 31)], total);
  }
  const int g4 = 4 * (tid >> 5);
  const bool whole = a.splits == 1;
  const float inv = !whole ? 1.0f : total == 0.0f ? 0.0f : 1.0f / total;
  if (tid < 32) {
    if (!whole) {
      ml[0] = top, ml[1] = total;
    } else if (a.lse) {
      a.lse[slot] = (top + __log2f(total)) * LN2;
    }
  }
#pragma unroll
  for (int d = 0; d < DB; ++d) {
    const int c = 32 * d + g4;
    if (c >= a.hd) continue;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = 0.0f;
#pragma unroll
      for (int k = 0; k < NW; ++k) v[e] = fmaf(weight[k], part_of(k)[(c + e) * 32 + (l & 31)], v[e]);
      v[e] *= inv;
    }
    if (whole) store4((T*)a.out + mine.query * a.ldout + mine.head * a.hd + c, v[0], v[1], v[2], v[3]);
    else *(float4*)(a.part + part * a.hd + c) = make_float4(v[0], v[1], v[2], v[3]);
  }
}

// The splits of a query's head, joined in their order.  A split without keys (of a segment with fewer tiles than
// splits) has the sum 0 and zeros for values, which have no part in the result.  FEW_SPLITS: 32 lanes to each; otherwise a workgroup of 1,024, whose
// 32 slices of the splits are added up.

__device__ __forceinline__ bool in_segments(const AttnArgs& a, int64_t query) {
  return query >= a.qb.at(0) && query < a.qb.at(a.n_seg);
}

template <typename T>
__device__ __forceinline__ void write_joined(const AttnArgs& a, int64_t slot, int64_t query, int c, const float* v, float top,
                                             float total) {
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
  if (c < a.hd)
    store4((T*)a.out + query * a.ldout + (slot - query * a.H) * a.hd + c, v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
  if (c == 0 && a.lse) a.lse[slot] = (top + __log2f(total)) * LN2;
}

template <typename T>
__global__ __launch_bounds__(NT) void k_attn_join_few(AttnArgs a) {
  const int64_t all = a.nq * a.H, slot = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (slot >= all) return;
  const int64_t query = slot / a.H;
  if (!in_segments(a, query)) return;
  const float2* ml = (const float2*)(a.part + (int64_t)a.splits * all * a.hd);
  const int c = 4 * ((int)threadIdx.x & 31);
  float2 x[FEW_SPLITS];
  float4 p[FEW_SPLITS];
  float top = -INFINITY;
#pragma unroll
  for (int s = 0; s < FEW_SPLITS; ++s) x[s] = s < a.splits ? ml[s * all + slot] : make_float2(-INFINITY, 0.0f);
#pragma unroll
  for (int s = 0; s < FEW_SPLITS; ++s)
    if (s < a.splits && c < a.hd) p[s] = *(const float4*)(a.part + (s * all + slot) * a.hd + c);
#pragma unroll
  for (int s = 0; s < FEW_SPLITS; ++s) top = fmaxf(top, x[s].x);
  const float base = top == -INFINITY ? 0.0f : top;
  float total = 0.0f, v[4] = {};
#pragma unroll
  for (int s = 0; s < FEW_SPLITS; ++s) {
    if (s >= a.splits || x[s].y == 0.0f) continue;
    const float weight = exp2_of(x[s].x - base);
    total = fmaf(weight, x[s].y, total);
    if (c < a.hd) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(weight, (&p[s].x)[e], v[e]);
    }
  }
  write_joined<T>(a, slot, query, c, v, top, total);
}

template <typename T>
__global__ __launch_bounds__(1024) void k_attn_join(AttnArgs a) {
  __shared__ float red[32][MAX_HEAD_DIM + 4];
  __shared__ float weight[MAX_SPLITS];
  __shared__ float wave[2][16];
  const int64_t slot = blockIdx.x, query = slot / a.H, all = a.nq * a.H;
  if (!in_segments(a, query)) return;
  const int tid = (int)threadIdx.x, c = 4 * (tid & 31), slice = tid >> 5;
  const float2 x = tid < a.splits ? ((const float2*)(a.part + (int64_t)a.splits * all * a.hd))[tid * all + slot]
                                  : make_float2(-INFINITY, 0.0f);
  // the first parts are on their way while the weights are formed
  constexpr int AHEAD = 8;
  const float* from = a.part + slot * a.hd + c;
  const int64_t step = all * a.hd;
  float4 p[AHEAD];
#pragma unroll
  for (int k = 0; k < AHEAD; ++k)
    if (c < a.hd && slice + 32 * k < a.splits) p[k] = *(const float4*)(from + (slice + 32 * k) * step);
  float top = x.x;
  for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  if ((tid & 63) == 0) wave[0][tid >> 6] = top;
  __syncthreads();
  top = wave[0][0];
#pragma unroll
  for (int k = 1; k < 16; ++k) top = fmaxf(top, wave[0][k]);
  const float mine = x.y == 0.0f ? 0.0f : exp2_of(x.x - (top == -INFINITY ? 0.0f : top));
  weight[tid] = mine;
  float total = mine * x.y;
  for (int o = 1; o < 64; o <<= 1) total += __shfl_xor(total, o, 64);
  if ((tid & 63) == 0) wave[1][tid >> 6] = total;
  __syncthreads();
  total = 0.0f;
#pragma unroll
  for (int k = 0; k < 16; ++k) total += wave[1][k];
  float v[4] = {};
  auto add = [&](int s, const float4& q) {
    const float w = weight[s];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = w == 0.0f ? v[e] : fmaf(w, (&q.x)[e], v[e]);
  };
  if (c < a.hd) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (slice + 32 * k < a.splits) add(slice + 32 * k, p[k]);
#pragma unroll 4
    for (int s = slice + 32 * AHEAD; s < a.splits; s += 32) add(s, *(const float4*)(from + s * step));
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) red[slice][c + e] = v[e];
  __syncthreads();
  if (slice) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = 0.0f;
#pragma unroll
    for (int s = 0; s < 32; ++s) v[e] += red[s][c + e];
  }
  write_joined<T>(a, slot, query, c, v, top, total);
}

size_t fwd_bytes(const dsmp_attention_desc& d, const dsmp_segments& qs, const dsmp_segments& ks) {
  const FwdPlan p = fwd_plan(d, qs, ks);
  return p.splits == 1 ? 0 : (size_t)p.splits * qs.n * d.heads * (d.head_dim + 2) * sizeof(float);
}

}  // namespace

namespace dsmp {

dsmp_status check_attention(dsmp_handle* h, const dsmp_attention_desc* d, const dsmp_segments* qs, const dsmp_segments* ks) {
  DSMP_CHECK(h, d && qs && ks, DSMP_INVALID_ARG, "the descriptor or the segments are NULL");
  DSMP_CHECK(h, d->heads >= 1 && d->kv_heads >= 1 && d->head_dim >= 1, DSMP_INVALID_ARG, "no heads or no values in them");
  DSMP_CHECK(h, d->heads % d->kv_heads == 0, DSMP_INVALID_ARG, "kv_heads must divide heads");
  DSMP_CHECK(h, d->heads <= MAX_HEADS, DSMP_UNSUPPORTED, "more than %d heads", MAX_HEADS);
  DSMP_CHECK(h, d->head_dim % 8 == 0 && d->head_dim <= MAX_HEAD_DIM, DSMP_UNSUPPORTED,
             "head_dim must be a multiple of 8 up to %d", MAX_HEAD_DIM);
  DSMP_CHECK(h, d->dtype == DSMP_F32 || d->dtype == DSMP_BF16, DSMP_INVALID_ARG, "unknown dtype");
  DSMP_CHECK(h, d->dim >= 0 && d->dim <= 3, DSMP_INVALID_ARG, "0 to 3 coordinates");
  DSMP_CHECK(h, std::isfinite(d->scale), DSMP_INVALID_ARG, "the scale must be finite");
  DSMP_CHECK(h, std::isfinite(d->cap) && d->cap >= 0.0f, DSMP_INVALID_ARG, "the cap must be finite and not negative");
  const float least = 0x1p-60f, most = 0x1p60f;   // slopes are divided by them, and one by the other: finite in float32
  DSMP_CHECK(h, d->scale == 0.0f || (std::fabs(d->scale) >= least && std::fabs(d->scale) <= most), DSMP_UNSUPPORTED,
             "a scale must be 0 or within 2^-60 and 2^60");
  DSMP_CHECK(h, d->cap == 0.0f || (d->cap >= least && d->cap <= most), DSMP_UNSUPPORTED,
             "a cap must be 0 or within 2^-60 and 2^60");
  // tanh is within 2^-22 there (see Score): 2^-12 of a score at 2^10, an eighth of what rounds its weight
  DSMP_CHECK(h, d->dtype == DSMP_F32 || d->cap <= 1024.0f, DSMP_UNSUPPORTED, "a cap over 1024 needs float32");
  const int G = d->heads / d->kv_heads;
  for (const dsmp_segments* s : {qs, ks}) {
    DSMP_CHECK(h, s->n >= 0 && s->n_seg >= 1, DSMP_INVALID_ARG, "negative rows or no segment");
    DSMP_CHECK(h, s->n < (int64_t)1 << 31 && s->n_seg < (int64_t)1 << 24, DSMP_UNSUPPORTED,
               "2^31 rows or 2^24 segments and more");
    DSMP_CHECK(h, s->ptr || s->n % s->n_seg == 0, DSMP_INVALID_ARG, "segments without ptr must divide the rows");
    DSMP_CHECK(h, tiles_of(s->n, s->n_seg, G, 32) * d->kv_heads <= MAX_GROUPS && s->n * G < (int64_t)1 << 31,
               DSMP_UNSUPPORTED, "too many rows, segments and heads for one call");
  }
  DSMP_CHECK(h, qs->n_seg == ks->n_seg, DSMP_INVALID_ARG, "queries and keys must have the same number of segments");
  return DSMP_OK;
}

}  // namespace dsmp

extern "C" dsmp_status dsmp_attention_workspace(const dsmp_attention_desc* desc, const dsmp_segments* qs,
                                                const dsmp_segments* ks, size_t* fwd_ws_bytes, size_t* bwd_ws_bytes) {
  const dsmp_status st = check_attention(nullptr, desc, qs, ks);
  if (st != DSMP_OK) return st;
  if (!fwd_ws_bytes || !bwd_ws_bytes) return DSMP_INVALID_ARG;
  *fwd_ws_bytes = fwd_bytes(*desc, *qs, *ks);
  *bwd_ws_bytes = attention_bwd_bytes(*desc, *qs, *ks);
  return DSMP_OK;
}

extern "C" dsmp_status dsmp_attention_forward(dsmp_handle* h, const dsmp_attention_desc* desc, const dsmp_segments* qs,
                                              const dsmp_segments* ks, const void* q, int64_t ldq, const void* k,
                                              int64_t ldk, const void* v, int64_t ldv, const float* pos_q,
                                              const float* pos_k, const float* slopes, void* out, int64_t ldo,
                                              float* lse, void* ws, size_t ws_bytes) {
  if (!h) return DSMP_INVALID_ARG;
  dsmp_status st = check_attention(h, desc, qs, ks);
  if (st != DSMP_OK || qs->n == 0) return st;
  DSMP_CHECK(h, q && out && (ks->n == 0 || (k && v)), DSMP_INVALID_ARG, "a data pointer is NULL");
  DSMP_CHECK(h, desc->dim == 0 || (pos_q && slopes && (ks->n == 0 || pos_k)), DSMP_INVALID_ARG,
             "coordinates and slopes are needed");
  const int es = desc->dtype == DSMP_BF16 ? 2 : 4, wq = desc->heads * desc->head_dim, wk = desc->kv_heads * desc->head_dim;
  st = check_matrices(h, es, {{q, ldq, wq, "q"}, {k, ldk, wk, "k"}, {v, ldv, wk, "v"}, {out, ldo, wq, "out"}});
  if (st != DSMP_OK) return st;
  const size_t need = fwd_bytes(*desc, *qs, *ks);
  DSMP_CHECK(h, !need || (ws && ws_bytes >= need), DSMP_WORKSPACE_TOO_SMALL, "workspace needs %zu bytes", need);
  DSMP_CHECK(h, !need || reinterpret_cast<uintptr_t>(ws) % 16 == 0, DSMP_INVALID_ARG, "the workspace must be 16-byte aligned");
  const FwdPlan plan = fwd_plan(*desc, *qs, *ks);
  AttnArgs a = attn_args(*desc, *qs, *ks);
  a.q = q, a.ldq = ldq, a.k = k, a.ldk = ldk, a.v = v, a.ldv = ldv, a.out = out, a.ldout = ldo, a.lse = lse;
  a.pos_q = pos_q, a.pos_k = pos_k, a.slopes = slopes;
  a.splits = plan.splits, a.part = (float*)ws;
  DeviceScope dev(h);
  ProfScope prof(h, DSMP_K_ATTN_FWD);
  by_attention(*desc, [&](auto t, auto width, auto mode) {
    using T = decltype(t);
    constexpr int D = decltype(width)::value;
    using M = decltype(mode);
    if (plan.few) hipLaunchKernelGGL((k_attn_fwd<T, D, true, M>), dim3((unsigned)plan.grid), dim3(NT), 0, h->stream, a);
    else hipLaunchKernelGGL((k_attn_fwd<T, D, false, M>), dim3((unsigned)plan.grid), dim3(NT), 0, h->stream, a);
    const int64_t slots = qs->n * desc->heads;
    if (plan.splits > FEW_SPLITS)
      hipLaunchKernelGGL((k_attn_join<T>), dim3((unsigned)slots), dim3(1024), 0, h->stream, a);
    else if (plan.splits > 1)
      hipLaunchKernelGGL((k_attn_join_few<T>), dim3(ceil_div(slots, 8)), dim3(NT), 0, h->stream, a);
  });
  DSMP_LAUNCHED(h, "attention forward");
  return DSMP_OK;
}
