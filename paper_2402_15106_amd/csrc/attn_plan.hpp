// Which tiles an attention call takes, and how far they are cut over the other side: host code
// that needs no device.
#pragma once

#include "../../include/dsmpnn.h"

#include <algorithm>
#include <cmath>
#include <cstdint>

namespace dsmp {

constexpr int FEW_ROWS = 32, WIDE_ROWS = 128;   // rows (or keys) of a workgroup's tile
// parts of a forward call: up to FEW_SPLITS are joined by 32 lanes to each query's head, more by a workgroup
constexpr int FEW_SPLITS = 8, MAX_SPLITS = 1024;

inline int64_t tiles_of(int64_t n, int64_t n_seg, int M, int size) { return n * M / size + n_seg; }

constexpr int64_t MAX_GROUPS = ((int64_t)1 << 24) - 1;   // a launch has fewer than 2^32 threads

// ------------------------------------------------- which tiles, and how far they are cut
// A call takes tiles of 128 rows (WIDE) or of 32 (FEW), whichever its estimated time is shorter for, and
// either may be cut over the other side into parts that are added up afterwards.
//
// CU microseconds of a tile where the CUs are full, as measured (8,192 scores of a WIDE bfloat16 tile, 4,096 of the
// others; heads of up to 32, 64 and 128).  FEW tiles have four times the copies to LDS for a score, which
// bounds the keys' gradients: 16,384 x 8 heads of 64, two of keys, backward 3,346 us with FEW for the keys, 1,785 with
// WIDE, cut.  A distance and a cap are float32 work for each score.
enum Pass { FORWARD, GRAD_Q, GRAD_K };
inline int width_of(const dsmp_attention_desc& d) { return d.head_dim <= 32 ? 0 : d.head_dim <= 64 ? 1 : 2; }
inline double tile_us(const dsmp_attention_desc& d, Pass pass, bool wide) {
  static const double bf16[3][2][3] = {{{0.40, 0.58, 1.04}, {0.25, 0.36, 0.80}},
                                       {{0.50, 0.74, 1.40}, {0.33, 0.48, 1.20}},
                                       {{0.75, 1.04, 2.10}, {0.80, 1.26, 3.60}}};
  static const double f32[3][3] = {{1.9, 2.6, 9.0}, {2.8, 6.0, 14.0}, {3.7, 8.0, 18.0}};
  const int w = width_of(d);
  if (d.dtype == DSMP_F32) return f32[pass][w] + (d.dim ? 0.5 : 0.0) + (d.cap != 0.0f ? 0.5 : 0.0);
  const double more = (d.dim ? 0.50 : 0.0) + (d.cap != 0.0f ? 0.25 : 0.0);
  return bf16[pass][wide ? 0 : 1][w] + (wide ? more : 0.5 * more);
}
// workgroups that a CU's registers and LDS hold
inline int held(const dsmp_attention_desc& d, Pass pass, bool wide) {
  const int w = width_of(d);
  if (d.dtype == DSMP_F32) return w == 0 || (w == 1 && pass == FORWARD) ? 2 : 1;
  if (w == 2) return wide && pass != GRAD_K ? 2 : 1;
  return wide ? (w == 1 && pass == GRAD_K ? 2 : 3) : w == 1 ? 2 : 3;
}

// One or two kinds of workgroups in a launch, `groups` with `steps` tiles of `us` to go over, and the bytes
// of the parts of one split.  They are cut so that a workgroup has about the same amount of work,
// as far as the shortest estimated time asks: the work dealt to 256 CUs, which are full with `held`
// workgroups each, START for each workgroup, `end` of the longest workgroup for the uneven end (more with
// segments, whose lengths differ), and the launch that adds up the parts (5 us, and their bytes written and read at
// 4 TB/s).
struct Cut {
  int64_t groups, steps;
  double us, bytes;
  int splits;
};
inline double cut_evenly(Cut* c, int n, int held, int most, double end) {
  constexpr double CUS = 256, START = 1.2;
  double total = 0, best = 0;
  for (int i = 0; i < n; ++i) total += c[i].groups * c[i].steps * c[i].us;
  int now[2] = {1, 1};
  static const int targets[] = {0, 1, 2, 3, 4, 6, 8};   // workgroups to a CU; 0: uncut
  for (const int k : targets) {
    double sum = 0, longest = 0, join = 0;
    int64_t groups = 0;
    for (int i = 0; i < n; ++i) {
      const int64_t per = k ? std::max<int64_t>(1, (int64_t)std::ceil(total / (k * CUS * c[i].us))) : std::max<int64_t>(1, c[i].steps);
      now[i] = (int)std::min<int64_t>(most, std::max<int64_t>(1, (c[i].steps + per - 1) / per));
      const double time = c[i].groups ? (double)((c[i].steps + now[i] - 1) / now[i]) * c[i].us : 0.0;
      sum += c[i].groups * now[i] * time;
      longest = std::max(longest, time);
      groups += c[i].groups * now[i];
      if (now[i] > 1) join += 2 * now[i] * c[i].bytes / 4e6;
    }
    if (now[0] > 1 || (n > 1 && now[1] > 1)) join += 5.0;
    // what a CU does of its full rate with one workgroup, and with as many as there are for each
    const double each = groups / CUS, alone = held == 1 ? 1.0 : held == 2 ? 0.65 : 0.55;
    const double part = each >= held || held == 1 ? 1.0 : each <= 1 ? alone : alone + (1.0 - alone) * (each - 1) / (held - 1);
    const double time = (each <= 1 ? longest / part : sum / (CUS * part) + end * longest) + START * each + join;
    if (k == 0 || time < 0.98 * best) {
      best = time;
      for (int i = 0; i < n; ++i) c[i].splits = now[i];
    }
  }
  return best;
}
inline double uneven_end(const dsmp_segments& s) { return s.n_seg == 1 ? 0.3 : 1.0; }

// tiles of `size` rows that there are, for an estimate (a launch has tiles_of)
inline int64_t about_tiles(int64_t n, int64_t n_seg, int M, int size) {
  if (n * M <= n_seg * size) return std::min(n * M, n_seg);
  return (n * M + size - 1) / size + (n_seg > 1 ? n_seg / 2 : 0);
}

struct FwdPlan {
  bool few;
  int splits;
  int64_t grid;
};

inline FwdPlan fwd_plan(const dsmp_attention_desc& d, const dsmp_segments& qs, const dsmp_segments& ks) {
  const int G = d.heads / d.kv_heads;
  const int64_t keys = ks.n / ks.n_seg;
  const double bytes = 4.0 * qs.n * d.heads * d.head_dim;
  const int per_wide = d.dtype == DSMP_F32 ? 32 : 64;
  Cut wide{about_tiles(qs.n, qs.n_seg, G, WIDE_ROWS) * d.kv_heads, (keys + per_wide - 1) / per_wide, tile_us(d, FORWARD, true), bytes, 1};
  Cut few{about_tiles(qs.n, qs.n_seg, G, FEW_ROWS) * d.kv_heads, (keys + 127) / 128, tile_us(d, FORWARD, false), bytes, 1};
  double end = uneven_end(ks);
  // one tile of rows to a segment: keys and values come from memory, once, at 5 TB/s
  const bool once = qs.n * G <= 32 * qs.n_seg;
  if (once) end *= 2, few.us = std::max(few.us, 128 * d.head_dim * (d.dtype == DSMP_F32 ? 8.0 : 4.0) * 256 / 5e6);
  const double tw = cut_evenly(&wide, 1, held(d, FORWARD, true), 64, end);
  const double tf = cut_evenly(&few, 1, held(d, FORWARD, false), MAX_SPLITS, end);
  FwdPlan p{};
  p.few = once || tf <= tw;
  p.splits = p.few ? few.splits : wide.splits;
  p.grid = tiles_of(qs.n, qs.n_seg, G, p.few ? FEW_ROWS : WIDE_ROWS) * d.kv_heads;
  if (p.grid * p.splits > MAX_GROUPS) p.splits = 1;
  p.grid *= p.splits;
  return p;
}

struct BwdPlan {
  bool wide_q, wide_k;
  int splits_q, splits_k;
  int64_t grid_q, grid_k;
};

// The gradients of the queries and of the keys each WIDE or FEW, cut each for itself; or both FEW, in one launch.
inline BwdPlan bwd_plan(const dsmp_attention_desc& d, const dsmp_segments& qs, const dsmp_segments& ks) {
  const int G = d.heads / d.kv_heads, per_wide = d.dtype == DSMP_F32 ? 32 : 64;
  const int64_t keys = ks.n / ks.n_seg, rows = qs.n / qs.n_seg * G;
  const double bq = 4.0 * qs.n * d.heads * d.head_dim, bk = 8.0 * ks.n * d.kv_heads * d.head_dim;
  Cut q[2], k[2], both[2];
  double tq[2], tk[2];
  for (int wide = 0; wide < 2; ++wide) {
    const int own = wide ? WIDE_ROWS : FEW_ROWS, along = wide ? per_wide : 128;
    q[wide] = {qs.n ? about_tiles(qs.n, qs.n_seg, G, own) * d.kv_heads : 0, (keys + along - 1) / along, tile_us(d, GRAD_Q, wide), bq, 1};
    k[wide] = {ks.n ? about_tiles(ks.n, ks.n_seg, 1, own) * d.kv_heads : 0, (rows + along - 1) / along, tile_us(d, GRAD_K, wide), bk, 1};
  }
  both[0] = q[0], both[1] = k[0];
  const double together = cut_evenly(both, 2, held(d, GRAD_K, false), 64, uneven_end(ks));
  for (int wide = 0; wide < 2; ++wide) {
    tq[wide] = cut_evenly(&q[wide], 1, held(d, GRAD_Q, wide), 64, uneven_end(ks));
    tk[wide] = cut_evenly(&k[wide], 1, held(d, GRAD_K, wide), 64, uneven_end(ks));
  }
  // few keys to a segment: FEW tiles of queries take D from the weights
  if (d.dtype == DSMP_BF16 && ks.n <= 32 * ks.n_seg) tq[1] = 2 * tq[0] + tq[1];
  BwdPlan p{};
  p.wide_q = tq[1] < tq[0], p.wide_k = tk[1] < tk[0];
  p.splits_q = q[p.wide_q].splits, p.splits_k = k[p.wide_k].splits;
  if (together < std::min(tq[0], tq[1]) + std::min(tk[0], tk[1]) + 3.0) {
    p.wide_q = p.wide_k = false;
    p.splits_q = both[0].splits, p.splits_k = both[1].splits;
  }
  p.grid_q = qs.n ? tiles_of(qs.n, qs.n_seg, G, p.wide_q ? WIDE_ROWS : FEW_ROWS) * d.kv_heads : 0;
  p.grid_k = ks.n ? tiles_of(ks.n, ks.n_seg, 1, p.wide_k ? WIDE_ROWS : FEW_ROWS) * d.kv_heads : 0;
  if (p.grid_q * p.splits_q + p.grid_k * p.splits_k > MAX_GROUPS) p.splits_q = p.splits_k = 1;
  p.grid_q *= p.splits_q, p.grid_k *= p.splits_k;
  return p;
}

// Gradients of keys in WIDE tiles whose rows go two by two: an even number of heads shares them, so that two rows have
// one query, and its distance is formed once.
inline bool rows_paired(const dsmp_attention_desc& d) {
  return d.dtype == DSMP_BF16 && d.dim > 0 && (d.heads / d.kv_heads) % 2 == 0;
}

}  // namespace dsmp
