// What the kernels of attention with terms in its scores share: their arguments,
// the masks' bounds, the buckets of distances, and every result by its definition,
// one row a wave.
#pragma once

#include <algorithm>

#include "common.h"

namespace pb {

constexpr int kScoreMaxBuckets = 64;
constexpr int kScoreMap = 512;

struct ScoreArgs {
  const void *q, *k, *v;
  int ld_q, ld_kv;
  void* o;  // written by the forward, read by the backward
  int ld_o;
  float* lse;
  const void* d_o;
  int ld_do;
  void *dq, *dk, *dv;
  int ld_dq, ld_dkv;
  int batch, seq_q, seq_k, heads, kv_heads, group;  // group: heads / kv_heads
  int causal, window;
  float scale, cap;
  float dscale;  // scale; 0 where no query sees two keys (P is 1 and its gradient 0)
  const int *docs, *prefix;
  int n_docs;
  const float *slopes, *table;
  int buckets, side;            // side: buckets of one sign of the distance
  int first[kScoreMaxBuckets];  // first distance of each bucket of a side
  uint32_t map[kScoreMap / 4];  // a byte each: bucket of the distances below kScoreMap
  float* dtable;
  float* bias_part;  // sums of the table's gradient, [batch * row blocks][heads][buckets]
  int pack;                     // heads of one key head that a block of rows holds
  int wide;                     // products: factors that are computed keep 16 bits
  // minus sum of P dP of the rows, [batch][head / pack][position][head mod pack]; null: as
  // minus sum of dO O
  const float* minus_delta;
};

// How many workgroups may share a block's tiles.
struct ScorePlan {
  int chunks;
};
struct ScoreBwdPlan {
  ScorePlan kv, q, d;  // dK and dV by tiles of rows, dQ and the row terms by tiles of keys
};
// The most tiles (of `keys`) that a block of `rows` rows may visit, whatever the
// documents.
inline int score_most_tiles(const ScoreArgs& a, int rows, int keys) {
  const long long all = (a.seq_k + keys - 1) / keys;
  if (a.prefix) return (int)all;
  const long long span = (rows + a.pack - 1) / a.pack + 1;
  const long long reach = (long long)(a.causal ? 1 : 2) * a.window + span;
  return (int)std::min(all, reach / keys + 2);
}

namespace score {

constexpr float kNegInf = -__builtin_huge_valf();

// Positions of a batch row that a query at p may see by its document: keys ds .. de - 1,
// of them ds .. pe - 1 in the prefix.  Nothing: all 0.  (By a key's own document: the
// queries that may see it.)  Whatever the offsets hold, 0 <= ds <= p < de <= seq_k or
// all are 0.
struct Bounds {
  int ds, de, pe;
};
PB_DEV Bounds bounds_of(const ScoreArgs& a, int b, int p) {
  if (!a.docs) {
    const int pre = a.prefix ? a.prefix[b] : 0;
    return Bounds{0, a.seq_k, max(0, min(pre, a.seq_k))};
  }
  const int row0 = b * a.seq_k, t = row0 + p;
  if (a.n_docs < 1 || a.docs[0] > t) return Bounds{0, 0, 0};
  int lo = 0, hi = a.n_docs - 1;
  while (lo < hi) {
    const int mid = lo + ((hi - lo + 1) >> 1);
    if (a.docs[mid] <= t) lo = mid;
    else hi = mid - 1;
  }
  const long long s = a.docs[lo], e = a.docs[lo + 1], pre = a.prefix ? a.prefix[lo] : 0;
  if (e <= t) return Bounds{0, 0, 0};
  const int ds = (int)max(s - row0, 0LL), de = (int)min(e - row0, (long long)a.seq_k);
  return Bounds{ds, de, (int)max((long long)ds, min(s + pre - row0, (long long)de))};
}
// Keys of the window of a query at p (apart from its prefix): first .. last.
PB_DEV int window_first(const ScoreArgs& a, const Bounds& d, int p) {
  return max(d.ds, p - min(a.window, p + 1) + 1);
}
PB_DEV int window_last(const ScoreArgs& a, const Bounds& d, int p) {
  return a.causal ? min(p, d.de - 1) : min(d.de - 1, p + min(a.window - 1, a.seq_k));
}
// Queries that see the key at j: first .. last.
PB_DEV int seen_first(const ScoreArgs& a, const Bounds& d, int j) {
  if (j < d.pe) return d.ds;
  return a.causal ? max(d.ds, j) : max(d.ds, j - min(a.window, j + 1) + 1);
}
PB_DEV int seen_last(const ScoreArgs& a, const Bounds& d, int j) {
  return j < d.pe ? d.de - 1 : min(d.de - 1, j + min(a.window - 1, a.seq_k));
}

// Bucket of distance n = p - j.
PB_DEV int bucket_of(const ScoreArgs& a, int n) {
  const int d = a.causal ? max(n, 0) : abs(n);
  int lo = 0, hi = a.side - 1;  // the last bucket that begins at or before d
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.first[mid] <= d) lo = mid;
    else hi = mid - 1;
  }
  return lo + (!a.causal && n < 0 ? a.side : 0);
}

// A bias of the type's lowest value masks, as -infinity does (sums with it would lose
// the score, and the softmax's base 2 has no room for it).
constexpr float kMasks = -1e38f;
PB_DEV float bias_value(float v) { return v < kMasks ? kNegInf : v; }

// ---------------------------------------------------- rows by the definition
// One wave a row, 64 keys (or queries) at a time, a lane each; the products with rows
// of V, K, Q or dO then take features e = lane + 64 n, one visible row after another.
// Only visible rows enter any sum, so that what a mask hides may hold anything.
template <typename T, int D>
PB_DEV float dot_row(const T* __restrict__ x, const T* __restrict__ y) {
  float acc[2] = {0.f, 0.f};
#pragma unroll 4
  for (int e = 0; e < D; e += 8) {
    float u[8], v[8];
    load8(x + e, u);
    load8(y + e, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i & 1] = fmaf(u[i], v[i], acc[i & 1]);
  }
  return acc[0] + acc[1];
}
// Score of q.k = dot at distance n; slope: what the cap leaves of its gradient.
PB_DEV float score_of(const ScoreArgs& a, float dot, int h, int n, float& slope) {
  float s = dot * a.scale;
  slope = 1.f;
  if (a.cap > 0.f) {
    const float x = s / a.cap, e = expf(-2.f * fabsf(x)), r = 1.f / (1.f + e);
    s = a.cap * tanhf(x);
    slope = 4.f * e * r * r;  // 1 - tanh^2, to the last of it
  }
  if (a.slopes) s = fmaf(-a.slopes[h], (float)abs(n), s);
  if (a.table) s += bias_value(a.table[(size_t)bucket_of(a, n) * a.heads + h]);
  return s;
}
PB_DEV float lane_value(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}
template <int D>
struct RowSum {
  static constexpr int NE = (D + 63) / 64;
  float v[NE] = {};
  template <typename T>
  PB_DEV void add(const T* __restrict__ row, float f, int lane) {
#pragma unroll
    for (int n = 0; n < NE; ++n)
      if (lane + 64 * n < D) v[n] = fmaf(f, load1(row + lane + 64 * n), v[n]);
  }
  template <typename T>
  PB_DEV void store(T* __restrict__ row, float f, int lane) const {
#pragma unroll
    for (int n = 0; n < NE; ++n)
      if (lane + 64 * n < D) row[lane + 64 * n] = (T)(v[n] * f);
  }
};
template <typename T, int D>
PB_DEV const T* q_row(const ScoreArgs& a, int b, int i, int h) {
  return (const T*)a.q + ((size_t)b * a.seq_q + i) * a.ld_q + (size_t)h * D;
}
template <typename T, int D>
PB_DEV const T* do_row(const ScoreArgs& a, int b, int i, int h) {
  return (const T*)a.d_o + ((size_t)b * a.seq_q + i) * a.ld_do + (size_t)h * D;
}
template <typename T, int D>
PB_DEV T* o_row(const ScoreArgs& a, int b, int i, int h) {
  return (T*)a.o + ((size_t)b * a.seq_q + i) * a.ld_o + (size_t)h * D;
}
template <typename T, int D>
PB_DEV const T* kv_row(const ScoreArgs& a, const void* x, int b, int j, int kvh) {
  return (const T*)x + ((size_t)b * a.seq_k + j) * a.ld_kv + (size_t)kvh * D;
}
PB_DEV size_t lse_at(const ScoreArgs& a, int b, int h, int i) {
  return ((size_t)b * a.heads + h) * a.seq_q + i;
}

template <typename T, int D>
PB_DEV void fwd_row(const ScoreArgs& a, int b, int h, int i, int lane) {
  const int p = i + a.seq_k - a.seq_q, kvh = h / a.group;
  const Bounds d = bounds_of(a, b, p);
  const int first = window_first(a, d, p), last = window_last(a, d, p);
  const T* qr = q_row<T, D>(a, b, i, h);
  RowSum<D> acc;
  float m = kNegInf, l = 0.f;
  const int end = max(last + 1, d.pe);
  for (int j0 = d.pe > d.ds ? d.ds : first; j0 < end; j0 += 64) {
    const int j = j0 + lane;
    const bool sees = j < d.pe || (j >= first && j <= last);
    float s = kNegInf, slope;
    if (sees) s = score_of(a, dot_row<T, D>(qr, kv_row<T, D>(a, a.k, b, j, kvh)), h, p - j, slope);
    unsigned long long any = __builtin_amdgcn_ballot_w64(sees && s != kNegInf);
    if (!any) continue;
    const float mn = fmaxf(m, wave_max(s));
    const float pr = s == kNegInf ? 0.f : expf(s - mn), f = m == kNegInf ? 0.f : expf(m - mn);
    l = l * f + wave_sum(pr);
#pragma unroll
    for (int n = 0; n < RowSum<D>::NE; ++n) acc.v[n] *= f;
    while (any) {
      const int jj = __builtin_ctzll(any);
      any &= any - 1;
      acc.add(kv_row<T, D>(a, a.v, b, j0 + jj, kvh), lane_value(pr, jj), lane);
    }
    m = mn;
  }
  // (l = 0: nothing seen.  A NaN among the scores is one in l.)
  acc.store(o_row<T, D>(a, b, i, h), l == 0.f ? 0.f : 1.f / l, lane);
  if (lane == 0) a.lse[lse_at(a, b, h, i)] = l == 0.f ? kNegInf : m + logf(l);
}

// P of the pair and P (dP - delta), its gradient at the score.
struct Pair {
  float p, dz, slope;
};
template <typename T, int D>
PB_DEV Pair pair_of(const ScoreArgs& a, const T* qr, const T* gr, const T* kr, const T* vr, int h,
                    int n, float L, float delta) {
  Pair x{0.f, 0.f, 1.f};
  const float s = score_of(a, dot_row<T, D>(qr, kr), h, n, x.slope);
  if (s == kNegInf || L == kNegInf) return x;
  x.p = expf(s - L);
  x.dz = x.p * (dot_row<T, D>(gr, vr) - delta);
  return x;
}
template <typename T, int D>
PB_DEV float delta_of(const ScoreArgs& a, const T* gr, int b, int h, int i) {
  if (!a.minus_delta) return dot_row<T, D>(gr, o_row<T, D>(a, b, i, h));
  const size_t set = (size_t)b * (a.heads / a.pack) + h / a.pack;
  return -a.minus_delta[(set * a.seq_q + i) * a.pack + h % a.pack];
}
template <typename T, int D>
PB_DEV void dq_row(const ScoreArgs& a, int b, int h, int i, int lane) {
  const int p = i + a.seq_k - a.seq_q, kvh = h / a.group;
  const Bounds d = bounds_of(a, b, p);
  const int first = window_first(a, d, p), last = window_last(a, d, p);
  const T *qr = q_row<T, D>(a, b, i, h), *gr = do_row<T, D>(a, b, i, h);
  const float L = a.lse[lse_at(a, b, h, i)];
  const float delta = delta_of<T, D>(a, gr, b, h, i);
  RowSum<D> acc;
  const int end = L == kNegInf ? 0 : max(last + 1, d.pe);
  for (int j0 = d.pe > d.ds ? d.ds : first; j0 < end; j0 += 64) {
    const int j = j0 + lane;
    Pair x{0.f, 0.f, 1.f};
    if (j < d.pe || (j >= first && j <= last))
      x = pair_of<T, D>(a, qr, gr, kv_row<T, D>(a, a.k, b, j, kvh), kv_row<T, D>(a, a.v, b, j, kvh),
                        h, p - j, L, delta);
    const float du = x.dz * x.slope;
    unsigned long long any = __builtin_amdgcn_ballot_w64(x.p != 0.f);
    while (any) {
      const int jj = __builtin_ctzll(any);
      any &= any - 1;
      acc.add(kv_row<T, D>(a, a.k, b, j0 + jj, kvh), lane_value(du, jj), lane);
    }
  }
  acc.store((T*)a.dq + ((size_t)b * a.seq_q + i) * a.ld_dq + (size_t)h * D, a.dscale, lane);
}
template <typename T, int D>
PB_DEV void dkdv_row(const ScoreArgs& a, int b, int kvh, int j, int lane) {
  const Bounds d = bounds_of(a, b, j);
  const int off = a.seq_k - a.seq_q;
  const int first = max(seen_first(a, d, j) - off, 0);
  const int last = d.de > d.ds ? seen_last(a, d, j) - off : -1;
  const T *kr = kv_row<T, D>(a, a.k, b, j, kvh), *vr = kv_row<T, D>(a, a.v, b, j, kvh);
  RowSum<D> dk, dv;
  for (int h = kvh * a.group; h < (kvh + 1) * a.group; ++h)
    for (int i0 = first; i0 <= last; i0 += 64) {
      const int i = i0 + lane;
      Pair x{0.f, 0.f, 1.f};
      if (i <= last) {
        const T* gr = do_row<T, D>(a, b, i, h);
        x = pair_of<T, D>(a, q_row<T, D>(a, b, i, h), gr, kr, vr, h, i + off - j,
                          a.lse[lse_at(a, b, h, i)], delta_of<T, D>(a, gr, b, h, i));
      }
      const float du = x.dz * x.slope;
      unsigned long long any = __builtin_amdgcn_ballot_w64(x.p != 0.f);
      while (any) {
        const int ii = __builtin_ctzll(any);
        any &= any - 1;
        dv.add(do_row<T, D>(a, b, i0 + ii, h), lane_value(x.p, ii), lane);
        dk.add(q_row<T, D>(a, b, i0 + ii, h), lane_value(du, ii), lane);
      }
    }
  const size_t at = ((size_t)b * a.seq_k + j) * a.ld_dkv + (size_t)kvh * D;
  dk.store((T*)a.dk + at, a.dscale, lane);
  dv.store((T*)a.dv + at, 1.f, lane);
}

}  // namespace score
}  // namespace pb
