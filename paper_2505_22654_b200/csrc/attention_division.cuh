// Division of the work of attention over many query rows: tiles of rows against steps of keys, cut into equal stretches.
#pragma once

#include "kv_attention.cuh"

namespace vscan {
namespace kv {

// Threads of a CTA, query rows of a tile, keys of a step, and the steps up to which a tile is not cut.  ROWS 0: rows of a tile are known at
// run time only.  EXTRA: what a tile weighs, in steps, beside its own: its start and end.
template <int THREADS, int ROWS, int KEYS, int WHOLE, int EXTRA = 0>
struct TileShape {
  static constexpr int kThreads = THREADS, kKeys = KEYS, kWhole = WHOLE, kExtra = EXTRA;
  __host__ __device__ __forceinline__ static int rows(const AttnParams& p) { return ROWS > 0 ? ROWS : p.tile_rows; }
};

struct DivisionShared {
  long long weight[32];
  long long seq0;
  int b;
};

// As for few rows, but a place on the line is a key seen by a query row, so that the triangle of a causal prompt is divided
// evenly: tile k of a causal sequence weighs group * start + min(kRows (k + 1), rows), at least one step, which has a closed
// prefix sum.  The sum is exact whatever the rows of a tile are (125 for groups of five above 128 channels): a stretch that finds its start
// by it and one that gets there tile by tile have to agree on every place.
struct TcSequence {
  Sequence s;
  long long base;       // what every tile sees at least
  long long rows;       // query rows; causal tiles weigh more one after another
  long long weight;     // of all tiles of a KV head
  int tiles, light;     // light: tiles in front that weigh one step although they see less
};

template <typename S>
__host__ __device__ __forceinline__ long long step_weight(const AttnParams& p) { return static_cast<long long>(S::kKeys) * p.group; }

// What tile k weighs, and the k tiles in front of it
template <typename S>
__host__ __device__ __forceinline__ long long tile_weight(const AttnParams& p, const TcSequence& q, int k) {
  const long long one = step_weight<S>(p);
  const long long seen = !p.causal ? q.base : q.base + (k + 1 < q.tiles ? static_cast<long long>(S::rows(p)) * (k + 1) : q.rows);
  return max(seen, one) + S::kExtra * one;
}
template <typename S>
__host__ __device__ __forceinline__ long long tiles_before(const AttnParams& p, const TcSequence& q, long long k) {
  if (!p.causal) return k * tile_weight<S>(p, q, 0);
  const long long one = step_weight<S>(p);
  const long long n = min(k, static_cast<long long>(q.tiles - 1)), m = min(n, static_cast<long long>(q.light));
  const long long sum = m * one + (n - m) * q.base + ((n * (n + 1) - m * (m + 1)) >> 1) * S::rows(p) + n * one * S::kExtra;
  return k < q.tiles ? sum : sum + tile_weight<S>(p, q, q.tiles - 1);
}

// Quotient of numbers that nearly always fit 32 bits; bit by bit where they do not (a division of 64 bits is 2 KB of instructions
// wherever it stands, and the kernels that divide here have to stay in the instruction cache)
__host__ __device__ __forceinline__ long long quotient(long long a, long long b) {
  if (((a | b) >> 32) == 0) return static_cast<unsigned>(a) / static_cast<unsigned>(b);
  unsigned long long q = 0, r = 0;
#pragma unroll 1
  for (int i = 63; i >= 0; --i) {
    r = r << 1 | (static_cast<unsigned long long>(a) >> i & 1);
    q <<= 1;
    if (r >= static_cast<unsigned long long>(b)) { r -= b; q |= 1; }
  }
  return static_cast<long long>(q);
}

template <typename S, typename P>
__host__ __device__ __forceinline__ TcSequence tc_sequence_at(const P& p, int b) {
  TcSequence q;
  q.s = sequence_at(p, b);
  q.rows = static_cast<long long>(q.s.n) * p.group;
  q.tiles = static_cast<int>(quotient(q.rows + S::rows(p) - 1, S::rows(p)));
  q.base = p.causal ? max(q.s.start, 0ll) * p.group : static_cast<long long>(q.s.len) * p.group;
  q.light = static_cast<int>(max(quotient(max(step_weight<S>(p) - q.base, 0ll) + S::rows(p) - 1, S::rows(p)) - 1, 0ll));
  q.weight = q.tiles > 0 ? tiles_before<S>(p, q, q.tiles) : 0;
  return q;
}

struct TcStretch { long long begin, end, quota, seq0; int b; };

// Stretch k of `ctas` on a line of `total`; which sequence it starts in is another question
template <typename S>
__host__ __device__ __forceinline__ TcStretch stretch_of(const AttnParams& p, long long total, unsigned ctas, unsigned k) {
  TcStretch st = {};
  // a stretch is at least a step long, so that no two cuts fall into one step
  st.quota = max(quotient(total + ctas - 1, ctas), step_weight<S>(p) * (1 + S::kExtra));
  st.begin = min(k * st.quota, total);
  st.end = min(st.begin + st.quota, total);
  return st;
}

template <typename S, typename P>
__device__ __forceinline__ TcStretch tc_locate(const P& p, DivisionShared& sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per = (p.batch + S::kThreads - 1) / S::kThreads, b0 = min(static_cast<int>(threadIdx.x) * per, p.batch), b1 = min(b0 + per, p.batch);
  long long sum = 0;
#pragma unroll 1
  for (int b = b0; b < b1; ++b) sum += tc_sequence_at<S>(p, b).weight * p.kv_heads;
  long long incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long t = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += t;
  }
  if (lane == 31) sh.weight[warp] = incl;
  __syncthreads();
  long long before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < S::kThreads / 32; ++w) {
    if (w < warp) before += sh.weight[w];
    total += sh.weight[w];
  }
  TcStretch st = stretch_of<S>(p, total, gridDim.x, blockIdx.x);
  long long at = before + incl - sum;
  if (at <= st.begin && st.begin < at + sum) {
#pragma unroll 1
    for (int b = b0; b < b1; ++b) {
      const long long w = tc_sequence_at<S>(p, b).weight * p.kv_heads;
      if (st.begin < at + w) { sh.b = b; sh.seq0 = at; break; }
      at += w;
    }
  }
  __syncthreads();
  st.b = sh.b;
  st.seq0 = sh.seq0;
  return st;
}

// The step of a tile that place x of its weight falls into; what a tile weighs beside its steps lies in front of them
template <typename S>
__host__ __device__ __forceinline__ int step_at(long long x, long long per_unit, int units) {
  if (S::kExtra > 0) x = max(x - S::kExtra * per_unit, 0ll);
  return static_cast<int>(min(quotient(x, per_unit), static_cast<long long>(units)));
}

struct TcPiece {
  TcSequence q;
  long long seg0, seg1;   // seg1: the end of what there is to do, as a place on the line
  int b, head, tile, n_rows, most, u0, u1, units;
};

template <typename S, typename P>
__host__ __device__ __forceinline__ bool tc_next(const P& p, TcStretch& st, TcPiece& pc) {
  while (st.begin < st.end) {
    pc.q = tc_sequence_at<S>(p, st.b);
    const long long all = pc.q.weight * p.kv_heads;
    if (st.begin >= st.seq0 + all) { st.seq0 += all; ++st.b; continue; }
    const long long head = quotient(st.begin - st.seq0, pc.q.weight), rel = st.begin - st.seq0 - head * pc.q.weight;
    int lo = 0, hi = pc.q.tiles;
#pragma unroll 1
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (tiles_before<S>(p, pc.q, mid) <= rel) lo = mid; else hi = mid;
    }
    pc.head = static_cast<int>(head); pc.tile = lo; pc.b = st.b;
    pc.seg0 = st.begin - (rel - tiles_before<S>(p, pc.q, lo));
    const long long seg_end = pc.seg0 + tiles_before<S>(p, pc.q, lo + 1) - tiles_before<S>(p, pc.q, lo);
    pc.n_rows = static_cast<int>(min(static_cast<long long>(S::rows(p)), pc.q.rows - static_cast<long long>(lo) * S::rows(p)));
    pc.most = visible(p, pc.q.s, (lo * S::rows(p) + pc.n_rows - 1) / p.group);
    pc.units = max(1, (pc.most + S::kKeys - 1) / S::kKeys);
    const long long per_unit = step_weight<S>(p);
    pc.seg1 = min(seg_end, pc.seg0 + (pc.units + S::kExtra) * per_unit);
    pc.u0 = step_at<S>(st.begin - pc.seg0, per_unit, pc.units);
    pc.u1 = st.end >= seg_end ? pc.units : step_at<S>(st.end - pc.seg0, per_unit, pc.units);
    const bool whole = pc.units <= S::kWhole, starts = st.begin == pc.seg0;
    if (whole) { pc.u0 = 0; pc.u1 = pc.units; }
    st.begin = seg_end;
    if (whole ? starts : pc.u0 < pc.u1) return true;
  }
  return false;
}

}  // namespace kv
}  // namespace vscan
