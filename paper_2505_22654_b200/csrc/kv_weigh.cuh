// What the kernels that gather attention weights share: parameters, and where a sequence's rows, tokens and weights lie.
#pragma once

#include "kv_attention.cuh"

namespace vscan {
namespace kv {

struct WeighParams : AttnParams {
  float* weight;
  float decay;
  int window;
};

// One segment a KV head: rows of all tiles go to the same tokens
__device__ __forceinline__ Sequence sequence_at(const WeighParams& p, int b) {
  Sequence s;
  row_span(p.row_offset, p.kv_len, b, p.rows, p.padded, s.first, s.n, s.start);
  s.n = min(s.n, p.max_q_len);
  s.len = min(max(p.kv_len[b], 0), p.max_blocks << p.shift);
  s.tiles = s.n > 0 ? 1 : 0;
  s.units = max(1, (s.len + kUnit - 1) / kUnit);
  s.weight = static_cast<long long>(s.tiles) * p.kv_heads * s.units;
  return s;
}

// Row r of the window's rows x heads of the group
struct WindowRow { RowAt at; int seen; float lse; };   // seen: tokens, 0 where the row gives nothing; lse in base 2
__device__ __forceinline__ WindowRow window_row(const WeighParams& p, const Sequence& s, int b, int head, int r) {
  const int u = min(s.n, p.window), i = r / p.group;
  WindowRow w = {{s.n - u, head * p.group}, 0, 0.f};
  if (i >= u) return w;
  w.at.i += i;
  w.at.h += r - i * p.group;
  const float lse = *lse_at(p, b, s.first, w.at);
  w.lse = lse * 1.44269504088896341f;
  if (lse != -INFINITY) w.seen = visible(p, s, w.at.i);
  return w;
}
// Rows of a segment; no more than fit 32 bits, since rows x heads of the buffer do
__device__ __forceinline__ int window_rows(const WeighParams& p, const Sequence& s) { return min(s.n, p.window) * p.group; }

__device__ __forceinline__ float* weight_at(const WeighParams& p, int block, int head, int t) {
  return p.weight + ((static_cast<size_t>(block) * p.kv_heads + head) << p.shift) + (t & (p.block_size - 1));
}

}  // namespace kv
}  // namespace vscan
