// What the kernels of the attention over whole prompts share: parameters, and where a sequence's rows and keys lie.
#pragma once

#include "kv_attention.cuh"

namespace vscan {
namespace kv {

struct PromptParams : AttnParams {
  const char* k;
  const char* v;
  long long k_seq, k_head, k_row, v_seq, v_head, v_row;   // bytes
  const int32_t* kv_offset;
  int kv_rows;
};

// First key row of sequence b in the buffer (padded: 0), and its keys, held inside the buffer
__host__ __device__ __forceinline__ void key_span(const PromptParams& p, int b, int& first, int& n) {
  const long long lo = p.kv_offset[b], given = max(p.kv_offset[b + 1] - lo, 0ll);
  first = p.padded ? 0 : static_cast<int>(lo);
  const long long room = p.padded ? p.kv_rows : lo < 0 ? 0 : max(p.kv_rows - lo, 0ll);
  n = static_cast<int>(min(given, room));
}

__host__ __device__ __forceinline__ Sequence sequence_at(const PromptParams& p, int b) {
  Sequence s;
  const long long lo = p.row_offset[b], given = max(p.row_offset[b + 1] - lo, 0ll);
  s.first = p.padded ? 0 : static_cast<int>(lo);
  const long long room = p.padded ? p.rows : lo < 0 ? 0 : max(p.rows - lo, 0ll);
  s.n = static_cast<int>(min(min(given, room), static_cast<long long>(p.max_q_len)));
  int first;
  key_span(p, b, first, s.len);
  s.start = max(static_cast<long long>(p.kv_offset[b + 1]) - p.kv_offset[b], 0ll) - given;
  s.tiles = s.units = 0;
  s.weight = 0;
  return s;
}

}  // namespace kv
}  // namespace vscan
