// What the attention kernels over the paged 8-bit cache share: parameters, the division of the work among the CTAs, the
// layout of partial results.
#pragma once

#include "kv_common.cuh"

namespace vscan {
namespace kv {

struct AttnParams {
  const char* q;
  char* out;
  float* lse;
  long long q_seq, q_head, q_row, o_seq, o_head, o_row;   // bytes
  long long l_seq, l_head, l_row;                         // floats
  const int32_t* kv_len;
  const int32_t* row_offset;
  const int32_t* block_table;
  const uint8_t* k_cache;
  const uint8_t* v_cache;
  const float* k_scale;
  const float* v_scale;
  int batch, q_heads, kv_heads, group, head_dim, block_size, shift, num_blocks, max_blocks, rows, padded, max_q_len, causal;
  int tile_rows;        // query rows (new row x head of the group) of a tile
  float scale_log2e;
  uint32_t* status;
  uint32_t* flags;             // [ctas] 1: the CTA met a block or a length out of range
  struct Boundary* boundary;   // [ctas]
  float* partial;              // [ctas][2][tile_rows][head_dim + 2]
};

// The work is a line of units of kUnit tokens: sequences in order, in a sequence KV head by KV head, tile by tile, in a tile
// the units of its keys.  Each of the G CTAs of a launch takes an equal stretch, whatever the lengths are, so one long
// sequence among short ones does not hold up the launch.  A segment (one tile, one KV head) that is not longer than
// kWhole units stays with the CTA that reaches its start; a longer one may be cut, and its pieces are joined afterwards.
constexpr int kUnit = 64;
constexpr int kWhole = 4;

struct Boundary {       // what lies at the start of a CTA's stretch
  long long seg0, seg1; // the segment that is cut there, as places on the line; seg1 = 0: none
  long long quota;
  int b, head, tile, pad;
};

struct Sequence {       // of one sequence: new rows, keys, tiles, units of a segment
  int first, n, len, tiles, units;
  long long start, weight;
};

__device__ __forceinline__ Sequence sequence_at(const AttnParams& p, int b) {
  Sequence s;
  row_span(p.row_offset, p.kv_len, b, p.rows, p.padded, s.first, s.n, s.start);
  s.n = min(s.n, p.max_q_len);
  s.len = min(max(p.kv_len[b], 0), p.max_blocks << p.shift);
  s.tiles = (s.n * p.group + p.tile_rows - 1) / p.tile_rows;
  s.units = max(1, (s.len + kUnit - 1) / kUnit);
  s.weight = static_cast<long long>(s.tiles) * p.kv_heads * s.units;
  return s;
}

struct ScheduleShared {
  long long warp_sums[32];
  long long seq0;
  int b;
};

// Where this CTA's stretch starts: the sequence and its place on the line.  Called by all THREADS threads.
template <int THREADS>
__device__ __forceinline__ void locate(const AttnParams& p, ScheduleShared& sh, long long& begin, long long& quota, long long& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per = (p.batch + THREADS - 1) / THREADS, b0 = min(static_cast<int>(threadIdx.x) * per, p.batch), b1 = min(b0 + per, p.batch);
  long long sum = 0;
  for (int b = b0; b < b1; ++b) sum += sequence_at(p, b).weight;
  long long incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long t = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += t;
  }
  if (lane == 31) sh.warp_sums[warp] = incl;
  if (threadIdx.x == 0) sh.b = -1;
  __syncthreads();
  long long before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) before += sh.warp_sums[w];
    total += sh.warp_sums[w];
  }
  quota = max((total + gridDim.x - 1) / gridDim.x, 1ll);
  begin = blockIdx.x * quota;
  long long at = before + incl - sum;
  if (at <= begin && begin < at + sum) {
    for (int b = b0; b < b1; ++b) {
      const long long w = sequence_at(p, b).weight;
      if (begin < at + w) { sh.b = b; sh.seq0 = at; break; }
      at += w;
    }
  }
  __syncthreads();
}

// Floats of one partial result: tile_rows x head_dim sums, then their maxima, then their denominators
__host__ __device__ inline size_t partial_floats(int tile_rows, int head_dim) { return static_cast<size_t>(tile_rows) * (head_dim + 2); }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Where row r (new row x head of the group) of a tile lies
struct RowAt { int i, h; };
__device__ __forceinline__ RowAt row_at(const AttnParams& p, int tile, int head, int r) {
  const int flat = tile * p.tile_rows + r, i = flat / p.group;
  return {i, head * p.group + flat - i * p.group};
}
__device__ __forceinline__ char* out_at(const AttnParams& p, int b, int first, RowAt r) {
  return p.out + (p.padded ? b * p.o_seq : first * p.o_row) + r.i * p.o_row + r.h * p.o_head;
}
__device__ __forceinline__ float* lse_at(const AttnParams& p, int b, int first, RowAt r) {
  return p.lse + (p.padded ? b * p.l_seq : first * p.l_row) + r.i * p.l_row + r.h * p.l_head;
}
__device__ __forceinline__ const char* q_at(const AttnParams& p, int b, int first, RowAt r) {
  return p.q + (p.padded ? b * p.q_seq : first * p.q_row) + r.i * p.q_row + r.h * p.q_head;
}
// Tokens that new row i sees
__device__ __forceinline__ int visible(const AttnParams& p, const Sequence& s, int i) {
  if (!p.causal) return s.len;
  return static_cast<int>(min(max(s.start + i + 1, 0ll), static_cast<long long>(s.len)));
}

template <typename T>
__device__ __forceinline__ void store_out(char* row, int c, float v) {
  if constexpr (sizeof(T) == 4) reinterpret_cast<float*>(row)[c] = v;
  else reinterpret_cast<__nv_bfloat16*>(row)[c] = __float2bfloat16_rn(v);
}

}  // namespace kv
}  // namespace vscan
