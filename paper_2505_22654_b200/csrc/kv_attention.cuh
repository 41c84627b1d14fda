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
  float scale_log2e, scale_rest;   // scale * log2(e), and what float32 leaves of it
  uint32_t* status;
  uint32_t* flags;             // [ctas] vscan_status: the CTA met a block or a length out of range, or gave up a wait
  struct Boundary* boundary;   // [ctas]
  float* partial;              // [ctas][2][tile_rows][head_dim + 2]
};

// The work is a line of units of kUnit tokens: sequences in order, in a sequence KV head by KV head, tile by tile, in a tile
// the units of its keys.  Each worker of a launch takes an equal stretch, whatever the lengths are, so one long sequence
// among short ones does not hold up the launch.  A segment (one tile, one KV head) that is not longer than `whole` units
// stays with the worker that reaches its start; a longer one may be cut, and its pieces are joined afterwards.
// Workers are CTAs whose warps share the tokens of a segment, or, where there are at least as many segments as CTAs, single
// warps: then nothing has to be exchanged within a CTA, and the balance is finer.
constexpr int kUnit = 64;
constexpr int kWhole = 4;
constexpr int kWorkersPerCta = 4;

struct Boundary {       // what lies at the start of a worker's stretch
  long long seg0, seg1; // the segment that is cut there, as places on the line; seg1 = 0: none
  long long quota;
  int b, head, tile, first, rows, pad;   // first row of the sequence; query rows of the tile
};

struct Sequence {       // of one sequence: new rows, keys, tiles, units of a segment
  int first, n, len, tiles, units;
  long long start, weight;
};

__host__ __device__ __forceinline__ Sequence sequence_at(const AttnParams& p, int b) {
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
  long long weight[32], segments[32];
  long long seq0[kWorkersPerCta];
  Sequence s[kWorkersPerCta];
  int b[kWorkersPerCta];
};

struct Stretch {          // of a worker: [begin, end) of the line, and the segment that it is in
  long long begin, end, quota, seq0, seg0;
  Sequence s;
  int b, head, tile, worker, whole;
  bool solo, inside;
};

// The stretch of this thread's worker.  Called by all THREADS threads; SOLO: whether warps may be workers.  P: AttnParams, or what a
// call with another sequence_at() derives from it.
template <int THREADS, bool SOLO, typename P>
__device__ __forceinline__ Stretch locate(const P& p, ScheduleShared& sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per = (p.batch + THREADS - 1) / THREADS, b0 = min(static_cast<int>(threadIdx.x) * per, p.batch), b1 = min(b0 + per, p.batch);
  long long sum = 0, segments = 0;
  for (int b = b0; b < b1; ++b) {
    const Sequence s = sequence_at(p, b);
    sum += s.weight;
    segments += static_cast<long long>(s.tiles) * p.kv_heads;
  }
  long long incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long t = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += t;
    if (SOLO) segments += __shfl_xor_sync(0xffffffffu, segments, o);
  }
  if (lane == 31) { sh.weight[warp] = incl; sh.segments[warp] = segments; }
  __syncthreads();
  long long before = 0, total = 0, all_segments = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) before += sh.weight[w];
    total += sh.weight[w];
    all_segments += sh.segments[w];
  }
  Stretch st;
  st.solo = SOLO && all_segments >= gridDim.x;
  const int mine = st.solo ? kWorkersPerCta : 1;
  st.whole = st.solo && (static_cast<long long>(p.max_blocks) << p.shift) > kWhole * kUnit ? 1 : kWhole;
  const long long workers = static_cast<long long>(gridDim.x) * mine;
  st.quota = max((total + workers - 1) / workers, st.solo ? 1ll : 2ll);
  const long long at = before + incl - sum;
  for (int k = 0; k < mine; ++k) {
    const long long begin = (static_cast<long long>(blockIdx.x) * mine + k) * st.quota;
    if (at <= begin && begin < at + sum) {
      long long first = at;
      for (int b = b0; b < b1; ++b) {
        const Sequence s = sequence_at(p, b);
        if (begin < first + s.weight) { sh.b[k] = b; sh.seq0[k] = first; sh.s[k] = s; break; }
        first += s.weight;
      }
    }
  }
  __syncthreads();
  const int k = st.solo ? warp : 0;
  st.worker = blockIdx.x * mine + k;
  st.begin = min(st.worker * st.quota, total);
  st.end = min(st.begin + st.quota, total);
  st.b = sh.b[k];                   // not set, and not used, where the stretch is empty
  st.seq0 = sh.seq0[k];
  st.s = sh.s[k];
  st.inside = false;
  return st;
}

// The next piece of a worker's stretch: units u0 .. u1 - 1 of the segment that the stretch is in then.  Only the first takes
// divisions; from there on segment follows segment, and a sequence's lengths are read once.
struct Piece { int u0, u1; };
template <typename P>
__device__ __forceinline__ bool next_piece(const P& p, Stretch& st, Piece& pc) {
  while (st.begin < st.end) {
    if (!st.inside) {
      const unsigned long long at = st.begin - st.seq0, seg = (at >> 32) == 0 ? static_cast<unsigned>(at) / st.s.units : at / st.s.units;
      st.seg0 = st.seq0 + seg * st.s.units;
      st.head = (seg >> 32) == 0 ? static_cast<unsigned>(seg) / st.s.tiles : static_cast<int>(seg / st.s.tiles);
      st.tile = static_cast<int>(seg - static_cast<unsigned long long>(st.head) * st.s.tiles);
      st.inside = true;
    } else {                                             // the segment before is done with
      st.seg0 = st.begin;
      if (++st.tile == st.s.tiles) { st.tile = 0; ++st.head; }
      if (st.head == p.kv_heads) {
        st.seq0 += st.s.weight;
        do st.s = sequence_at(p, ++st.b); while (st.s.tiles == 0);     // there is one: the stretch goes on
        st.head = 0;
      }
    }
    const bool whole = st.s.units <= st.whole;
    pc.u0 = static_cast<int>(st.begin - st.seg0);
    st.begin = st.seg0 + st.s.units;
    if (whole && pc.u0 > 0) continue;                    // the worker before this one has it
    pc.u1 = whole ? st.s.units : static_cast<int>(min(st.end - st.seg0, static_cast<long long>(st.s.units)));
    return true;
  }
  return false;
}

// Floats of one partial result: tile_rows x head_dim sums, then their maxima, then their denominators; a multiple of 16 bytes
__host__ __device__ inline size_t partial_floats(int tile_rows, int head_dim) { return (static_cast<size_t>(tile_rows) * (head_dim + 2) + 3) & ~size_t{3}; }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// bf16 queries: the V scale of a block is part of the exponent of its weights, which are 2^8 where a token is the reference of its row.
// vscan_kv_write makes scales of 2^-48 .. 2^48.  A block may hold a scale far above what is left in it (its large tokens were taken
// back), so the reference comes down again behind it: once the scales that a row sees are more than kFollow binades lower, to the
// largest that it has been less the scale then, plus the scale now.  With scales held between 2^-30 and 2^30 for that, it is never
// more than 60 binades below what it has been, and the sums keep inside float32.
constexpr float kWeightShift = 8.f;
constexpr float kWeightScale = 256.f;
constexpr int kFollow = 3;

// log of l 2^m.  Where V scales are part of m, l makes up for them: a whole number is moved from m to l, so that two large
// numbers of opposite sign are not rounded before their sum is taken
__device__ __forceinline__ float log_sum(float m, float l) {
  if (l == 0.f) return -INFINITY;
  const float whole = fminf(fmaxf(rintf(m), -32.f), 32.f);
  return ((m - whole) + log2f(l * exp2_int(static_cast<int>(whole)))) * 0.69314718055994531f;
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
__host__ __device__ __forceinline__ int visible(const AttnParams& p, const Sequence& s, int i) {
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
