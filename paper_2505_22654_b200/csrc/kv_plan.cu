// vscan_kv_plan: block tables, slot maps and offsets of a paged KV cache from request lengths, in one launch.
//
// Integers only, a few bytes a request and 12 bytes a new row: launch and load latency bound it.  So that no second launch
// and no exchange between CTAs is needed, every CTA makes the same prefix sums over the batch for itself in shared memory
// (three ints a request) and then takes its share of the rows and of the table rows.  Measured: 256 requests with a row each 4.8 us,
// 1,024 requests with 260,000 rows 6.5 us.
#include "kv_common.cuh"

namespace vscan {
namespace kv {

constexpr int kPlanThreads = 256;
constexpr int kPlanRows = 4;      // neighbouring rows of a thread: one search, 16- and 32-byte stores

struct PlanParams {
  int batch, block_size, shift, num_blocks, max_blocks, rows;
  const int32_t* past_len;
  const int32_t* new_len;
  int32_t* block_table;
  int32_t* free_ring;
  const int64_t* ring_state;
  int32_t* kv_len;
  int32_t* row_offset;
  int64_t* slot_map;
  int32_t* row_pos;
  int64_t* ring_state_out;
  int32_t* report;
};

__device__ __forceinline__ long long block_scan64(long long v, long long* warp_sums, long long& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long t = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += t;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  long long before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 32; ++w) {
    const long long s = warp_sums[w];
    if (w < warp) before += s;
    total += s;
  }
  return before + incl - v;
}

// Blocks that hold n tokens; no sum that could leave 32 bits
__device__ __forceinline__ int blocks_of(int n, int shift) { return ((n - 1) >> shift) + 1; }
__device__ __forceinline__ int saturate(long long v) { return static_cast<int>(min(max(v, 0ll), 0x7fffffffll)); }

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(PlanParams p) {
  extern __shared__ int plan_smem[];
  int* row0 = plan_smem;                    // [batch + 1] prefix sums of new rows
  int* take0 = row0 + p.batch + 1;          // [batch] of blocks taken
  int* give0 = take0 + p.batch;             // [batch] of blocks put back
  __shared__ long long warp_sums[kPlanThreads / 32];
  __shared__ int code_sh;
  grid_dependency_wait();
  if (threadIdx.x == 0) code_sh = 0;
  const long long head = p.ring_state[0], tail = p.ring_state[1];

  // ---- prefix sums: a thread owns neighbouring requests
  const int per = (p.batch + kPlanThreads - 1) / kPlanThreads, b0 = min(static_cast<int>(threadIdx.x) * per, p.batch), b1 = min(b0 + per, p.batch);
  const long long room = static_cast<long long>(p.max_blocks) << p.shift;
  int code = 0;
  long long rows = 0, take = 0, give = 0;
  auto counts = [&](int b, long long& r, long long& t, long long& g) {
    const long long past = p.past_len[b], end = past + p.new_len[b];
    if (past < 0 || end < 0) { code |= 8; r = t = g = 0; return; }
    if (past > room || end > room) code |= 2;
    const long long have = (past + p.block_size - 1) >> p.shift, need = (end + p.block_size - 1) >> p.shift;
    r = max(end - past, 0ll); t = max(need - have, 0ll); g = max(have - need, 0ll);
  };
  for (int b = b0; b < b1; ++b) {
    long long r, t, g;
    counts(b, r, t, g);
    rows += r; take += t; give += g;
  }
  long long all_rows, all_take, all_give;
  long long r_at = block_scan64(rows, warp_sums, all_rows);
  long long t_at = block_scan64(take, warp_sums, all_take);
  long long g_at = block_scan64(give, warp_sums, all_give);
  const long long free_now = tail - head;
  if (all_rows > p.rows) code |= 4;
  if (head < 0 || free_now < 0 || free_now > p.num_blocks || free_now + all_give > p.num_blocks) code |= 16;
  if (all_take > free_now) code |= 1;
  if (code) atomicOr(&code_sh, code);
  __syncthreads();
  code = code_sh;
  if (code) {                                // nothing is planned; what follows finds an empty step
    if (blockIdx.x == 0) {
      for (int b = threadIdx.x; b <= p.batch; b += kPlanThreads) {
        p.row_offset[b] = 0;
        if (b < p.batch) p.kv_len[b] = saturate(min(static_cast<long long>(p.past_len[b]), room));
      }
      if (threadIdx.x == 0) {
        p.report[0] = code; p.report[1] = saturate(all_take); p.report[2] = saturate(all_give); p.report[3] = saturate(all_rows);
        p.ring_state_out[0] = head; p.ring_state_out[1] = tail;
      }
    }
    return;
  }
  for (int b = b0; b < b1; ++b) {            // the totals fit 32 bits here
    long long r, t, g;
    counts(b, r, t, g);
    row0[b] = static_cast<int>(r_at); take0[b] = static_cast<int>(t_at); give0[b] = static_cast<int>(g_at);
    r_at += r; t_at += t; g_at += g;
  }
  if (threadIdx.x == 0) row0[p.batch] = static_cast<int>(all_rows);
  __syncthreads();

  const int n_blocks = p.num_blocks;
  const int head_at = n_blocks > 0 ? static_cast<int>(head % n_blocks) : 0, tail_at = n_blocks > 0 ? static_cast<int>(tail % n_blocks) : 0;
  auto wrapped = [&](int base, int off) {    // both below the ring's size
    const unsigned at = static_cast<unsigned>(base) + static_cast<unsigned>(off);
    return static_cast<int>(at >= static_cast<unsigned>(n_blocks) ? at - n_blocks : at);
  };

  // ---- requests: lengths, offsets, table columns, ring entries (a warp a request)
  const int gthread = blockIdx.x * kPlanThreads + threadIdx.x, gthreads = gridDim.x * kPlanThreads;
  for (int b = gthread; b <= p.batch; b += gthreads) {
    p.row_offset[b] = row0[b];
    if (b < p.batch) p.kv_len[b] = p.past_len[b] + p.new_len[b];
  }
  if (gthread == 0) {
    p.report[0] = 0; p.report[1] = static_cast<int>(all_take); p.report[2] = static_cast<int>(all_give); p.report[3] = static_cast<int>(all_rows);
    p.ring_state_out[0] = head + all_take; p.ring_state_out[1] = tail + all_give;
  }
  const int lane = threadIdx.x & 31;
  for (int b = gthread >> 5; b < p.batch; b += gthreads >> 5) {
    const int past = p.past_len[b], end = past + p.new_len[b];
    const int have = blocks_of(past, p.shift), need = blocks_of(end, p.shift);
    int32_t* row = p.block_table + static_cast<size_t>(b) * p.max_blocks;
    for (int c = have + lane; c < need; c += 32) row[c] = p.free_ring[wrapped(head_at, take0[b] + c - have)];
    for (int c = need + lane; c < have; c += 32) p.free_ring[wrapped(tail_at, give0[b] + c - need)] = row[c];
  }

  // ---- rows: slot and position of each new row.  A new block's number comes from the ring, not from the table, which
  // another CTA may still be writing.
  if (!p.slot_map && !p.row_pos) return;
  const int total = static_cast<int>(all_rows);
  for (long long i0 = static_cast<long long>(gthread) * kPlanRows; i0 < total; i0 += static_cast<long long>(gthreads) * kPlanRows) {
    const int i = static_cast<int>(i0);
    int lo = 0, hi = p.batch;                // the last request that starts at or before row i has it
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (row0[mid] <= i) lo = mid; else hi = mid;
    }
    int b = lo, next = row0[b + 1], past = p.past_len[b], cached = -1, block = 0;
    long long slot[kPlanRows];
    int pos[kPlanRows];
#pragma unroll
    for (int k = 0; k < kPlanRows; ++k) {
      if (i + k >= total) break;
      while (i + k >= next) { ++b; next = row0[b + 1]; past = p.past_len[b]; cached = -1; }
      pos[k] = past + (i + k - row0[b]);
      const int col = pos[k] >> p.shift;
      if (col != cached) {
        const int have = blocks_of(past, p.shift);
        block = col < have ? p.block_table[static_cast<size_t>(b) * p.max_blocks + col] : p.free_ring[wrapped(head_at, take0[b] + col - have)];
        cached = col;
      }
      slot[k] = (static_cast<long long>(block) << p.shift) + (pos[k] & (p.block_size - 1));
    }
    if (i + kPlanRows <= total) {
      if (p.slot_map) {
        longlong2* out = reinterpret_cast<longlong2*>(p.slot_map + i);
        out[0] = make_longlong2(slot[0], slot[1]);
        out[1] = make_longlong2(slot[2], slot[3]);
      }
      if (p.row_pos) *reinterpret_cast<int4*>(p.row_pos + i) = make_int4(pos[0], pos[1], pos[2], pos[3]);
    } else {
#pragma unroll
      for (int k = 0; k < kPlanRows; ++k) {
        if (i + k >= total) break;
        if (p.slot_map) p.slot_map[i + k] = slot[k];
        if (p.row_pos) p.row_pos[i + k] = pos[k];
      }
    }
  }
}

static vscan_status validate_plan(const vscan_kv_plan_desc* d) {
  if (!d) return VSCAN_ERR_INVALID_ARG;
  if (d->batch < 0 || d->num_blocks < 0 || d->max_blocks < 0 || d->rows < 0 || !block_size_ok(d->block_size)) return VSCAN_ERR_INVALID_ARG;
  if (!d->ring_state || !d->row_offset || !d->ring_state_out || !d->report) return VSCAN_ERR_INVALID_ARG;
  if (d->batch > 0 && (!d->past_len || !d->new_len || !d->kv_len)) return VSCAN_ERR_INVALID_ARG;
  if (d->batch > 0 && d->max_blocks > 0 && !d->block_table) return VSCAN_ERR_INVALID_ARG;
  if (d->num_blocks > 0 && !d->free_ring) return VSCAN_ERR_INVALID_ARG;
  // lengths are 32 bits: a table for more than 2^31 - 1 tokens could not be filled
  if (d->batch > kMaxBatch || static_cast<int64_t>(d->max_blocks) * d->block_size > 0x7fffffff) return VSCAN_ERR_UNSUPPORTED;
  struct Rng { const void* p; size_t n; };
  const size_t B = d->batch;
  const Rng all[] = {{d->past_len, B * 4}, {d->new_len, B * 4}, {d->ring_state, 16}, {d->block_table, B * d->max_blocks * 4},
                     {d->free_ring, static_cast<size_t>(d->num_blocks) * 4}, {d->kv_len, B * 4}, {d->row_offset, (B + 1) * 4},
                     {d->slot_map, static_cast<size_t>(d->rows) * 8}, {d->row_pos, static_cast<size_t>(d->rows) * 4},
                     {d->ring_state_out, 16}, {d->report, 16}};
  constexpr int kInputs = 3;
  for (const Rng& r : all)
    if (r.p && !aligned16(r.p)) return VSCAN_ERR_INVALID_ARG;
  for (int o = kInputs; o < 11; ++o)
    for (int i = 0; i < o; ++i)
      if (overlaps(all[o].p, all[o].n, all[i].p, all[i].n)) return VSCAN_ERR_INVALID_ARG;
  return VSCAN_OK;
}

}  // namespace kv
}  // namespace vscan

using namespace vscan;

extern "C" vscan_status vscan_kv_plan(const vscan_kv_plan_desc* d, void* stream_) {
  const vscan_status st = kv::validate_plan(d);
  if (st != VSCAN_OK) return st;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  kv::PlanParams p = {d->batch, d->block_size, 0, d->num_blocks, d->max_blocks, d->rows, d->past_len, d->new_len, d->block_table,
                      d->free_ring, d->ring_state, d->kv_len, d->row_offset, d->slot_map, d->row_pos, d->ring_state_out, d->report};
  while ((1 << p.shift) < p.block_size) ++p.shift;
  // as many CTAs as the rows (four a thread) or the table rows (a warp each) can use, at most one per SM: each repeats
  // the prefix sums
  const long long by_rows = !d->slot_map && !d->row_pos ? 0 : (static_cast<long long>(d->rows) + kv::kPlanThreads * kv::kPlanRows - 1) / (kv::kPlanThreads * kv::kPlanRows);
  const long long by_batch = (static_cast<long long>(d->batch) + 7) / 8;
  long long grid = by_rows > by_batch ? by_rows : by_batch;
  grid = grid < 1 ? 1 : grid > 148 ? 148 : grid;
  const size_t smem = (3 * static_cast<size_t>(d->batch) + 1) * sizeof(int);
  VSCAN_CUDA_TRY(allow_smem(kv::plan_kernel, smem));
  prof_before("kv_plan", stream);
  VSCAN_CUDA_TRY(launch_dependent(kv::plan_kernel, dim3(static_cast<unsigned>(grid)), dim3(kv::kPlanThreads), smem, stream, p));
  prof_after(stream);
  VSCAN_AFTER_LAUNCH();
  return VSCAN_OK;
}
