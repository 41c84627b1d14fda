// vscan_kv_weigh: attention weights gathered for each cached token and KV head.
//
// exp(scale q k - lse) needs no maximum and no sum of its own: every token's sum over the query rows stands alone.  So the line of
// (sequence, head, 64 tokens) is cut into equal stretches as for the attention over few rows, but nothing is joined afterwards, and a token's
// weight is read and written once by the lane that owns it, in a fixed order of the rows.
// For bf16 queries scale log2(e) is one float32 (two for float32 queries), and lse log2(e) is for both: a weight is off by 2^-24 of the sizes of score
// and lse, times itself, beside the error of the product.
#include "kv_weigh_tc.cuh"

namespace vscan {
namespace kv {

// ---------------------------------------------------------------------------------------------- bf16 queries, few rows
// m16n8k16 products of 16 tokens x 8 rows as in the attention over few rows: codes from global memory straight into fragments.  More
// rows than the 8 NT of a pass (heads of more than 128 channels) take more passes over the worker's tokens, which L2 holds by then.
// Bound by the codes' bytes: 256 decode steps, 196 to 301 tokens, 32 heads of 128, 277 MB: 67 us, 4.1 TB/s; one step of 701 tokens 6.7 us.
template <int KV, int DP, int NT, bool FULL>
__global__ void __launch_bounds__(kMmaThreads, DP == 256 ? 3 : NT > 1 ? 4 : 6) weigh_mma_kernel(WeighParams p) {
  constexpr int R = 8 * NT, KS = DP / 16, kPieces = DP / 64;
  __shared__ ScheduleShared sched;
  __shared__ Stretch stretches[kMmaThreads / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const int D = FULL ? DP : p.head_dim;
  grid_dependency_wait();
  Stretch& st = stretches[warp];
  {
    const Stretch found = locate<kMmaThreads, true>(p, sched);
    if (lane == 0) st = found;
    __syncwarp();
  }
  const bool solo = st.solo;
  const size_t cell_bytes = static_cast<size_t>(p.block_size) * D;
  while (true) {
    Piece pc = {0, 0};
    __syncwarp();
    if (lane == 0) next_piece(p, st, pc);
    __syncwarp();
    pc.u0 = __shfl_sync(0xffffffffu, pc.u0, 0);
    pc.u1 = __shfl_sync(0xffffffffu, pc.u1, 0);
    if (pc.u1 == 0) break;
    const Sequence& s = st.s;
    const int b = st.b, head = st.head, n_rows = window_rows(p, s);
    const int32_t* table = p.block_table + static_cast<size_t>(b) * p.max_blocks;
    const int stop = min(s.len, pc.u1 * kUnit);
    const int t_first = pc.u0 * kUnit + (solo ? 0 : warp * 16), t_stride = solo ? 16 : 64;
    for (int r0 = 0; r0 < n_rows; r0 += R) {
      const bool first_pass = r0 == 0;
      int blk, blk_next;
      float ks, old = 0.f;
      uint4 kraw[2][kPieces];
      auto block_of = [&](int t) {
        int x = -1;
        if (t < stop) {
          x = table[t >> p.shift];
          if (x < 0 || x >= p.num_blocks) x = -1;
        }
        return x;
      };
      auto load = [&](int t) {
        const bool full = FULL && t + 16 <= stop && blk >= 0;
        const size_t cell = static_cast<size_t>(max(blk, 0)) * p.kv_heads + head;
        const uint8_t* base = p.k_cache + cell * cell_bytes + ((t & (p.block_size - 1)) + g) * D + c * 16;
        ks = 0.f;
        if (blk >= 0) ks = __ldg(p.k_scale + cell);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < kPieces; ++i) {
            if (full) {
              kraw[h][i] = ld_nc_16(base + h * 8 * D + i * 64);
            } else {
              kraw[h][i] = make_uint4(0, 0, 0, 0);
              if (blk >= 0 && t + 8 * h + g < stop && i * 64 + c * 16 < D) kraw[h][i] = ld_nc_16(base + h * 8 * D + i * 64);
            }
          }
        const int mine = t + g + 8 * c;                   // lanes 0, 1 of four own a token each
        if (c < 2 && blk >= 0 && mine < stop && (!first_pass || mine < s.start)) old = *weight_at(p, blk, head, mine);
      };
      blk = block_of(t_first);
      load(t_first);
      blk_next = block_of(t_first + t_stride);

      // ---- queries: fragments of rows r0 + g of each tile, scaled by a power of two; what a score is multiplied by
      uint32_t qf[KS][NT][2];
      float cq[NT][2], lse[NT][2];
      int seen[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int r = r0 + nt * 8 + g;
        const WindowRow row = window_row(p, s, b, head, r);
        const char* src = q_at(p, b, s.first, row.at);
        uint4 raw[kPieces][2];
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            raw[i][k] = make_uint4(0, 0, 0, 0);
            if (r < n_rows && i * 64 + c * 16 < D) raw[i][k] = ld_nc_16(src + (i * 64 + c * 16) * 2 + k * 16);
            float f[8];
            Vec16<__nv_bfloat16>::unpack(raw[i][k], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(f[j]));
          }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int e = max(static_cast<int>(__float_as_uint(top) >> 23) - 127, -100);
        const float up = exp2_int(min(14 - e, 127)), down = exp2_int(max(e - 14, -126));
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float f[8];
            Vec16<__nv_bfloat16>::unpack(raw[i][k], f);
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              qf[i * 4 + k * 2 + w][nt][0] = pack_f16(f[4 * w] * up, f[4 * w + 1] * up);
              qf[i * 4 + k * 2 + w][nt][1] = pack_f16(f[4 * w + 2] * up, f[4 * w + 3] * up);
            }
          }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int from = (2 * c + k) * 4;
          cq[nt][k] = __shfl_sync(0xffffffffu, down, from) * p.scale_log2e;
          lse[nt][k] = __shfl_sync(0xffffffffu, row.lse, from);
          seen[nt][k] = __shfl_sync(0xffffffffu, row.seen, from);
        }
      }

      for (int t0 = t_first; t0 < stop; t0 += t_stride) {
        float x[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int k = 0; k < 4; ++k) x[nt][k] = 0.f;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          const uint32_t w0[4] = {kraw[0][i].x, kraw[0][i].y, kraw[0][i].z, kraw[0][i].w};
          const uint32_t w1[4] = {kraw[1][i].x, kraw[1][i].y, kraw[1][i].z, kraw[1][i].w};
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            uint32_t a[4];
            codes_to_f16<KV>(w0[w], a[0], a[2]);
            codes_to_f16<KV>(w1[w], a[1], a[3]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_f16(x[nt], a, qf[i * 4 + w][nt][0], qf[i * 4 + w][nt][1]);
          }
        }
        const int block = blk;
        const float ks_now = ks, before = old;
        old = 0.f;
        blk = blk_next;
        load(t0 + t_stride);
        blk_next = block_of(t0 + 2 * t_stride);
        float sum[2] = {0.f, 0.f};                        // of tokens t0 + g and t0 + g + 8
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float e = ex2(fmaf(x[nt][k], cq[nt][k & 1] * ks_now, -lse[nt][k & 1]));
            if (t0 + g + (k >> 1) * 8 < seen[nt][k & 1]) sum[k >> 1] += e;
          }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 1);
          sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 2);
        }
        const int mine = t0 + g + 8 * c;
        if (c < 2 && block >= 0 && mine < stop) {
          const float gain = c == 0 ? sum[0] : sum[1];
          *weight_at(p, block, head, mine) = first_pass ? (mine < s.start ? p.decay * before : 0.f) + gain : before + gain;
        }
      }
    }
  }
  grid_dependency_launch();
}

// ---------------------------------------------------------------------------------------------- float32 queries
// Products on the CUDA cores, a lane a token, R rows a pass; codes are read and decoded anew in each.  The exact kernel: for checking, and for models
// that run in float32.  256 decode steps, 196 to 301 tokens, 32 heads of 128, 277 MB: 127 us, 2.2 TB/s, bound by instructions (a lane reads a
// token's codes 16 bytes at a time); windows of 512 rows of 900 to 1,000 behind 15,000 tokens, twice, 28 / 4 heads (448 passes): 10.1 ms, 12 TFLOP/s.
template <int KV, int R>
__global__ void __launch_bounds__(128) weigh_fma_kernel(WeighParams p) {
  __shared__ __align__(16) float q_sh[R][256];
  __shared__ ScheduleShared sched;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = p.head_dim;
  grid_dependency_wait();
  Stretch st = locate<128, false>(p, sched);
  const size_t cell_bytes = static_cast<size_t>(p.block_size) * D;
  Piece pc;
  while (next_piece(p, st, pc)) {
    const Sequence& s = st.s;
    const int b = st.b, head = st.head, n_rows = window_rows(p, s);
    const int32_t* table = p.block_table + static_cast<size_t>(b) * p.max_blocks;
    const int stop = min(s.len, pc.u1 * kUnit);
    for (int r0 = 0; r0 < n_rows; r0 += R) {
      __syncthreads();                              // the rows of the pass before are done with
      for (int i = threadIdx.x; i < R * D; i += 128) {
        const int r = i / D, c = i - r * D;
        float v = 0.f;
        if (r0 + r < n_rows) v = reinterpret_cast<const float*>(q_at(p, b, s.first, window_row(p, s, b, head, r0 + r).at))[c];
        q_sh[r][c] = v;
      }
      __syncthreads();
      int seen[R];
      float lse[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const WindowRow row = window_row(p, s, b, head, r0 + r);
        seen[r] = row.seen;
        lse[r] = row.lse;
      }
      for (int t = pc.u0 * kUnit + warp * 32 + lane; t < stop; t += 128) {
        const int block = table[t >> p.shift];
        if (block < 0 || block >= p.num_blocks) continue;
        float* at = weight_at(p, block, head, t);
        float w = 0.f;
        if (r0 > 0) w = *at;
        else if (t < s.start) w = p.decay * *at;
        const size_t cell = static_cast<size_t>(block) * p.kv_heads + head;
        const uint8_t* key = p.k_cache + cell * cell_bytes + static_cast<size_t>(t & (p.block_size - 1)) * D;
        const float ks = p.k_scale[cell];
        float dot[R], odd[R];                       // two chains of sums
#pragma unroll
        for (int r = 0; r < R; ++r) dot[r] = odd[r] = 0.f;
        for (int c = 0; c < D; c += 16) {
          const uint4 raw = ld_nc_16(key + c);
          const uint32_t words[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            float f[4];
            decode4<KV>(words[k], f);
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const float4 qv = *reinterpret_cast<const float4*>(&q_sh[r][c + 4 * k]);
              float& d = (k & 1) ? odd[r] : dot[r];
              d = fmaf(qv.x, f[0], fmaf(qv.y, f[1], fmaf(qv.z, f[2], fmaf(qv.w, f[3], d))));
            }
          }
        }
        float gain = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float sum = dot[r] + odd[r], hi = ks * p.scale_log2e;
          // (infinity times a rest of the other sign, or of 0, would make a NaN of an infinite score)
          const float lo = fabsf(sum) < INFINITY ? sum * (ks * p.scale_rest) : 0.f;
          if (t < seen[r]) gain += ex2(fmaf(sum, hi, lo - lse[r]));
        }
        *at = w + gain;
      }
    }
  }
  grid_dependency_launch();
}

// ---------------------------------------------------------------------------------------------- host side
static vscan_status validate_weigh(const vscan_kv_weigh_desc* d) {
  if (!d) return VSCAN_ERR_INVALID_ARG;
  if (d->dtype != VSCAN_F32 && d->dtype != VSCAN_BF16) return VSCAN_ERR_INVALID_ARG;
  if (d->kv_dtype != VSCAN_KV_E4M3 && d->kv_dtype != VSCAN_KV_I8) return VSCAN_ERR_INVALID_ARG;
  if (d->batch < 0 || d->q_heads <= 0 || d->kv_heads <= 0 || d->q_heads % d->kv_heads || d->head_dim <= 0 || d->head_dim % 16 ||
      d->num_blocks < 0 || d->max_blocks < 0 || d->rows < 0 || d->max_q_len < 0 || d->window < 1 || !block_size_ok(d->block_size))
    return VSCAN_ERR_INVALID_ARG;
  if (d->scale - d->scale != 0.f || d->decay - d->decay != 0.f) return VSCAN_ERR_INVALID_ARG;
  if (d->batch == 0 || d->rows == 0 || d->max_q_len == 0 || d->num_blocks == 0 || d->max_blocks == 0) return VSCAN_OK;
  if (!d->q || !d->lse || !d->kv_len || !d->row_offset || !d->block_table || !d->k_cache || !d->k_scale || !d->weight) return VSCAN_ERR_INVALID_ARG;
  if (d->head_dim > 256 || d->q_heads / d->kv_heads > 64 || d->batch > kMaxBatch || d->kv_heads > 65535 ||
      static_cast<int64_t>(d->max_blocks) * d->block_size > 0x7ffff000 || static_cast<int64_t>(d->rows) * d->q_heads > 0x7ffff000)
    return VSCAN_ERR_UNSUPPORTED;
  const size_t e = dtype_bytes(d->dtype), B = d->batch, H = d->kv_heads, pool = static_cast<size_t>(d->num_blocks) * H;
  const bool padded = d->padded != 0;
  if (!strides_ok(d->q_stride, e, padded)) return VSCAN_ERR_INVALID_ARG;
  for (int i = padded ? 0 : 1; i < 3; ++i)
    if (d->lse_stride[i] < 0 || d->lse_stride[i] > (int64_t{1} << 40)) return VSCAN_ERR_INVALID_ARG;
  struct Rng { const void* p; size_t n; };
  const Rng all[] = {{d->q, rows_extent(d->q_stride, B, d->q_heads, d->rows, d->head_dim, e, padded)},
                     {d->lse, rows_extent(d->lse_stride, B, d->q_heads, d->rows, 1, 4, padded)}, {d->kv_len, B * 4}, {d->row_offset, (B + 1) * 4},
                     {d->block_table, B * d->max_blocks * 4}, {d->k_cache, pool * d->block_size * d->head_dim}, {d->k_scale, pool * 4},
                     {d->weight, pool * d->block_size * 4}};
  constexpr int kInputs = 7;
  for (const Rng& r : all)
    if (!aligned16(r.p)) return VSCAN_ERR_INVALID_ARG;
  for (int i = 0; i < kInputs; ++i)
    if (overlaps(all[kInputs].p, all[kInputs].n, all[i].p, all[i].n)) return VSCAN_ERR_INVALID_ARG;
  return VSCAN_OK;
}

// CTAs of a launch: as many as fit the SMs at once, no more than there can be units
static unsigned weigh_ctas(const WeighParams& p, int per_sm) {
  const int64_t units = (static_cast<int64_t>(p.max_blocks) * p.block_size + kUnit - 1) / kUnit, segments = static_cast<int64_t>(p.batch) * p.kv_heads;
  const int64_t most = 148 * per_sm;
  return static_cast<unsigned>(segments <= most / units ? segments * units : most);
}

template <int KV, int DP, bool FULL>
static vscan_status launch_weigh_mma(const WeighParams& p, int rows, cudaStream_t stream) {
  prof_before("kv_weigh_mma", stream);
  if (rows <= 8 || DP > 128)
    VSCAN_CUDA_TRY(launch_dependent(weigh_mma_kernel<KV, DP, 1, FULL>, dim3(weigh_ctas(p, DP == 256 ? 3 : 6)), dim3(kMmaThreads), 0, stream, p));
  else
    VSCAN_CUDA_TRY(launch_dependent(weigh_mma_kernel<KV, DP, (DP > 128 ? 1 : 2), FULL>, dim3(weigh_ctas(p, 4)), dim3(kMmaThreads), 0, stream, p));
  prof_after(stream);
  VSCAN_AFTER_LAUNCH();
  return VSCAN_OK;
}

template <int KV, int DP>
static vscan_status launch_weigh_tc(const WeighParams& p, const CUtensorMap& q, cudaStream_t stream) {
  constexpr size_t smem = 1024 + (wt_tiles(DP) + wt_stages(DP)) * static_cast<size_t>(DP / 64) * kChunk;
  VSCAN_CUDA_TRY(allow_smem(weigh_tc_kernel<KV, DP>, smem));
  prof_before("kv_weigh_tc", stream);
  VSCAN_CUDA_TRY(launch_dependent(weigh_tc_kernel<KV, DP>, dim3(weigh_ctas(p, 1)), dim3(kWtThreads), smem, stream, p, q));
  prof_after(stream);
  VSCAN_AFTER_LAUNCH();
  return VSCAN_OK;
}

template <int KV>
static vscan_status launch_weigh(const WeighParams& p, int dtype, const CUtensorMap* q, cudaStream_t stream) {
  const int64_t used = p.max_q_len < p.window ? p.max_q_len : p.window;
  const int rows = static_cast<int>(used * p.group < (1 << 20) ? used * p.group : 1 << 20), d = p.head_dim;
  if (q)
    return d <= 64 ? launch_weigh_tc<KV, 64>(p, *q, stream) : d <= 128 ? launch_weigh_tc<KV, 128>(p, *q, stream)
           : d <= 192 ? launch_weigh_tc<KV, 192>(p, *q, stream) : launch_weigh_tc<KV, 256>(p, *q, stream);
  if (dtype == VSCAN_BF16) {
    if (d == 64) return launch_weigh_mma<KV, 64, true>(p, rows, stream);
    if (d == 128) return launch_weigh_mma<KV, 128, true>(p, rows, stream);
    if (d == 256) return launch_weigh_mma<KV, 256, true>(p, rows, stream);
    return d < 64 ? launch_weigh_mma<KV, 64, false>(p, rows, stream)
                  : d < 128 ? launch_weigh_mma<KV, 128, false>(p, rows, stream) : launch_weigh_mma<KV, 256, false>(p, rows, stream);
  }
  prof_before("kv_weigh_fma", stream);
  const dim3 grid(weigh_ctas(p, 4));
  VSCAN_CUDA_TRY(rows <= 1 ? launch_dependent(weigh_fma_kernel<KV, 1>, grid, dim3(128), 0, stream, p)
                           : launch_dependent(weigh_fma_kernel<KV, 8>, grid, dim3(128), 0, stream, p));
  prof_after(stream);
  VSCAN_AFTER_LAUNCH();
  return VSCAN_OK;
}

}  // namespace kv
}  // namespace vscan

using namespace vscan;

extern "C" vscan_status vscan_kv_weigh(const vscan_kv_weigh_desc* d, void* stream_) {
  const vscan_status st = kv::validate_weigh(d);
  if (st != VSCAN_OK) return st;
  if (d->batch == 0 || d->rows == 0 || d->max_q_len == 0 || d->num_blocks == 0 || d->max_blocks == 0) return VSCAN_OK;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  const long long e = static_cast<long long>(dtype_bytes(d->dtype));
  kv::WeighParams p = {};
  p.q = static_cast<const char*>(d->q); p.lse = const_cast<float*>(d->lse);
  p.q_seq = d->q_stride[0] * e; p.q_head = d->q_stride[1] * e; p.q_row = d->q_stride[2] * e;
  p.l_seq = d->lse_stride[0]; p.l_head = d->lse_stride[1]; p.l_row = d->lse_stride[2];
  p.kv_len = d->kv_len; p.row_offset = d->row_offset; p.block_table = d->block_table;
  p.k_cache = static_cast<const uint8_t*>(d->k_cache); p.k_scale = d->k_scale; p.weight = d->weight;
  p.batch = d->batch; p.q_heads = d->q_heads; p.kv_heads = d->kv_heads; p.group = d->q_heads / d->kv_heads;
  p.head_dim = d->head_dim; p.block_size = d->block_size; p.num_blocks = d->num_blocks; p.max_blocks = d->max_blocks;
  p.rows = d->rows; p.padded = d->padded ? 1 : 0; p.max_q_len = d->max_q_len; p.causal = d->causal ? 1 : 0;
  p.window = d->window; p.decay = d->decay;
  while ((1 << p.shift) < p.block_size) ++p.shift;
  const double factor = static_cast<double>(d->scale) * 1.4426950408889634074;
  p.scale_log2e = static_cast<float>(factor);
  p.scale_rest = static_cast<float>(factor - p.scale_log2e);
  // 5th-generation tensor cores from 65 query rows of a sequence and KV head on (49 above 128 channels), where TMA takes the rows: a tile of that
  // kernel costs the same with 17 rows as with 128, while the other one takes a pass of 16 rows (8 above 128 channels) after the other over
  // codes that L2 holds after the first.  Microseconds, passes / tiles, 28 / 4 heads of 128: 16 x 2,000 tokens: 16 / 41 at 28 rows, 28 / 41 at 49,
  // 34 / 42 at 70, 47 / 42 at 98, 59 / 48 at 133, 109 / 56 at 259; 256 x 300: 36 / 125 at 28, 80 / 125 at 70, 110 / 126 at 98, 257 / 176 at 259; one
  // of 1,000: 9 / 11 at 28, 14 / 11 at 49, 18 / 11 at 70, 53 / 15 at 259.  32 heads, 16,000 tokens: 80 / 139 at 64, 152 / 126 at 128; 256 x 300: 330 /
  // 959 at 64, 651 / 900 at 128, 1,302 / 1,044 at 256 (short sequences of many heads would cross later than this, one short one earlier).  14 / 2 heads
  // of 256, 16 x 2,000: 35 / 50 at 35, 47 / 50 at 49, 60 / 50 at 70.  Windows of 3,584 rows, twice: 1,857 / 214.
  CUtensorMap map;
  const int64_t used = d->max_q_len < d->window ? d->max_q_len : d->window;
  const int64_t sizes[2] = {d->q_heads, d->rows}, steps[2] = {d->q_stride[1], d->q_stride[2]};
  const bool tensor = d->dtype == VSCAN_BF16 && used * p.group > (d->head_dim > 128 ? 48 : 64) &&
                      kv::rows_map(d->q, d->head_dim, sizes, steps, d->padded ? d->batch : 1, d->q_stride[0], p.group, 128 / p.group, &map);
  return d->kv_dtype == VSCAN_KV_E4M3 ? kv::launch_weigh<VSCAN_KV_E4M3>(p, d->dtype, tensor ? &map : nullptr, stream)
                                      : kv::launch_weigh<VSCAN_KV_I8>(p, d->dtype, tensor ? &map : nullptr, stream);
}
