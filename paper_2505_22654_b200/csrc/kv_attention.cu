// vscan_kv_attention: softmax(scale * q K^T) V over the paged 8-bit cache.
//
// One pass over the keys with a running maximum and sum per query row.  K and V are turned from codes in registers, the
// block's scale goes onto the scores (K) and onto the weights (V).  Queries of the heads that share a KV head, and of
// neighbouring new rows, form a tile, so that a key that was read once serves all of them.
#include "attention_join.cuh"
#include "kv_attention_tc.cuh"

namespace vscan {
namespace kv {

// ---------------------------------------------------------------------------------------------- float32 kernel
// Products on the CUDA cores: no rounding of queries or weights to 16 bits.  A warp takes 32 neighbouring tokens at a time:
// for the scores a lane owns a token, for the weighted sum a lane owns 4 or 8 channels.  Bound by its loads (a lane's key
// comes 16 bytes at a time, a row of the cache apart from its neighbour's) and by instructions, about four a code for one row.
// Measured: 256 sequences of 195 to 300 tokens, 32 heads of 128, 522 MB: 302 us, 1.7 TB/s; 4 of 9,000 to 16,500 tokens, 28 / 4
// heads, 44 MB: 78 us.  Keys kept in L1 for their second half: 290 and 89 us.  2 x 200 new rows behind 4,000 tokens, 28 / 4 heads: 1.27 ms.
constexpr int kFmaThreads = 128;
constexpr int kFmaWarps = kFmaThreads / 32;

template <typename T, int KV, int R>
__global__ void __launch_bounds__(kFmaThreads) fma_kernel(AttnParams p) {
  extern __shared__ __align__(16) float attn_smem[];
  const int D = p.head_dim;
  float* q_sh = attn_smem;                       // [R][D]
  float* w_sh = q_sh + R * D;                    // [warps][32][R] weights
  float* o_sh = w_sh + kFmaWarps * 32 * R;       // [warps][R][D]
  float* m_sh = o_sh + kFmaWarps * R * D;        // [warps][R]
  float* l_sh = m_sh + kFmaWarps * R;            // [warps][R]
  __shared__ ScheduleShared sched;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  grid_dependency_wait();
  if (blockIdx.x == 0 && threadIdx.x == 0) { p.status[0] = kStatusFlags | gridDim.x; p.status[1] = 0; }
  Stretch st = locate<kFmaThreads, false>(p, sched);
  if (threadIdx.x == 0) { p.boundary[blockIdx.x].seg1 = 0; p.flags[blockIdx.x] = 0; }
  bool bad = false;
  Piece pc;
  while (next_piece(p, st, pc)) {
    const Sequence& s = st.s;
    const int b = st.b, head = st.head, tile = st.tile, u0 = pc.u0, u1 = pc.u1;
    const int n_rows = min(R, s.n * p.group - tile * R);
    if (u0 > 0 && threadIdx.x == 0) p.boundary[blockIdx.x] = {st.seg0, st.seg0 + s.units, st.quota, b, head, tile, s.first, n_rows, 0};
    if (p.kv_len[b] > s.len) bad = true;

    __syncthreads();                              // the shared buffers of the segment before are done with
    for (int i = threadIdx.x; i < R * D; i += kFmaThreads) {
      const int r = i / D, c = i - r * D;
      float v = 0.f;
      if (r < n_rows) v = to_float<T>(reinterpret_cast<const T*>(q_at(p, b, s.first, row_at(p, tile, head, r)))[c]);
      q_sh[i] = v;
    }
    __syncthreads();
    int seen[R];
    float m[R], l[R], acc[R][8];
    int most = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      seen[r] = r < n_rows ? visible(p, s, row_at(p, tile, head, r).i) : 0;
      most = max(most, seen[r]);
      m[r] = -INFINITY; l[r] = 0.f;
#pragma unroll
      for (int c = 0; c < 8; ++c) acc[r][c] = 0.f;
    }
    const int stop = min(most, u1 * kUnit);
    const int32_t* table = p.block_table + static_cast<size_t>(b) * p.max_blocks;
    const size_t cell_bytes = static_cast<size_t>(p.block_size) * D;
    float* w_mine = w_sh + warp * 32 * R;
    for (int t0 = u0 * kUnit + warp * 32; t0 < stop; t0 += kFmaWarps * 32) {
      const int t = t0 + lane;
      int block = -1;
      if (t < stop) {
        block = table[t >> p.shift];
        if (block < 0 || block >= p.num_blocks) { block = -1; bad = true; }
      }
      const size_t cell = static_cast<size_t>(max(block, 0)) * p.kv_heads + head;
      float dot[R], odd[R];                       // two chains of sums
#pragma unroll
      for (int r = 0; r < R; ++r) dot[r] = odd[r] = 0.f;
      float ks = 0.f, vsc = 0.f;
      if (block >= 0) {
        ks = p.k_scale[cell]; vsc = p.v_scale[cell];
        const uint8_t* key = p.k_cache + cell * cell_bytes + static_cast<size_t>(t & (p.block_size - 1)) * D;
        for (int c = 0; c < D; c += 16) {
          const uint4 raw = ld_nc_16(key + c);
          const uint32_t words[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            float f[4];
            decode4<KV>(words[k], f);
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const float4 qv = *reinterpret_cast<const float4*>(q_sh + r * D + c + 4 * k);
              float& d = (k & 1) ? odd[r] : dot[r];
              d = fmaf(qv.x, f[0], fmaf(qv.y, f[1], fmaf(qv.z, f[2], fmaf(qv.w, f[3], d))));
            }
          }
        }
      }
      __syncwarp();
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const bool on = block >= 0 && t < seen[r];
        // the factor in two floats and the maximum taken off before the rounding: a weight near 1 is off by the exponential's
        // error and the dot product's, not by the rounding of a large score
        const float sum = dot[r] + odd[r], hi = ks * p.scale_log2e, lo = sum * (ks * p.scale_rest);
        const float x = on ? fmaf(sum, hi, lo) : -INFINITY;
        const float top = fmaxf(m[r], warp_max(x)), base = top == -INFINITY ? 0.f : top;
        const float e = on ? ex2(fmaf(sum, hi, lo - base)) : 0.f;
        if (top != m[r]) {
          const float f = ex2(m[r] - base);
          l[r] *= f;
#pragma unroll
          for (int c = 0; c < 8; ++c) acc[r][c] *= f;
          m[r] = top;
        }
        l[r] += e;
        w_mine[lane * R + r] = on ? e * vsc : 0.f;
      }
      __syncwarp();
#pragma unroll 1
      for (int half = 0; half < 2; ++half) {      // 16 neighbouring tokens lie in one block
        const int first = t0 + half * 16, count = min(16, stop - first);
        const int blk = __shfl_sync(0xffffffffu, block, half * 16);
        if (count <= 0 || blk < 0) continue;
        const uint8_t* value = p.v_cache + (static_cast<size_t>(blk) * p.kv_heads + head) * cell_bytes +
                               static_cast<size_t>(first & (p.block_size - 1)) * D;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          const int c = (part * 32 + lane) * 4;
          if (c < D) {
#pragma unroll 4
            for (int j = 0; j < count; ++j) {
              float f[4];
              decode4<KV>(__ldg(reinterpret_cast<const uint32_t*>(value + static_cast<size_t>(j) * D + c)), f);
#pragma unroll
              for (int r = 0; r < R; ++r) {
                const float e = w_mine[(half * 16 + j) * R + r];
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[r][part * 4 + k] = fmaf(e, f[k], acc[r][part * 4 + k]);
              }
            }
          }
        }
      }
    }
    // ---- the warps' shares of the segment are joined
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float sum = warp_sum(l[r]);
      if (lane == 0) { m_sh[warp * R + r] = m[r]; l_sh[warp * R + r] = sum; }
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        const int c = (part * 32 + lane) * 4;
        if (c < D) *reinterpret_cast<float4*>(o_sh + (warp * R + r) * D + c) =
                       make_float4(acc[r][part * 4], acc[r][part * 4 + 1], acc[r][part * 4 + 2], acc[r][part * 4 + 3]);
      }
    }
    __syncthreads();
    const bool complete = u0 == 0 && u1 == s.units;
    float* part = p.partial + (static_cast<size_t>(blockIdx.x) * 2 + (u0 == 0 ? 1 : 0)) * partial_floats(R, D);
    for (int i = threadIdx.x; i < n_rows * D; i += kFmaThreads) {
      const int r = i / D, c = i - r * D;
      float top = -INFINITY;
#pragma unroll
      for (int k = 0; k < kFmaWarps; ++k) top = fmaxf(top, m_sh[k * R + r]);
      const float base = top == -INFINITY ? 0.f : top;
      float o = 0.f, den = 0.f;
#pragma unroll
      for (int k = 0; k < kFmaWarps; ++k) {
        const float f = ex2(m_sh[k * R + r] - base);
        o = fmaf(f, o_sh[(k * R + r) * D + c], o);
        den = fmaf(f, l_sh[k * R + r], den);
      }
      if (complete) {
        const RowAt at = row_at(p, tile, head, r);
        store_out<T>(out_at(p, b, s.first, at), c, den == 0.f ? 0.f : o / den);
        if (c == 0 && p.lse) *lse_at(p, b, s.first, at) = den == 0.f ? -INFINITY : (top + log2f(den)) * 0.69314718055994531f;
      } else {
        part[r * D + c] = o;
        if (c == 0) { part[R * D + r] = top; part[R * D + R + r] = den; }
      }
    }
  }
  if (bad) p.flags[blockIdx.x] = VSCAN_ERR_INVALID_ARG;
  grid_dependency_launch();
}

// ---------------------------------------------------------------------------------------------- host side
constexpr int64_t kMostTokens = 0x7ffff000;   // a step or a tile more still fits 32 bits

static vscan_status validate_attention(const vscan_kv_attention_desc* d) {
  if (!d) return VSCAN_ERR_INVALID_ARG;
  if (d->dtype != VSCAN_F32 && d->dtype != VSCAN_BF16) return VSCAN_ERR_INVALID_ARG;
  if (d->kv_dtype != VSCAN_KV_E4M3 && d->kv_dtype != VSCAN_KV_I8) return VSCAN_ERR_INVALID_ARG;
  if (d->batch < 0 || d->q_heads <= 0 || d->kv_heads <= 0 || d->q_heads % d->kv_heads || d->head_dim <= 0 || d->head_dim % 16 ||
      d->num_blocks < 0 || d->max_blocks < 0 || d->rows < 0 || d->max_q_len < 0 || !block_size_ok(d->block_size))
    return VSCAN_ERR_INVALID_ARG;
  if (!(d->scale == d->scale) || d->scale - d->scale != 0.f) return VSCAN_ERR_INVALID_ARG;
  if (d->batch == 0 || d->rows == 0 || d->max_q_len == 0) return VSCAN_OK;
  const bool cache = d->num_blocks > 0 && d->max_blocks > 0;
  if (!d->q || !d->out || !d->kv_len || !d->row_offset) return VSCAN_ERR_INVALID_ARG;
  if (cache && (!d->block_table || !d->k_cache || !d->v_cache || !d->k_scale || !d->v_scale)) return VSCAN_ERR_INVALID_ARG;
  if (d->head_dim > 256 || d->q_heads / d->kv_heads > 64 || d->batch > kMaxBatch || d->kv_heads > 65535 ||
      static_cast<int64_t>(d->max_blocks) * d->block_size > kMostTokens || static_cast<int64_t>(d->rows) * d->q_heads > kMostTokens)
    return VSCAN_ERR_UNSUPPORTED;
  const size_t e = dtype_bytes(d->dtype), B = d->batch, H = d->kv_heads;
  const bool padded = d->padded != 0;
  if (!strides_ok(d->q_stride, e, padded) || !strides_ok(d->out_stride, e, padded)) return VSCAN_ERR_INVALID_ARG;
  if (d->lse)
    for (int i = padded ? 0 : 1; i < 3; ++i)
      if (d->lse_stride[i] < 0 || d->lse_stride[i] > (int64_t{1} << 40)) return VSCAN_ERR_INVALID_ARG;
  const int64_t sizes[3] = {padded ? d->batch : 1, d->q_heads, d->rows};
  if (!strides_apart(d->out_stride, sizes, 3, d->head_dim) || (d->lse && !strides_apart(d->lse_stride, sizes, 3, 1))) return VSCAN_ERR_INVALID_ARG;
  struct Rng { const void* p; size_t n; };
  const size_t pool = static_cast<size_t>(d->num_blocks) * H;
  const Rng all[] = {{d->q, rows_extent(d->q_stride, B, d->q_heads, d->rows, d->head_dim, e, padded)},
                     {d->kv_len, B * 4}, {d->row_offset, (B + 1) * 4}, {d->block_table, B * d->max_blocks * 4},
                     {d->k_cache, pool * d->block_size * d->head_dim}, {d->v_cache, pool * d->block_size * d->head_dim},
                     {d->k_scale, pool * 4}, {d->v_scale, pool * 4},
                     {d->out, rows_extent(d->out_stride, B, d->q_heads, d->rows, d->head_dim, e, padded)},
                     {d->lse, d->lse ? rows_extent(d->lse_stride, B, d->q_heads, d->rows, 1, 4, padded) : 0}};
  constexpr int kInputs = 8;
  for (const Rng& r : all)
    if (r.p && !aligned16(r.p)) return VSCAN_ERR_INVALID_ARG;
  for (int o = kInputs; o < 10; ++o)
    for (int i = 0; i < o; ++i)
      if (overlaps(all[o].p, all[o].n, all[i].p, all[i].n)) return VSCAN_ERR_INVALID_ARG;
  return VSCAN_OK;
}

// Rows of a tile and CTAs of the launch
struct Plan { int tile_rows; unsigned ctas; bool mma, tensor; };

static Plan plan_launch(const vscan_kv_attention_desc* d) {
  Plan pl;
  const int group = d->q_heads / d->kv_heads;
  const int64_t want = static_cast<int64_t>(group) * d->max_q_len;
  pl.mma = d->dtype == VSCAN_BF16;
  // 5th-generation tensor cores from 17 query rows of a sequence and KV head on: below that the other kernel reads the cache
  // once as well
  pl.tensor = pl.mma && want > 16 && d->head_dim <= 128;
  int64_t resident;
  if (pl.tensor) {
    pl.tile_rows = kTcRows;
    resident = 1;
  } else if (pl.mma) {
    pl.tile_rows = want <= 8 || d->head_dim > 128 ? 8 : 16;   // 16 rows of 256 channels do not fit the registers
    resident = d->head_dim > 128 || pl.tile_rows > 8 ? 2 : 4;
  } else {
    pl.tile_rows = want <= 1 ? 1 : want <= 2 ? 2 : want <= 4 ? 4 : 8;
    resident = pl.tile_rows > 4 ? 2 : 4;   // 8 rows take 243 to 254 registers of 128 threads
  }
  // as many CTAs as fit the SMs at once, no more than there can be units
  const int64_t rows = d->padded ? static_cast<int64_t>(d->batch) * (d->rows < d->max_q_len ? d->rows : d->max_q_len) : d->rows;
  const int64_t tiles = rows * group / pl.tile_rows + d->batch;
  const int64_t units = (static_cast<int64_t>(d->max_blocks) * d->block_size + kUnit - 1) / kUnit;
  int64_t most = 148 * resident;
  if (units < 1) { if (tiles * d->kv_heads < most) most = tiles * d->kv_heads; }
  else if (tiles * d->kv_heads <= most / units) most = tiles * d->kv_heads * units;
  pl.ctas = static_cast<unsigned>(most < 1 ? 1 : most);
  return pl;
}

// workspace: status word | a flag per CTA | boundaries | partial results
static size_t flag_bytes(const Plan& pl) { return round_up(pl.ctas * sizeof(uint32_t), 256); }
static size_t workers(const Plan& pl) { return static_cast<size_t>(pl.ctas) * (pl.mma && !pl.tensor ? kWorkersPerCta : 1); }
static size_t boundary_bytes(const Plan& pl) { return round_up(workers(pl) * sizeof(Boundary), 256); }

static size_t fma_smem(int R, int D) { return (static_cast<size_t>(R) * D * (1 + kFmaWarps) + kFmaWarps * 32 * R + 2 * kFmaWarps * R) * 4; }

template <typename T, int KV>
static vscan_status launch_fma(const AttnParams& p, const Plan& pl, cudaStream_t stream) {
  const size_t smem = fma_smem(pl.tile_rows, p.head_dim);
#define VSCAN_FMA_CASE(R)                                                                                           \
  if (pl.tile_rows == R) {                                                                                          \
    VSCAN_CUDA_TRY(allow_smem(fma_kernel<T, KV, R>, smem));                                                         \
    prof_before("kv_attention_fma", stream);                                                                        \
    VSCAN_CUDA_TRY(launch_dependent(fma_kernel<T, KV, R>, dim3(pl.ctas), dim3(kFmaThreads), smem, stream, p));      \
    prof_after(stream);                                                                                             \
    VSCAN_AFTER_LAUNCH();                                                                                           \
  }
  VSCAN_FMA_CASE(1)
  VSCAN_FMA_CASE(2)
  VSCAN_FMA_CASE(4)
  VSCAN_FMA_CASE(8)
#undef VSCAN_FMA_CASE
  return VSCAN_OK;
}

template <int KV, int DP, bool FULL>
static vscan_status launch_mma(const AttnParams& p, const Plan& pl, cudaStream_t stream) {
  const size_t smem = (static_cast<size_t>(4) * pl.tile_rows * (DP + 2)) * sizeof(float);
  constexpr int MT = 1;
#define VSCAN_MMA_CASE(NT)                                                                                          \
  if (pl.tile_rows == 8 * NT) {                                                                                     \
    auto kernel = mma_kernel<KV, DP, NT, MT, FULL>;                                                                 \
    VSCAN_CUDA_TRY(allow_smem(kernel, smem));                                                                       \
    prof_before("kv_attention_mma", stream);                                                                        \
    VSCAN_CUDA_TRY(launch_dependent(kernel, dim3(pl.ctas), dim3(kMmaThreads), smem, stream, p));                    \
    prof_after(stream);                                                                                             \
    VSCAN_AFTER_LAUNCH();                                                                                           \
  }
  VSCAN_MMA_CASE(1)
  if constexpr (DP <= 128) { VSCAN_MMA_CASE(2) }
#undef VSCAN_MMA_CASE
  return VSCAN_OK;
}

template <int KV, int DP>
static vscan_status launch_tc(const AttnParams& p, const Plan& pl, cudaStream_t stream) {
  constexpr size_t smem = 1024 + 6 * static_cast<size_t>(DP / 64) * kChunk;
  VSCAN_CUDA_TRY(allow_smem(tc_kernel<KV, DP>, smem));
  prof_before("kv_attention_tc", stream);
  VSCAN_CUDA_TRY(launch_dependent(tc_kernel<KV, DP>, dim3(pl.ctas), dim3(kTcThreads), smem, stream, p));
  prof_after(stream);
  VSCAN_AFTER_LAUNCH();
  return VSCAN_OK;
}

template <typename T, int KV>
static vscan_status launch_scores(const AttnParams& p, const Plan& pl, cudaStream_t stream) {
  if constexpr (sizeof(T) == 2) {
    const int d = p.head_dim;
    if (pl.tensor) return d <= 64 ? launch_tc<KV, 64>(p, pl, stream) : launch_tc<KV, 128>(p, pl, stream);
    if (d == 64) return launch_mma<KV, 64, true>(p, pl, stream);
    if (d == 128) return launch_mma<KV, 128, true>(p, pl, stream);
    if (d == 256) return launch_mma<KV, 256, true>(p, pl, stream);
    return d < 64 ? launch_mma<KV, 64, false>(p, pl, stream) : d < 128 ? launch_mma<KV, 128, false>(p, pl, stream)
                                                                       : launch_mma<KV, 256, false>(p, pl, stream);
  }
  else return launch_fma<T, KV>(p, pl, stream);
}

template <typename T>
static vscan_status launch_attention(const AttnParams& p, const Plan& pl, int kv_dtype, cudaStream_t stream) {
  const vscan_status st = kv_dtype == VSCAN_KV_E4M3 ? launch_scores<T, VSCAN_KV_E4M3>(p, pl, stream) : launch_scores<T, VSCAN_KV_I8>(p, pl, stream);
  if (st != VSCAN_OK) return st;
  // nothing can have been cut when the table has room for kWhole units only (many rows: kTcWhole steps), or when one CTA did
  // it all
  if (static_cast<int64_t>(p.max_blocks) * p.block_size <= (pl.tensor ? kTcWhole * kTcKeys : kWhole * kUnit) || pl.ctas == 1) return VSCAN_OK;
  prof_before("kv_attention_join", stream);
  const dim3 grid = pl.tensor ? dim3(pl.ctas, kTcRows / kJoinRows) : dim3((pl.ctas + kJoinLook - 1) / kJoinLook);
  static_assert(kJoinWarps == kJoinLook * kWorkersPerCta, "as many boundaries a CTA whichever the workers are");
  VSCAN_CUDA_TRY(launch_dependent(join_kernel<T>, grid, dim3(kJoinThreads), 0, stream, p, static_cast<int>(pl.ctas)));
  prof_after(stream);
  VSCAN_AFTER_LAUNCH();
  return VSCAN_OK;
}

}  // namespace kv
}  // namespace vscan

using namespace vscan;

extern "C" size_t vscan_kv_attention_workspace_bytes(const vscan_kv_attention_desc* d) {
  if (!d || d->batch <= 0 || d->rows <= 0 || d->max_q_len <= 0 || d->q_heads <= 0 || d->kv_heads <= 0 || d->head_dim <= 0 ||
      d->head_dim > 256 || d->q_heads / d->kv_heads > 64)
    return kStatusBytes;
  const kv::Plan pl = kv::plan_launch(d);
  return kStatusBytes + kv::flag_bytes(pl) + kv::boundary_bytes(pl) + round_up(2 * kv::workers(pl) * kv::partial_floats(pl.tile_rows, d->head_dim) * 4, 256);
}

extern "C" vscan_status vscan_kv_attention(const vscan_kv_attention_desc* d, void* workspace, size_t workspace_bytes, void* stream_) {
  const vscan_status st = kv::validate_attention(d);
  if (st != VSCAN_OK) return st;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  if (!workspace || !aligned256(workspace) || workspace_bytes < vscan_kv_attention_workspace_bytes(d)) return VSCAN_ERR_WORKSPACE;
  if (d->batch == 0 || d->rows == 0 || d->max_q_len == 0) {
    VSCAN_CUDA_TRY(cudaMemsetAsync(workspace, 0, sizeof(uint32_t), stream));
    return VSCAN_OK;
  }
  const kv::Plan pl = kv::plan_launch(d);
  const long long e = static_cast<long long>(dtype_bytes(d->dtype));
  char* ws = static_cast<char*>(workspace);
  kv::AttnParams p = {};
  p.q = static_cast<const char*>(d->q); p.out = static_cast<char*>(d->out); p.lse = d->lse;
  p.q_seq = d->q_stride[0] * e; p.q_head = d->q_stride[1] * e; p.q_row = d->q_stride[2] * e;
  p.o_seq = d->out_stride[0] * e; p.o_head = d->out_stride[1] * e; p.o_row = d->out_stride[2] * e;
  p.l_seq = d->lse_stride[0]; p.l_head = d->lse_stride[1]; p.l_row = d->lse_stride[2];
  p.kv_len = d->kv_len; p.row_offset = d->row_offset; p.block_table = d->block_table;
  p.k_cache = static_cast<const uint8_t*>(d->k_cache); p.v_cache = static_cast<const uint8_t*>(d->v_cache);
  p.k_scale = d->k_scale; p.v_scale = d->v_scale;
  p.batch = d->batch; p.q_heads = d->q_heads; p.kv_heads = d->kv_heads; p.group = d->q_heads / d->kv_heads;
  p.head_dim = d->head_dim; p.block_size = d->block_size; p.num_blocks = d->num_blocks;
  p.max_blocks = d->num_blocks > 0 ? d->max_blocks : 0;
  p.rows = d->rows; p.padded = d->padded ? 1 : 0; p.max_q_len = d->max_q_len; p.causal = d->causal ? 1 : 0;
  while ((1 << p.shift) < p.block_size) ++p.shift;
  p.tile_rows = pl.tile_rows;
  const double factor = static_cast<double>(d->scale) * 1.4426950408889634074;
  p.scale_log2e = static_cast<float>(factor);
  p.scale_rest = static_cast<float>(factor - p.scale_log2e);
  p.status = reinterpret_cast<uint32_t*>(ws);
  ws += kStatusBytes;
  p.flags = reinterpret_cast<uint32_t*>(ws);
  ws += kv::flag_bytes(pl);
  p.boundary = reinterpret_cast<kv::Boundary*>(ws);
  p.partial = reinterpret_cast<float*>(ws + kv::boundary_bytes(pl));
  return d->dtype == VSCAN_F32 ? kv::launch_attention<float>(p, pl, d->kv_dtype, stream)
                               : kv::launch_attention<__nv_bfloat16>(p, pl, d->kv_dtype, stream);
}
