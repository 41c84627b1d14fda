// vscan_attention: softmax(scale * q K^T) V of packed or padded sequences, K and V in the queries' own type.
//
// The division of the work, and the join of what it cuts, are those of the attention over the paged cache: a line of tiles of query
// rows (new rows x heads of a group, so that a key that was read serves all of them) against steps of keys, in equal stretches.
#include "attention_join.cuh"
#include "attention_tc.cuh"

#include <type_traits>

namespace vscan {
namespace kv {

// ---------------------------------------------------------------------------------------------- products on the CUDA cores
// float32 queries (no rounding of queries or weights to 16 bits), and bf16 where the other kernel does not go.  A CTA takes 64 query rows and
// 64 keys a step; a thread 4 x 4 scores, then 4 rows x DP / 16 channels of the sums.  The next step's keys are on
// their way while the weights meet the values, and the values while the scores are made.  Weights pass between the 16 threads of a row only.
// Four floats that lie together stay together; which four of a row lie where depends on the row, so that the rows that a warp reads at
// once lie in different banks, and two CTAs of 128 channels fit an SM.
// Bound by the instructions of the products and their operands from shared memory, which do not overlap in full with two CTAs an SM: 3 x 250 to
// 1,030 rows, 16 heads of 80, 4.1 GFLOP: 185 us; 1,500 to 2,000 rows: 28 TFLOP/s of 74 (23 without copies in the background).  8 rows a thread,
// or two sums to an instruction, gave the same.
constexpr int kFlatThreads = 256, kFlatRows = 64, kFlatKeys = 64, kFlatWhole = 4;
using FlatShape = TileShape<kFlatThreads, kFlatRows, kFlatKeys, kFlatWhole>;
template <int DP>
constexpr size_t flat_smem() { return (static_cast<size_t>(kFlatRows + 2 * kFlatKeys) * DP + kFlatRows * kFlatKeys) * 4; }

__device__ __forceinline__ void copy_16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(tc::smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All copies have arrived but those of the last N groups
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <typename T, int DP>
__global__ void __launch_bounds__(kFlatThreads, DP == 256 ? 1 : 2) flat_kernel(PromptParams p) {
  // a thread's channels: 4 of every 64, or 2 of every 32 (heads of 72 to 96)
  constexpr int kVec = DP == 96 ? 2 : 4, kChunks = DP / (16 * kVec), kEach = kFlatRows * 16 / kFlatThreads;   // kEach: rows of a thread
  extern __shared__ __align__(16) float flat_sh[];
  float* q_sh = flat_sh;                        // [rows][DP]
  float* k_sh = q_sh + kFlatRows * DP;          // [keys][DP]
  float* v_sh = k_sh + kFlatKeys * DP;          // [keys][DP]
  float* w_sh = v_sh + kFlatKeys * DP;          // [rows][keys]
  __shared__ DivisionShared division;
  const int tid = threadIdx.x, x = tid & 15, y = tid >> 4, D = p.head_dim;
  grid_dependency_wait();
  TcStretch st = tc_locate<FlatShape>(p, division);
  if (tid == 0) {
    if (blockIdx.x == 0) { p.status[0] = kStatusFlags | gridDim.x; p.status[1] = 0; }
    p.boundary[blockIdx.x].seg1 = 0;
    p.flags[blockIdx.x] = 0;
  }
  // A dot product whose score is -infinity, of weight 0 (the two parts of the factor would make a NaN of it where their signs differ or one is 0)
  const float gone = p.scale_log2e > 0.f ? -INFINITY : p.scale_log2e < 0.f ? INFINITY : __uint_as_float(0x7fc00000u);
  TcPiece pc;
  // Rows of a buffer as floats into shared memory, zeros beyond `there` rows; turn(r): what the places of a row's fours are xored with
  auto fill = [&](float* dst, int there, auto turn, auto at) {
    constexpr int kElems = Vec16<T>::kElems, kVecs = DP / kElems;
    for (int i = tid; i < 64 * kVecs; i += kFlatThreads) {
      const int r = i / kVecs, c = (i - r * kVecs) * kElems;
      if (c >= D) continue;
      float* row = dst + r * DP;
      if constexpr (sizeof(T) == 4) {
        float* to = row + (c ^ turn(r) * 4);
        if (r < there) copy_16(to, at(r) + c * 4);
        else *reinterpret_cast<float4*>(to) = make_float4(0.f, 0.f, 0.f, 0.f);
      } else {
        float f[kElems];
#pragma unroll
        for (int j = 0; j < kElems; ++j) f[j] = 0.f;
        if (r < there) Vec16<T>::unpack(ld_nc_16(at(r) + c * static_cast<int>(sizeof(T))), f);
#pragma unroll
        for (int j = 0; j < kElems; j += 4) *reinterpret_cast<float4*>(row + ((c + j) ^ turn(r) * 4)) = make_float4(f[j], f[j + 1], f[j + 2], f[j + 3]);
      }
    }
    copy_commit();
  };
  while (tc_next<FlatShape>(p, st, pc)) {
    const Sequence& s = pc.q.s;
    if (pc.u0 > 0 && tid == 0) p.boundary[blockIdx.x] = {pc.seg0, pc.seg1, st.quota, pc.b, pc.head, pc.tile, s.first, pc.n_rows, 0};
    int key0, keys;
    key_span(p, pc.b, key0, keys);
    const char* k = p.k + (p.padded ? pc.b * p.k_seq : key0 * p.k_row) + pc.head * p.k_head;
    const char* v = p.v + (p.padded ? pc.b * p.v_seq : key0 * p.v_row) + pc.head * p.v_head;
    auto row_of = [&](int r) {
      const int flat = pc.tile * kFlatRows + r, i = flat / p.group;
      return RowAt{i, pc.head * p.group + flat - i * p.group};
    };
    auto fill_keys = [&](int u) {
      fill(k_sh, min(pc.most - u * kFlatKeys, kFlatKeys), [](int r) { return r & 7; }, [&](int r) { return k + (u * kFlatKeys + r) * p.k_row; });
    };
    __syncthreads();                            // the buffers of the piece before are done with
    fill(q_sh, pc.n_rows, [](int r) { return r / kEach & 7; }, [&](int r) { return q_at(p, pc.b, s.first, row_of(r)); });
    fill_keys(pc.u0);
    int seen[kEach];
    float m[kEach], l[kEach];
    float o[kEach][kChunks * kVec];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int r = y * kEach + i;
      seen[i] = r < pc.n_rows ? visible(p, s, row_of(r).i) : 0;
      m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
      for (int c = 0; c < kChunks * kVec; ++c) o[i][c] = 0.f;
    }
    for (int u = pc.u0; u < pc.u1; ++u) {
      const int t0 = u * kFlatKeys, there = min(pc.most - t0, kFlatKeys);
      copy_wait<0>();
      __syncthreads();                          // queries and keys are there; values of the step before are done with
      fill(v_sh, there, [](int) { return 0; }, [&](int r) { return v + (t0 + r) * p.v_row; });
      float dot[kEach][4];                      // rows kEach y + i, keys x + 16 j
#pragma unroll
      for (int i = 0; i < kEach; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) dot[i][j] = 0.f;
#pragma unroll 2
      for (int c = 0; c < D; c += 4) {
        float4 b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = *reinterpret_cast<const float4*>(k_sh + (x + 16 * j) * DP + (c ^ (x & 7) * 4));
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          const float4 a = *reinterpret_cast<const float4*>(q_sh + (y * kEach + i) * DP + (c ^ (y & 7) * 4));
#pragma unroll
          for (int j = 0; j < 4; ++j) dot[i][j] = fmaf(a.x, b[j].x, dot[i][j]);
#pragma unroll
          for (int j = 0; j < 4; ++j) dot[i][j] = fmaf(a.y, b[j].y, dot[i][j]);
#pragma unroll
          for (int j = 0; j < 4; ++j) dot[i][j] = fmaf(a.z, b[j].z, dot[i][j]);
#pragma unroll
          for (int j = 0; j < 4; ++j) dot[i][j] = fmaf(a.w, b[j].w, dot[i][j]);
        }
      }
      __syncthreads();                          // keys are done with
      if (u + 1 < pc.u1) fill_keys(u + 1);
      else copy_commit();
      float* w_row = w_sh + y * kEach * kFlatKeys;      // of the thread's rows; places xored with w_turn
      const int w_turn = (y & 1) * 16;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        // the factor in two floats and the maximum taken off before the rounding: a weight near 1 is off by the exponential's error and
        // the dot product's, not by the rounding of a large score
        float top = m[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (t0 + x + 16 * j < seen[i]) top = fmaxf(top, fmaf(dot[i][j], p.scale_log2e, dot[i][j] * p.scale_rest));
        }
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
        const float base = top == -INFINITY ? 0.f : top, f = ex2(m[i] - base);
        if (top != m[i]) {
          l[i] *= f;
#pragma unroll
          for (int c = 0; c < kChunks * kVec; ++c) o[i][c] *= f;
          m[i] = top;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bool on = t0 + x + 16 * j < seen[i] && dot[i][j] != gone;
          const float e = on ? ex2(fmaf(dot[i][j], p.scale_log2e, fmaf(dot[i][j], p.scale_rest, -base))) : 0.f;
          l[i] += e;
          w_row[i * kFlatKeys + ((x + 16 * j) ^ w_turn)] = e;
        }
      }
      copy_wait<1>();
      __syncthreads();                          // values are there, and the weights
      // a row's own keys only: what lies in the others may be infinite
      int fewest = seen[0];
#pragma unroll
      for (int i = 1; i < kEach; ++i) fewest = min(fewest, seen[i]);
      fewest -= t0;
      auto add = [&](auto masked) {
#pragma unroll 2
        for (int t = 0; t < there; t += 4) {
          float w[kEach][4];
#pragma unroll
          for (int i = 0; i < kEach; ++i) {
            const float4 f = *reinterpret_cast<const float4*>(w_row + i * kFlatKeys + (t ^ w_turn));
            w[i][0] = f.x; w[i][1] = f.y; w[i][2] = f.z; w[i][3] = f.w;
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float f[kChunks * kVec];
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
              const float* from = v_sh + (t + j) * DP + (c * 16 + x) * kVec;
              if constexpr (kVec == 4) {
                const float4 four = *reinterpret_cast<const float4*>(from);
                f[4 * c] = four.x; f[4 * c + 1] = four.y; f[4 * c + 2] = four.z; f[4 * c + 3] = four.w;
              } else {
                const float2 two = *reinterpret_cast<const float2*>(from);
                f[2 * c] = two.x; f[2 * c + 1] = two.y;
              }
            }
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
              if (decltype(masked)::value && t0 + t + j >= seen[i]) continue;
#pragma unroll
              for (int c = 0; c < kChunks * kVec; ++c) o[i][c] = fmaf(w[i][j], f[c], o[i][c]);
            }
          }
        }
      };
      if (fewest >= there) add(std::false_type{});
      else add(std::true_type{});
    }
    const bool complete = pc.u0 == 0 && pc.u1 == pc.units;
    float* part = p.partial + (static_cast<size_t>(blockIdx.x) * 2 + (pc.u0 == 0 ? 1 : 0)) * partial_floats(kFlatRows, D);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      float sum = l[i];
#pragma unroll
      for (int off = 1; off < 16; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
      const int r = y * kEach + i;
      if (r >= pc.n_rows) continue;
      const RowAt at = row_of(r);
      char* out = out_at(p, pc.b, s.first, at);
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        const int ch = (c * 16 + x) * kVec;
        if (ch >= D) continue;
#pragma unroll
        for (int e = 0; e < kVec / 2; ++e) {
          const float2 both = make_float2(o[i][kVec * c + 2 * e], o[i][kVec * c + 2 * e + 1]);
          if (complete) {
            store_out<T>(out, ch + 2 * e, sum == 0.f ? 0.f : both.x / sum);
            store_out<T>(out, ch + 2 * e + 1, sum == 0.f ? 0.f : both.y / sum);
          } else {
            *reinterpret_cast<float2*>(part + static_cast<size_t>(r) * D + ch + 2 * e) = both;
          }
        }
      }
      if (x == 0) {
        if (!complete) { part[kFlatRows * D + r] = m[i]; part[kFlatRows * D + kFlatRows + r] = sum; }
        else if (p.lse) *lse_at(p, pc.b, s.first, at) = sum == 0.f ? -INFINITY : (m[i] + log2f(sum)) * 0.69314718055994531f;
      }
    }
  }
  grid_dependency_launch();
}

// ---------------------------------------------------------------------------------------------- host side
constexpr int64_t kMostRows = 0x7ffff000;   // a step or a tile more still fits 32 bits

static vscan_status validate_prompt(const vscan_attention_desc* d) {
  if (!d) return VSCAN_ERR_INVALID_ARG;
  if (d->dtype != VSCAN_F32 && d->dtype != VSCAN_BF16) return VSCAN_ERR_INVALID_ARG;
  if (d->batch < 0 || d->q_heads <= 0 || d->kv_heads <= 0 || d->q_heads % d->kv_heads || d->head_dim <= 0 || d->head_dim % 8 || d->rows < 0 ||
      d->kv_rows < 0 || d->max_q_len < 0)
    return VSCAN_ERR_INVALID_ARG;
  if (d->scale - d->scale != 0.f) return VSCAN_ERR_INVALID_ARG;
  if (d->batch == 0 || d->rows == 0 || d->max_q_len == 0) return VSCAN_OK;
  if (!d->q || !d->out || !d->row_offset || (d->kv_rows > 0 && (!d->k || !d->v))) return VSCAN_ERR_INVALID_ARG;
  if (d->head_dim > 256 || d->q_heads / d->kv_heads > 64 || d->batch > kMaxBatch || d->kv_heads > 65535 ||
      static_cast<int64_t>(d->rows) * d->q_heads > kMostRows || d->kv_rows > kMostRows)
    return VSCAN_ERR_UNSUPPORTED;
  const size_t e = dtype_bytes(d->dtype), B = d->batch;
  const bool padded = d->padded != 0;
  if (!strides_ok(d->q_stride, e, padded) || !strides_ok(d->out_stride, e, padded) || !strides_ok(d->k_stride, e, padded) ||
      !strides_ok(d->v_stride, e, padded))
    return VSCAN_ERR_INVALID_ARG;
  if (d->lse)
    for (int i = padded ? 0 : 1; i < 3; ++i)
      if (d->lse_stride[i] < 0 || d->lse_stride[i] > (int64_t{1} << 40)) return VSCAN_ERR_INVALID_ARG;
  const int64_t sizes[3] = {padded ? d->batch : 1, d->q_heads, d->rows};
  if (!strides_apart(d->out_stride, sizes, 3, d->head_dim) || (d->lse && !strides_apart(d->lse_stride, sizes, 3, 1))) return VSCAN_ERR_INVALID_ARG;
  struct Rng { const void* p; size_t n; };
  const Rng all[] = {{d->q, rows_extent(d->q_stride, B, d->q_heads, d->rows, d->head_dim, e, padded)},
                     {d->k, rows_extent(d->k_stride, B, d->kv_heads, d->kv_rows, d->head_dim, e, padded)},
                     {d->v, rows_extent(d->v_stride, B, d->kv_heads, d->kv_rows, d->head_dim, e, padded)},
                     {d->row_offset, (B + 1) * 4}, {d->kv_offset, (B + 1) * 4},
                     {d->out, rows_extent(d->out_stride, B, d->q_heads, d->rows, d->head_dim, e, padded)},
                     {d->lse, d->lse ? rows_extent(d->lse_stride, B, d->q_heads, d->rows, 1, 4, padded) : 0}};
  constexpr int kInputs = 5, kAll = 7;
  for (const Rng& r : all)
    if (r.p && !aligned16(r.p)) return VSCAN_ERR_INVALID_ARG;
  for (int o = kInputs; o < kAll; ++o)
    for (int i = 0; i < o; ++i)
      if (overlaps(all[o].p, all[o].n, all[i].p, all[i].n)) return VSCAN_ERR_INVALID_ARG;
  return VSCAN_OK;
}

// Rows of a tile, keys of a step, CTAs of the launch
struct PromptPlan { int tile_rows, keys, whole; unsigned ctas; };

// (a negative factor would turn the masks around: no model has one)
static bool prompt_tensor(const vscan_attention_desc* d) { return d->dtype == VSCAN_BF16 && d->kv_rows > 0 && d->scale >= 0.f; }

static PromptPlan plan_prompt(const vscan_attention_desc* d, bool tensor) {
  PromptPlan pl;
  const int group = d->q_heads / d->kv_heads;
  pl.tile_rows = tensor ? pt_tiles(d->head_dim) * (128 / group) * group : kFlatRows;      // whole tokens of the group's heads
  pl.keys = tensor ? kPtKeys : kFlatKeys;
  pl.whole = tensor ? kPtWhole : kFlatWhole;
  const int64_t resident = tensor || d->head_dim > 128 ? 1 : 2;
  // as many CTAs as fit the SMs at once, no more than there can be steps
  const int64_t rows = d->padded ? static_cast<int64_t>(d->batch) * (d->rows < d->max_q_len ? d->rows : d->max_q_len) : d->rows;
  const int64_t tiles = rows * group / pl.tile_rows + d->batch, steps = (static_cast<int64_t>(d->kv_rows) + pl.keys - 1) / pl.keys;
  int64_t most = 148 * resident;
  if (steps < 1) { if (tiles * d->kv_heads < most) most = tiles * d->kv_heads; }
  else if (tiles * d->kv_heads <= most / steps) most = tiles * d->kv_heads * steps;
  pl.ctas = static_cast<unsigned>(most < 1 ? 1 : most);
  return pl;
}

// workspace: status word | a flag per CTA | boundaries | partial results
static size_t prompt_flag_bytes(const PromptPlan& pl) { return round_up(pl.ctas * sizeof(uint32_t), 256); }
static size_t prompt_boundary_bytes(const PromptPlan& pl) { return round_up(pl.ctas * sizeof(Boundary), 256); }
static size_t prompt_bytes(const PromptPlan& pl, int head_dim) {
  return kStatusBytes + prompt_flag_bytes(pl) + prompt_boundary_bytes(pl) + round_up(2 * static_cast<size_t>(pl.ctas) * partial_floats(pl.tile_rows, head_dim) * 4, 256);
}

struct PromptMaps { CUtensorMap q, k, v; };
static bool prompt_maps(const vscan_attention_desc* d, PromptMaps& m) {
  const int group = d->q_heads / d->kv_heads;
  const int64_t q_sizes[2] = {d->q_heads, d->rows}, kv_sizes[2] = {d->kv_rows, d->kv_heads};
  const int64_t q_steps[2] = {d->q_stride[1], d->q_stride[2]}, k_steps[2] = {d->k_stride[2], d->k_stride[1]}, v_steps[2] = {d->v_stride[2], d->v_stride[1]};
  const int batch = d->padded ? d->batch : 1;
  return rows_map(d->q, d->head_dim, q_sizes, q_steps, batch, d->q_stride[0], group, 128 / group, &m.q) &&
         rows_map(d->k, d->head_dim, kv_sizes, k_steps, batch, d->k_stride[0], kPtKeys, 1, &m.k) &&
         rows_map(d->v, d->head_dim, kv_sizes, v_steps, batch, d->v_stride[0], kPtKeys, 1, &m.v);
}

template <int DP>
static vscan_status launch_prompt_tc(const PromptParams& p, const PromptPlan& pl, const PromptMaps& m, cudaStream_t stream) {
  constexpr size_t smem = 1024 + (pt_tiles(DP) + pt_stages(DP)) * static_cast<size_t>(DP / 64) * kChunk;
  VSCAN_CUDA_TRY(allow_smem(prompt_tc_kernel<DP>, smem));
  prof_before("attention_tc", stream);
  VSCAN_CUDA_TRY(launch_dependent(prompt_tc_kernel<DP>, dim3(pl.ctas), dim3(kPtThreads), smem, stream, p, m.q, m.k, m.v));
  prof_after(stream);
  VSCAN_AFTER_LAUNCH();
  return VSCAN_OK;
}

static vscan_status launch_prompt_tcs(const PromptParams& p, const PromptPlan& pl, const PromptMaps& m, cudaStream_t stream) {
  return p.head_dim <= 64 ? launch_prompt_tc<64>(p, pl, m, stream) : p.head_dim <= 128 ? launch_prompt_tc<128>(p, pl, m, stream)
         : p.head_dim <= 192 ? launch_prompt_tc<192>(p, pl, m, stream) : launch_prompt_tc<256>(p, pl, m, stream);
}

template <typename T, int DP>
static vscan_status launch_flat(const PromptParams& p, const PromptPlan& pl, cudaStream_t stream) {
  constexpr size_t smem = flat_smem<DP>();
  VSCAN_CUDA_TRY(allow_smem(flat_kernel<T, DP>, smem));
  prof_before("attention_flat", stream);
  VSCAN_CUDA_TRY(launch_dependent(flat_kernel<T, DP>, dim3(pl.ctas), dim3(kFlatThreads), smem, stream, p));
  prof_after(stream);
  VSCAN_AFTER_LAUNCH();
  return VSCAN_OK;
}

template <typename T>
static vscan_status launch_flats(const PromptParams& p, const PromptPlan& pl, cudaStream_t stream) {
  return p.head_dim <= 64 ? launch_flat<T, 64>(p, pl, stream) : p.head_dim <= 96 ? launch_flat<T, 96>(p, pl, stream) : p.head_dim <= 128 ? launch_flat<T, 128>(p, pl, stream) : launch_flat<T, 256>(p, pl, stream);
}

template <typename T>
static vscan_status launch_prompt_join(const PromptParams& p, const PromptPlan& pl, cudaStream_t stream) {
  // nothing can have been cut when no sequence has more keys than a tile that stays whole, or when one CTA did it all
  if (p.kv_rows <= pl.whole * pl.keys || pl.ctas == 1) return VSCAN_OK;
  prof_before("attention_join", stream);
  const int rows = join_rows(p.head_dim);
  const dim3 grid(pl.ctas, (pl.tile_rows + rows - 1) / rows);
  VSCAN_CUDA_TRY(launch_dependent(join_kernel<T>, grid, dim3(kJoinThreads), 0, stream, static_cast<const AttnParams&>(p), static_cast<int>(pl.ctas)));
  prof_after(stream);
  VSCAN_AFTER_LAUNCH();
  return VSCAN_OK;
}

}  // namespace kv
}  // namespace vscan

using namespace vscan;

extern "C" size_t vscan_attention_workspace_bytes(const vscan_attention_desc* d) {
  if (!d || d->batch <= 0 || d->rows <= 0 || d->max_q_len <= 0 || d->q_heads <= 0 || d->kv_heads <= 0 || d->head_dim <= 0 || d->head_dim > 256 ||
      d->q_heads % d->kv_heads || d->q_heads / d->kv_heads > 64 || d->kv_rows < 0)      // (sizes that the call refuses; a plan divides by the group)
    return kStatusBytes;
  const size_t flat = kv::prompt_bytes(kv::plan_prompt(d, false), d->head_dim);      // strides decide between the two
  const size_t tensor = d->dtype == VSCAN_BF16 ? kv::prompt_bytes(kv::plan_prompt(d, true), d->head_dim) : 0;
  return flat > tensor ? flat : tensor;
}

extern "C" vscan_status vscan_attention(const vscan_attention_desc* d, void* workspace, size_t workspace_bytes, void* stream_) {
  const vscan_status st = kv::validate_prompt(d);
  if (st != VSCAN_OK) return st;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  if (!workspace || !aligned256(workspace) || workspace_bytes < vscan_attention_workspace_bytes(d)) return VSCAN_ERR_WORKSPACE;
  if (d->batch == 0 || d->rows == 0 || d->max_q_len == 0) {
    VSCAN_CUDA_TRY(cudaMemsetAsync(workspace, 0, sizeof(uint32_t), stream));
    return VSCAN_OK;
  }
  kv::PromptMaps maps;
  const bool tensor = kv::prompt_tensor(d) && kv::prompt_maps(d, maps);
  const kv::PromptPlan pl = kv::plan_prompt(d, tensor);
  const long long e = static_cast<long long>(dtype_bytes(d->dtype));
  char* ws = static_cast<char*>(workspace);
  kv::PromptParams p = {};
  p.q = static_cast<const char*>(d->q); p.k = static_cast<const char*>(d->k); p.v = static_cast<const char*>(d->v);
  p.out = static_cast<char*>(d->out); p.lse = d->lse;
  p.q_seq = d->q_stride[0] * e; p.q_head = d->q_stride[1] * e; p.q_row = d->q_stride[2] * e;
  p.k_seq = d->k_stride[0] * e; p.k_head = d->k_stride[1] * e; p.k_row = d->k_stride[2] * e;
  p.v_seq = d->v_stride[0] * e; p.v_head = d->v_stride[1] * e; p.v_row = d->v_stride[2] * e;
  p.o_seq = d->out_stride[0] * e; p.o_head = d->out_stride[1] * e; p.o_row = d->out_stride[2] * e;
  p.l_seq = d->lse_stride[0]; p.l_head = d->lse_stride[1]; p.l_row = d->lse_stride[2];
  p.row_offset = d->row_offset; p.kv_offset = d->kv_offset ? d->kv_offset : d->row_offset;
  p.batch = d->batch; p.q_heads = d->q_heads; p.kv_heads = d->kv_heads; p.group = d->q_heads / d->kv_heads; p.head_dim = d->head_dim;
  p.rows = d->rows; p.kv_rows = d->kv_rows; p.padded = d->padded ? 1 : 0; p.max_q_len = d->max_q_len; p.causal = d->causal ? 1 : 0;
  p.tile_rows = pl.tile_rows;
  const double factor = static_cast<double>(d->scale) * 1.4426950408889634074;
  p.scale_log2e = static_cast<float>(factor);
  p.scale_rest = static_cast<float>(factor - p.scale_log2e);
  p.status = reinterpret_cast<uint32_t*>(ws);
  ws += kStatusBytes;
  p.flags = reinterpret_cast<uint32_t*>(ws);
  ws += kv::prompt_flag_bytes(pl);
  p.boundary = reinterpret_cast<kv::Boundary*>(ws);
  p.partial = reinterpret_cast<float*>(ws + kv::prompt_boundary_bytes(pl));
  const vscan_status done = tensor ? kv::launch_prompt_tcs(p, pl, maps, stream)
                            : d->dtype == VSCAN_F32 ? kv::launch_flats<float>(p, pl, stream) : kv::launch_flats<__nv_bfloat16>(p, pl, stream);
  if (done != VSCAN_OK) return done;
  return d->dtype == VSCAN_F32 ? kv::launch_prompt_join<float>(p, pl, stream) : kv::launch_prompt_join<__nv_bfloat16>(p, pl, stream);
}
