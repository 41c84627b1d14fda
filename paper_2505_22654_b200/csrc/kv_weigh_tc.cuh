// Attention weights of many query rows (the window of a prompt) for bf16 queries on the 5th-generation tensor cores.
//
// A CTA takes 256 tokens of one KV head as two tiles of 128, turned from codes to bf16 (exactly) once, and runs over all query rows of the window,
// a tile of up to 128 (whole tokens of the group's heads) at a time:
//   warps 0-7, 8-15  tile 0, 1: two threads a token, 64 of the rows each.  S^T [128 tokens x 128 rows] from tensor memory, exponentials, their sum
//                    in registers: nothing goes back but one number a token at the end.  Before that, the tile's codes into shared memory
//   warp 16          issues the products: two buffers of scores a tile, so that they run beside the exponentials
//   warp 17          the rows' queries by TMA, a ring of four tiles
//   warp 18          the rows' logarithms, beside them
// Bound by the exponentials: 32,768 a tile of rows, 16 a cycle, twice what the products take.  Two prompts' windows of 512 rows of 900 to 1,024
// behind 15,000 to 16,000 tokens, 28 / 4 heads of 128 (118 GFLOP, 102 us of exponentials): 214 us (351 with a thread a token and masks
// everywhere; 1,857 as m16n8k16 products in passes of 16 rows).
// Heads of more than 128 channels: one tile of tokens, and fewer tiles of queries in the ring.  The same windows at 256 channels: 334 us.
// Every wait is bounded; on expiry the CTA's tokens keep the weights that they had (there is no workspace to say so in).
#pragma once

#include "kv_weigh.cuh"
#include "tc_rows.cuh"

namespace vscan {
namespace kv {

constexpr int kWtThreads = 640, kWtIssuer = 16, kWtLoader = 17, kWtLogs = 18;
constexpr int kWtStages = 4;
// Tiles of tokens of a CTA, and of queries in the ring: what 192 KB hold
__host__ __device__ constexpr int wt_tiles(int dp) { return dp > 128 ? 1 : 2; }
__host__ __device__ constexpr int wt_stages(int dp) { return dp > 192 ? 2 : dp > 128 ? 3 : kWtStages; }

struct WtShared {
  uint64_t k_full[2], s_full[2][2], s_empty[2][2], other[2][4];   // other: of the two warps that share 32 tokens
  uint64_t q_full[kWtStages], q_empty[kWtStages], log_full[kWtStages], log_empty[kWtStages];
  uint32_t tmem_base;
  int abort_flag;
  alignas(16) float log[kWtStages][128];      // minus the rows' logarithms in base 2; -inf where a row gives nothing
  int silent[kWtStages];                      // some row of the tile gives nothing
  float part[2][128];                         // sums of the second threads
  ScheduleShared sched;
};

// What a piece of a stretch is cut into: the CTA's 256 (or 128) tokens from t0 on, against the rows' tiles first .. tiles - 1
struct WtChunk { int t0, n, first, tiles, row0, rows; };      // row0, rows: tokens of the window, the first as a row of the sequence

__device__ __forceinline__ WtChunk wt_chunk(const WeighParams& p, const Sequence& s, int t0, int stop, int per_tile, int tokens) {
  WtChunk c;
  c.t0 = t0;
  c.n = min(stop - t0, tokens);
  c.rows = min(s.n, p.window);
  c.row0 = s.n - c.rows;
  c.tiles = (c.rows + per_tile - 1) / per_tile;
  // rows in front of token t0 do not see it
  const long long unseen = p.causal ? t0 - s.start - c.row0 : 0;
  c.first = static_cast<int>(min(max(unseen, 0ll) / per_tile, static_cast<long long>(c.tiles)));
  return c;
}

template <int KV, int DP>
__global__ void __launch_bounds__(kWtThreads, 1) weigh_tc_kernel(WeighParams p, const __grid_constant__ CUtensorMap q_map) {
  using namespace tc;
  constexpr int kDChunks = DP / 64, kTileBytes = kDChunks * kChunk, kTiles = wt_tiles(DP), kTokens = kTiles * 128, kStages = wt_stages(DP);
  extern __shared__ unsigned char smem_dyn[];
  __shared__ WtShared sh;
  unsigned char* base = smem_dyn + ((1024u - (smem_u32(smem_dyn) & 1023u)) & 1023u);
  unsigned char* k_sh = base;                      // [tiles]
  unsigned char* q_sh = k_sh + kTiles * kTileBytes;     // [stages]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int D = p.head_dim;
  volatile int* abort_flag = &sh.abort_flag;

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.k_full[i], 8);
      for (int k = 0; k < 2; ++k) { mbar_init(&sh.s_full[i][k], 1); mbar_init(&sh.s_empty[i][k], 8); }
      for (int k = 0; k < 4; ++k) mbar_init(&sh.other[i][k], 1);
    }
    for (int i = 0; i < kStages; ++i) { mbar_init(&sh.q_full[i], 1); mbar_init(&sh.q_empty[i], 1); mbar_init(&sh.log_full[i], 1); mbar_init(&sh.log_empty[i], 16); }
    sh.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // rows of a stage behind the whole tokens of a tile are never loaded: their scores have to be finite
  for (int i = threadIdx.x; i < kStages * kDChunks * 128 * 8; i += kWtThreads) {
    const int row = (i >> 3) & 127;
    if (row >= 128 / p.group * p.group) *reinterpret_cast<uint4*>(q_sh + static_cast<size_t>(i >> 10) * kChunk + (i & 1023) * 16) = make_uint4(0, 0, 0, 0);
  }
  fence_async();
  if (warp == kWtIssuer) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)), "n"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem_base;              // scores of tile t, buffer i at column 256 t + 128 i
  grid_dependency_wait();
  Stretch st = locate<kWtThreads, false>(p, sh.sched);
  Piece pc;
  const int per_tile = 128 / p.group;              // tokens of a tile of rows
  bool ok = true;

  if (warp < kWtIssuer) {
    // ============================================================ two threads a token
    const int tile = warp >> 3, half = (warp >> 2) & 1, quarter = warp & 3, r = quarter * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
    int n_it = 0, n_row = 0, n_sum = 0;            // tiles of rows that this tile has had; of the CTA; sums told so far
    while (ok && next_piece(p, st, pc)) {
      const int stop = min(st.s.len, pc.u1 * kUnit);
      for (int t0 = pc.u0 * kUnit; t0 < stop && ok; t0 += kTokens) {
        const WtChunk c = wt_chunk(p, st.s, t0, stop, per_tile, kTokens);
        if (tile * 128 >= c.n) {                   // nothing for this tile
          for (int j = c.first; j < c.tiles && ok; ++j, ++n_row) {
            ok = mbar_wait_warp(&sh.log_full[n_row % kStages], (n_row / kStages) & 1, abort_flag);
            if (ok && lane == 0) mbar_arrive(&sh.log_empty[n_row % kStages]);
          }
          continue;
        }
        const int t = t0 + tile * 128 + r;
        int block = -1;
        if (t < stop) {
          block = p.block_table[static_cast<size_t>(st.b) * p.max_blocks + (t >> p.shift)];
          if (block < 0 || block >= p.num_blocks) block = -1;
        }
        float factor = 0.f, sum = 0.f;
        float* weight = nullptr;
        if (block >= 0) {
          factor = __ldg(p.k_scale + static_cast<size_t>(block) * p.kv_heads + st.head) * p.scale_log2e;
          weight = weight_at(p, block, st.head, t);
          if (half == 0 && t < st.s.start) sum = p.decay * *weight;
        }
        if (c.first == c.tiles) {                  // no row of the window sees any of the tokens (rows that are not there would)
          if (weight && half == 0) *weight = sum;
          continue;
        }
        // ---- codes to bf16 into the tile (whose products before are done: this warp has read their scores); rows of the group of
        // lanes that has a token's pieces in turn
        {
          constexpr int kPer = DP / 16;                                  // pieces of 16 codes of a token
#pragma unroll
          for (int i = half * 16 * kPer + lane; i < (half + 1) * 16 * kPer; i += 32) {
            const int row = i / kPer, piece = i % kPer, mine = quarter * 32 + row, tok = t0 + tile * 128 + mine;
            const int blk = __shfl_sync(0xffffffffu, block, row);
            uint4 raw = make_uint4(0, 0, 0, 0);
            if (blk >= 0 && piece * 16 < D)
              raw = ld_nc_16(p.k_cache + ((static_cast<size_t>(blk) * p.kv_heads + st.head) * p.block_size + (tok & (p.block_size - 1))) * D + piece * 16);
            const uint32_t words[4] = {raw.x, raw.y, raw.z, raw.w};
            uint32_t h[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              float f[4];
              decode4<KV>(words[k], f);
              const __nv_bfloat162 lo = __floats2bfloat162_rn(f[0], f[1]), hi = __floats2bfloat162_rn(f[2], f[3]);
              h[2 * k] = *reinterpret_cast<const uint32_t*>(&lo);
              h[2 * k + 1] = *reinterpret_cast<const uint32_t*>(&hi);
            }
            unsigned char* at = k_sh + tile * kTileBytes + (piece >> 2) * kChunk + mine * 128;
            const int c16 = (piece & 3) * 2;
            *reinterpret_cast<uint4*>(at + ((c16 ^ (mine & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
            *reinterpret_cast<uint4*>(at + (((c16 + 1) ^ (mine & 7)) << 4)) = make_uint4(h[4], h[5], h[6], h[7]);
          }
          fence_async();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.k_full[tile]);
        }
        // ---- rows that see the token: from this one of the window on
        const long long from = p.causal ? max(t - st.s.start - c.row0, 0ll) : 0;
        // tiles of rows from this one on see all of the warp's tokens, up to the last one, which may have fewer rows
        const int clear = __reduce_max_sync(0xffffffffu, static_cast<int>(min((from + per_tile - 1) / per_tile, static_cast<long long>(c.tiles))));
        const int full = c.rows / per_tile;
        uint64_t sums[2] = {0, 0};
        const uint64_t mul = pair(factor, factor);
#pragma unroll 1
        for (int j = c.first; j < c.tiles && ok; ++j, ++n_it, ++n_row) {
          const int stage = n_row % kStages, buf = n_it & 1;
          ok = mbar_wait_warp(&sh.log_full[stage], (n_row / kStages) & 1, abort_flag) &&
               mbar_wait_warp(&sh.s_full[tile][buf], (n_it >> 1) & 1, abort_flag);
          if (!ok) break;
          tc_fence_after();
          const float* log = sh.log[stage];
          const bool masked = j < clear || j >= full || sh.silent[stage];
          const uint32_t s_addr = tmem + lanes + tile * 256 + buf * 128;
#pragma unroll 1
          for (int q = 2 * half; q < 2 * half + 2; ++q) {
            uint32_t v[32];
            tmem_read32(s_addr + q * 32, v);
            float e[32];
#pragma unroll
            for (int k = 0; k < 32; k += 4) {
              const float4 z = *reinterpret_cast<const float4*>(log + q * 32 + k);
              const float2 a = unpair(fma2(pair(__uint_as_float(v[k]), __uint_as_float(v[k + 1])), mul, pair(z.x, z.y)));
              const float2 b = unpair(fma2(pair(__uint_as_float(v[k + 2]), __uint_as_float(v[k + 3])), mul, pair(z.z, z.w)));
              e[k] = ex2(a.x); e[k + 1] = ex2(a.y); e[k + 2] = ex2(b.x); e[k + 3] = ex2(b.y);
            }
            if (masked) {                            // columns of the tile that count
              const int c0 = static_cast<int>(min(max(from - static_cast<long long>(j) * per_tile, 0ll), 128ll)) * p.group;
              const int c1 = min(c.rows - j * per_tile, per_tile) * p.group;
#pragma unroll
              for (int k = 0; k < 32; ++k)
                if (q * 32 + k < c0 || q * 32 + k >= c1 || log[q * 32 + k] == -INFINITY) e[k] = 0.f;
            }
#pragma unroll
            for (int k = 0; k < 32; k += 4) {
              sums[0] = add2(sums[0], pair(e[k], e[k + 1]));
              sums[1] = add2(sums[1], pair(e[k + 2], e[k + 3]));
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) { mbar_arrive(&sh.s_empty[tile][buf]); mbar_arrive(&sh.log_empty[stage]); }
        }
        const float2 a = unpair(sums[0]), b = unpair(sums[1]);
        sum += (a.x + a.y) + (b.x + b.y);
        if (!ok) break;
        if (half == 1) {
          sh.part[tile][r] = sum;
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.other[tile][quarter]);
        } else {
          ok = mbar_wait_warp(&sh.other[tile][quarter], n_sum++ & 1, abort_flag);
          if (ok && weight) *weight = sum + sh.part[tile][r];
        }
      }
    }
  } else if (warp == kWtIssuer) {
    // ============================================================ products
    const uint32_t idesc = idesc_bf16(128, false), k_addr = smem_u32(k_sh), q_addr = smem_u32(q_sh);
    int n_it[2] = {0, 0}, n_chunk[2] = {0, 0}, n_row = 0;
    while (ok && next_piece(p, st, pc)) {
      const int stop = min(st.s.len, pc.u1 * kUnit);
      for (int t0 = pc.u0 * kUnit; t0 < stop && ok; t0 += kTokens) {
        const WtChunk c = wt_chunk(p, st.s, t0, stop, per_tile, kTokens);
        const int two = c.n > 128;                 // never where a CTA has one tile
#pragma unroll
        for (int t = 0; t < 2; ++t)
          if (t <= two && c.first < c.tiles && ok) ok = mbar_wait_warp(&sh.k_full[t], n_chunk[t]++ & 1, abort_flag);
        for (int j = c.first; j < c.tiles && ok; ++j, ++n_row) {
          const int stage = n_row % kStages;
          ok = mbar_wait_warp(&sh.q_full[stage], (n_row / kStages) & 1, abort_flag);
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (t > two || !ok) continue;
            const int buf = n_it[t] & 1;
            if (n_it[t] >= 2) ok = mbar_wait_warp(&sh.s_empty[t][buf], ((n_it[t] >> 1) - 1) & 1, abort_flag);
            if (!ok) continue;
            tc_fence_after();
            const uint64_t a = smem_desc_sw128(k_addr + t * kTileBytes), b = smem_desc_sw128(q_addr + stage * kTileBytes);
#pragma unroll
            for (int d = 0; d < kDChunks; ++d) umma_f16_ss_x4(tmem + t * 256 + buf * 128, a + d * (kChunk >> 4), b + d * (kChunk >> 4), idesc, d > 0);
            umma_commit_warp(&sh.s_full[t][buf]);
            ++n_it[t];
          }
          if (ok) umma_commit_warp(&sh.q_empty[stage]);
        }
      }
    }
    __syncwarp();
  } else if (warp == kWtLoader || warp == kWtLogs) {
    // ============================================================ queries; logarithms
    int n_row = 0, token_of[4], head_of[4];        // of rows lane, lane + 32, ... of a tile
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      token_of[i] = (i * 32 + lane) / p.group;
      head_of[i] = i * 32 + lane - token_of[i] * p.group;
    }
    while (ok && next_piece(p, st, pc)) {
      const int stop = min(st.s.len, pc.u1 * kUnit);
      for (int t0 = pc.u0 * kUnit; t0 < stop && ok; t0 += kTokens) {
        const WtChunk c = wt_chunk(p, st.s, t0, stop, per_tile, kTokens);
        for (int j = c.first; j < c.tiles && ok; ++j, ++n_row) {
          const int stage = n_row % kStages, token = c.row0 + j * per_tile;
          uint64_t* empty = warp == kWtLoader ? &sh.q_empty[stage] : &sh.log_empty[stage];
          if (n_row >= kStages) ok = mbar_wait_warp(empty, (n_row / kStages - 1) & 1, abort_flag);
          if (!ok) break;
          if (warp == kWtLoader) {
            if (lane == 0) {
              mbar_arrive_expect_tx(&sh.q_full[stage], kDChunks * per_tile * p.group * 128);
#pragma unroll
              for (int d = 0; d < kDChunks; ++d)
                tma_load_4d(q_sh + stage * kTileBytes + d * kChunk, &q_map, &sh.q_full[stage], d * 64, st.head * p.group, st.s.first + token, p.padded ? st.b : 0);
            }
          } else {
            bool silent = false;
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              x[i] = INFINITY;
              if (token_of[i] < per_tile && j * per_tile + token_of[i] < c.rows)
                x[i] = __ldg(lse_at(p, st.b, st.s.first, RowAt{token + token_of[i], st.head * p.group + head_of[i]}));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (x[i] == -INFINITY) { x[i] = INFINITY; silent = true; }
              sh.log[stage][i * 32 + lane] = x[i] * -1.44269504088896341f;
            }
            silent = __any_sync(0xffffffffu, silent);
            __syncwarp();
            if (lane == 0) { sh.silent[stage] = silent; mbar_arrive(&sh.log_full[stage]); }
          }
          __syncwarp();
        }
      }
    }
  }

  // ------------------------------------------------------------ teardown
  tc_fence_before();
  __syncthreads();
  if (sh.abort_flag) {
    for (int i = 0; i < 64; ++i) __nanosleep(2000);   // products and copies still in flight end before their memory is given back
    __syncthreads();
  }
  if (warp == kWtIssuer) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
  }
}

}  // namespace kv
}  // namespace vscan
