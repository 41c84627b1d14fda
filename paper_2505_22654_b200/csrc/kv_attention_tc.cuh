// Attention of many query rows (prompts, chunks) for bf16 queries on the 5th-generation tensor cores.
//
// A CTA takes 256 query rows (new rows x heads of a group) of one KV head as two tiles of 128 and runs over its stretch of
// the keys, 128 at a time:
//   warps 0-3, 4-7   one query row a thread of tile 0, 1: scores from tensor memory, running maximum and sum, weights back
//                    to tensor memory, over the scores that they come from; the results at the end
//   warps 8-11       K and V from codes to f16 in shared memory (128-byte swizzle), two stages each; a key that was turned
//                    once serves both tiles
//   warp 12          issues the products: S[128 x 128] = Q K^T (operands in shared memory), O[128 x d] += P V with P read
//                    from tensor memory and V, tokens down and channels across, as the MN-major operand
// The two tiles take turns: while one's weights are made, the other's products run.  Tensor memory is full: two tiles of
// scores and two of sums, 128 columns each.
//
// Roundings as in the kernel for few rows: queries exact in f16 but for a power of two, weights in f16 relative to a
// reference of the V scales, all else float32.  Per element of S: one fused multiply-add, one exponential, one add, one
// multiply, half a conversion; 16 exponentials a cycle and SM take as long as the products at the tensor cores' rate.
// Every wait is bounded; on expiry the CTA says so in its flag word, frees its tensor memory and returns.
#pragma once

#include "kv_attention_mma.cuh"
#include "tc_common.cuh"

namespace vscan {
namespace kv {

constexpr int kTcThreads = 416;
constexpr int kTcRows = 256;          // query rows of a CTA
constexpr int kTcKeys = 128;          // keys of a step
constexpr int kTcRing = 4;            // steps whose scales are kept: a converter is at most three steps ahead of a reader
constexpr int kChunk = 128 * 128;     // bytes of [128 rows x 64 f16]

struct TcShared {
  uint64_t q_full[2], s_full[2], p_full[2], o_done[2];
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t scale_full[kTcRing];
  uint32_t tmem_base;
  int abort_flag;
  int missing[kTcRing];
  float ks[kTcRing][8], vs[kTcRing][8];   // of the 16-token groups of a step
  long long weight[kTcThreads / 32];
  long long seq0;
  int b;
};

// ---------------------------------------------------------------------------------------------- division of the work
// As for few rows, but a place on the line is a key seen by a query row, so that the triangle of a causal prompt is divided
// evenly: tile k of a causal sequence weighs group * start + min(256 (k + 1), rows), which has a closed prefix sum.
struct TcSequence {
  Sequence s;
  long long base;       // what every tile weighs at least
  long long rows;       // query rows; causal tiles weigh more one after another
  long long weight;     // of all tiles of a KV head
  int tiles;
};

__device__ __forceinline__ long long tiles_before(const TcSequence& q, bool causal, long long k) {
  if (!causal) return k * q.base;
  const long long grown = k < q.tiles ? k * (k + 1) * (kTcRows / 2) : static_cast<long long>(q.tiles - 1) * q.tiles * (kTcRows / 2) + q.rows;
  return k * q.base + grown;
}

__device__ __forceinline__ TcSequence tc_sequence_at(const AttnParams& p, int b) {
  TcSequence q;
  q.s = sequence_at(p, b);
  q.rows = static_cast<long long>(q.s.n) * p.group;
  q.tiles = static_cast<int>((q.rows + kTcRows - 1) / kTcRows);
  q.base = p.causal ? max(q.s.start, 0ll) * p.group : max(static_cast<long long>(q.s.len) * p.group, 1ll);
  q.weight = q.tiles > 0 ? tiles_before(q, p.causal, q.tiles) : 0;
  return q;
}

struct TcStretch { long long begin, end, quota, seq0; int b; };

__device__ __forceinline__ TcStretch tc_locate(const AttnParams& p, TcShared& sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per = (p.batch + kTcThreads - 1) / kTcThreads, b0 = min(static_cast<int>(threadIdx.x) * per, p.batch), b1 = min(b0 + per, p.batch);
  long long sum = 0;
  for (int b = b0; b < b1; ++b) sum += tc_sequence_at(p, b).weight * p.kv_heads;
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
  for (int w = 0; w < kTcThreads / 32; ++w) {
    if (w < warp) before += sh.weight[w];
    total += sh.weight[w];
  }
  TcStretch st;
  // a stretch is at least four steps long, so that no two cuts fall into one step
  st.quota = max((total + gridDim.x - 1) / gridDim.x, 4ll * kTcKeys * p.group);
  st.begin = min(blockIdx.x * st.quota, total);
  st.end = min(st.begin + st.quota, total);
  long long at = before + incl - sum;
  if (at <= st.begin && st.begin < at + sum) {
    for (int b = b0; b < b1; ++b) {
      const long long w = tc_sequence_at(p, b).weight * p.kv_heads;
      if (st.begin < at + w) { sh.b = b; sh.seq0 = at; break; }
      at += w;
    }
  }
  __syncthreads();
  st.b = sh.b;
  st.seq0 = sh.seq0;
  return st;
}

struct TcPiece {
  TcSequence q;
  long long seg0, seg1;   // seg1: the end of what there is to do, as a place on the line
  int b, head, tile, n_rows, most, u0, u1, units;
};

__device__ __forceinline__ bool tc_next(const AttnParams& p, TcStretch& st, TcPiece& pc) {
  while (st.begin < st.end) {
    pc.q = tc_sequence_at(p, st.b);
    const long long all = pc.q.weight * p.kv_heads;
    if (st.begin >= st.seq0 + all) { st.seq0 += all; ++st.b; continue; }
    const long long head = (st.begin - st.seq0) / pc.q.weight, rel = st.begin - st.seq0 - head * pc.q.weight;
    int lo = 0, hi = pc.q.tiles;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (tiles_before(pc.q, p.causal, mid) <= rel) lo = mid; else hi = mid;
    }
    pc.head = static_cast<int>(head); pc.tile = lo; pc.b = st.b;
    pc.seg0 = st.begin - (rel - tiles_before(pc.q, p.causal, lo));
    const long long seg_end = pc.seg0 + tiles_before(pc.q, p.causal, lo + 1) - tiles_before(pc.q, p.causal, lo);
    pc.n_rows = static_cast<int>(min(static_cast<long long>(kTcRows), pc.q.rows - static_cast<long long>(lo) * kTcRows));
    pc.most = visible(p, pc.q.s, (lo * kTcRows + pc.n_rows - 1) / p.group);
    pc.units = max(1, (pc.most + kTcKeys - 1) / kTcKeys);
    const long long per_unit = static_cast<long long>(kTcKeys) * p.group;
    pc.seg1 = min(seg_end, pc.seg0 + pc.units * per_unit);
    pc.u0 = static_cast<int>(min((st.begin - pc.seg0) / per_unit, static_cast<long long>(pc.units)));
    pc.u1 = st.end >= seg_end ? pc.units : static_cast<int>(min((st.end - pc.seg0) / per_unit, static_cast<long long>(pc.units)));
    st.begin = seg_end;
    if (pc.u0 < pc.u1) return true;
  }
  return false;
}

// ---------------------------------------------------------------------------------------------- instructions
__device__ __forceinline__ void umma_f16_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) { tc::umma_bf16(d, a, b, idesc, accumulate); }
// A operand in tensor memory: row i in lane i, two f16 in a column
__device__ __forceinline__ void umma_f16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(accumulate))
      : "memory");
}
// f16 x f16 -> float32, M = 128; b_mn: the second operand MN-major
__device__ __forceinline__ uint32_t idesc_f16(int n, bool b_mn) {
  return (1u << 4) | (b_mn ? 1u << 16 : 0u) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(128 >> 4) << 24);
}
// MN-major operand, 128-byte swizzle: 64 channels a row, rows (tokens) in groups of 8 of 1024 bytes, kChunk bytes from 64
// channels to the next 64
__device__ __forceinline__ uint64_t desc_mn(uint32_t addr) {
  return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | static_cast<uint64_t>(kChunk >> 4) << 16 | static_cast<uint64_t>(1024 >> 4) << 32 |
         1ull << 46 | 2ull << 61;
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

template <int KV, int DP>
__global__ void __launch_bounds__(kTcThreads, 1) tc_kernel(AttnParams p) {
  using namespace tc;
  constexpr int kDChunks = DP / 64, kTileBytes = kDChunks * kChunk;
  extern __shared__ unsigned char smem_dyn[];
  __shared__ TcShared sh;
  unsigned char* base = smem_dyn + ((1024u - (smem_u32(smem_dyn) & 1023u)) & 1023u);
  unsigned char* q_sh = base;                      // [2 tiles]
  unsigned char* k_sh = q_sh + 2 * kTileBytes;     // [2 stages]
  unsigned char* v_sh = k_sh + 2 * kTileBytes;     // [2 stages]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int D = p.head_dim;
  volatile int* abort_flag = &sh.abort_flag;

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.q_full[i], 4); mbar_init(&sh.s_full[i], 1); mbar_init(&sh.p_full[i], 4); mbar_init(&sh.o_done[i], 1);
      mbar_init(&sh.k_full[i], 4); mbar_init(&sh.k_empty[i], 1); mbar_init(&sh.v_full[i], 4); mbar_init(&sh.v_empty[i], 1);
    }
    for (int i = 0; i < kTcRing; ++i) mbar_init(&sh.scale_full[i], 1);
    sh.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 12) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)), "n"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem_base;              // scores of tile 0, 1 at columns 0, 128; sums at 256, 384
  grid_dependency_wait();
  TcStretch st = tc_locate(p, sh);
  if (threadIdx.x == 0) {
    if (blockIdx.x == 0) { p.status[0] = kStatusFlags | gridDim.x; p.status[1] = 0; }
    p.boundary[blockIdx.x].seg1 = 0;
    p.flags[blockIdx.x] = 0;
  }
  __syncthreads();
  bool bad = false;
  TcPiece pc;

  if (warp < 8) {
    // ============================================================ a query row a thread
    const int tile = warp >> 2, r = (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem + lanes + tile * 128, o_addr = tmem + lanes + 256 + tile * 128;
    unsigned char* q_row = q_sh + tile * kTileBytes + r * 128;
    int n_it = 0;            // steps of this tile so far
    int step = 0;            // steps of the CTA so far
    bool ok = true;
    while (ok && tc_next(p, st, pc)) {
      const int steps = pc.u1 - pc.u0;
      if (pc.u0 > 0 && threadIdx.x == 0)
        p.boundary[blockIdx.x] = {pc.seg0, pc.seg1, st.quota, pc.b, pc.head, pc.tile, 0};
      if (tile * 128 >= pc.n_rows) { step += steps; continue; }
      if (p.kv_len[pc.b] > pc.q.s.len) bad = true;
      const int in_tile = tile * 128 + r;
      const bool on = in_tile < pc.n_rows;
      const int flat = pc.tile * kTcRows + (on ? in_tile : 0), i_row = flat / p.group;
      const RowAt at = {i_row, pc.head * p.group + flat - i_row * p.group};
      const int seen = on ? visible(p, pc.q.s, i_row) : 0;

      // ---- the query row: largest element, power of two, f16 into the swizzled tile
      float cq;
      {
        const char* src = q_at(p, pc.b, pc.q.s.first, at);
        uint4 raw[DP / 8];
#pragma unroll
        for (int c = 0; c < DP / 8; ++c) {
          raw[c] = make_uint4(0, 0, 0, 0);
          if (on && c * 8 < D) raw[c] = ld_nc_16(src + c * 16);
        }
        float top = 0.f;
#pragma unroll
        for (int c = 0; c < DP / 8; ++c) {
          float f[8];
          Vec16<__nv_bfloat16>::unpack(raw[c], f);
#pragma unroll
          for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(f[j]));
        }
        const int e = max(static_cast<int>(__float_as_uint(top) >> 23) - 127, -100);
        const float up = copysignf(exp2_int(min(14 - e, 127)), p.scale_log2e);   // the factor of a score is kept positive
        cq = exp2_int(max(e - 14, -126)) * fabsf(p.scale_log2e);
#pragma unroll
        for (int c = 0; c < DP / 8; ++c) {
          float f[8];
          Vec16<__nv_bfloat16>::unpack(raw[c], f);
          const uint4 w = make_uint4(pack_f16(f[0] * up, f[1] * up), pack_f16(f[2] * up, f[3] * up), pack_f16(f[4] * up, f[5] * up),
                                     pack_f16(f[6] * up, f[7] * up));
          *reinterpret_cast<uint4*>(q_row + (c >> 3) * kChunk + (((c & 7) ^ (r & 7)) << 4)) = w;
        }
        fence_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_full[tile]);
      }

      float m = -INFINITY, l = 0.f, ref = 0.f;
      for (int j = 0; j < steps && ok; ++j, ++n_it, ++step) {
        const int slot = step & (kTcRing - 1);
        ok = mbar_wait_warp(&sh.scale_full[slot], (step / kTcRing) & 1, abort_flag) && mbar_wait_warp(&sh.s_full[tile], n_it & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        const float* ks = sh.ks[slot];
        const float* vs = sh.vs[slot];
        const int vis = seen - (pc.u0 + j) * kTcKeys;             // columns that this row sees
        const bool masked = __any_sync(0xffffffffu, vis < kTcKeys) || sh.missing[slot];
        auto hidden = [&](int g, int c) { return c >= vis || ks[g] < 0.f; };

        // ---- largest score
        float top = -INFINITY;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t v[64];
          tmem_ld32(s_addr + half * 64, v);
          tmem_ld32(s_addr + half * 64 + 32, v + 32);
          tmem_wait_ld();
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            float x = -INFINITY;
            if (!masked) {
#pragma unroll
              for (int k = 0; k < 16; ++k) x = fmaxf(x, __uint_as_float(v[g * 16 + k]));
            } else {
#pragma unroll
              for (int k = 0; k < 16; ++k)
                if (!hidden(half * 4 + g, half * 64 + g * 16 + k)) x = fmaxf(x, __uint_as_float(v[g * 16 + k]));
            }
            if (x > -INFINITY) top = fmaxf(top, x * (cq * ks[half * 4 + g]));
          }
        }
        // ---- a new maximum or a new reference of the V scales rescales the sums; both are rare
        float v_top = 0.f;
#pragma unroll
        for (int g = 0; g < 8; ++g) v_top = fmaxf(v_top, vs[g]);
        float f = 1.f;
        const bool over = top > m + kLazy;
        if (__any_sync(0xffffffffu, over)) {
          const float now = fmaxf(m, top);
          f = now == -INFINITY ? 1.f : ex2(m - now);
          m = now;
          l *= f;
        }
        const bool moved = v_top > ref || (v_top < 0.125f * ref && v_top > 0.f);
        if (moved) { f *= ref / v_top; ref = v_top; }
        if (j > 0 && __any_sync(0xffffffffu, f != 1.f)) {
          ok = mbar_wait_warp(&sh.o_done[tile], (n_it - 1) & 1, abort_flag);
          if (!ok) break;
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < DP; c += 16) {
            uint32_t v[16];
            tmem_ld16(o_addr + c, v);
            tmem_wait_ld();
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * f);
            tmem_st16(o_addr + c, v);
          }
        }
        // ---- weights over the scores: the columns a chunk is written to have been read before
        const float inv_ref = ref > 0.f ? kWeightScale / ref : 0.f, minus_m = m == -INFINITY ? 0.f : -m;
        float l0 = 0.f, l1 = 0.f;
#pragma unroll
        for (int quarter = 0; quarter < 4; ++quarter) {
          uint32_t v[32], w[16];
          tmem_ld32(s_addr + quarter * 32, v);
          tmem_wait_ld();
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const float fk = cq * ks[quarter * 2 + g], fv = vs[quarter * 2 + g] * inv_ref;
#pragma unroll
            for (int k = 0; k < 16; k += 2) {
              float e0 = ex2(fmaf(__uint_as_float(v[g * 16 + k]), fk, minus_m)), e1 = ex2(fmaf(__uint_as_float(v[g * 16 + k + 1]), fk, minus_m));
              float w0 = e0 * fv, w1 = e1 * fv;
              if (masked) {
                const int c = quarter * 32 + g * 16 + k;
                if (hidden(quarter * 2 + g, c)) e0 = w0 = 0.f;
                if (hidden(quarter * 2 + g, c + 1)) e1 = w1 = 0.f;
              }
              l0 += e0;
              l1 += e1;
              w[g * 8 + k / 2] = pack_f16(w0, w1);
            }
          }
          tmem_st16(s_addr + quarter * 16, w);
        }
        l += l0 + l1;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_full[tile]);
      }
      if (!ok) break;
      // ---- results
      ok = mbar_wait_warp(&sh.o_done[tile], (n_it - 1) & 1, abort_flag);
      if (!ok) break;
      tc_fence_after();
      const bool complete = pc.u0 == 0 && pc.u1 == pc.units;
      const float unit = ref * (1.f / kWeightScale), mul = complete ? (l == 0.f ? 0.f : unit / l) : unit;
      float* part = p.partial + (static_cast<size_t>(blockIdx.x) * 2 + (pc.u0 == 0 ? 1 : 0)) * partial_floats(kTcRows, D);
      char* out = out_at(p, pc.b, pc.q.s.first, at);
#pragma unroll 1
      for (int c = 0; c < DP; c += 16) {
        uint32_t v[16];
        tmem_ld16(o_addr + c, v);
        tmem_wait_ld();
        if (on && c < D) {
          float x[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) x[k] = __uint_as_float(v[k]) * mul;
          if (complete) {
            st_16(out + c * 2, Vec16<__nv_bfloat16>::pack(x));
            st_16(out + c * 2 + 16, Vec16<__nv_bfloat16>::pack(x + 8));
          } else {
#pragma unroll
            for (int k = 0; k < 16; k += 4)
              *reinterpret_cast<float4*>(part + static_cast<size_t>(in_tile) * D + c + k) = make_float4(x[k], x[k + 1], x[k + 2], x[k + 3]);
          }
        }
      }
      tc_fence_before();
      if (on) {
        if (!complete) { part[kTcRows * D + in_tile] = m; part[kTcRows * D + kTcRows + in_tile] = l; }
        else if (p.lse) *lse_at(p, pc.b, pc.q.s.first, at) = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
      }
    }
  } else if (warp < 12) {
    // ============================================================ codes to f16
    constexpr int kPer = DP / 16, kRowsPass = 128 / kPer, kLoads = 128 / kRowsPass;   // pieces of a token; tokens and loads of a pass
    const int tid = threadIdx.x - 256, piece = tid % kPer, row0 = tid / kPer;
    const bool in_dim = piece * 16 < D;
    const size_t cell_bytes = static_cast<size_t>(p.block_size) * D;
    int step = 0;
    bool ok = true;
    while (ok && tc_next(p, st, pc)) {
      const int32_t* table = p.block_table + static_cast<size_t>(pc.b) * p.max_blocks;
      // lanes 0-7 know the blocks of the 16-token groups of a step
      auto blocks_at = [&](int t0) {
        int x = -1;
        const int t = t0 + lane * 16;
        if (lane < 8 && t < pc.most) {
          x = table[t >> p.shift];
          if (x < 0 || x >= p.num_blocks) { x = -1; bad = true; }
        }
        return x;
      };
      uint4 raw[kLoads];
      auto load = [&](const uint8_t* cache, int blk, int t0) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int row = row0 + i * kRowsPass, t = t0 + row;
          const int block = __shfl_sync(0xffffffffu, blk, row >> 4);
          raw[i] = make_uint4(0, 0, 0, 0);
          if (in_dim && t < pc.most && block >= 0)
            raw[i] = ld_nc_16(cache + (static_cast<size_t>(block) * p.kv_heads + pc.head) * cell_bytes +
                              static_cast<size_t>(t & (p.block_size - 1)) * D + piece * 16);
        }
      };
      auto store = [&](unsigned char* dst) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int row = row0 + i * kRowsPass;
          const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
          uint32_t h[8];
#pragma unroll
          for (int k = 0; k < 4; ++k) codes_to_f16<KV>(w[k], h[2 * k], h[2 * k + 1]);
          unsigned char* at = dst + (piece >> 2) * kChunk + row * 128;
          const int c16 = (piece & 3) * 2;
          *reinterpret_cast<uint4*>(at + ((c16 ^ (row & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
          *reinterpret_cast<uint4*>(at + (((c16 + 1) ^ (row & 7)) << 4)) = make_uint4(h[4], h[5], h[6], h[7]);
        }
        fence_async();
        __syncwarp();
      };
      int blk = blocks_at(pc.u0 * kTcKeys);
      load(p.k_cache, blk, pc.u0 * kTcKeys);
      for (int u = pc.u0; u < pc.u1 && ok; ++u, ++step) {
        const int s = step & 1, slot = step & (kTcRing - 1), t0 = u * kTcKeys;
        if (step >= 2) ok = mbar_wait_warp(&sh.k_empty[s], ((step >> 1) - 1) & 1, abort_flag);
        if (!ok) break;
        store(k_sh + s * kTileBytes);
        if (lane == 0) mbar_arrive(&sh.k_full[s]);
        load(p.v_cache, blk, t0);
        if (warp == 8) {
          const bool none = lane < 8 && blk < 0 && t0 + lane * 16 < pc.most;
          if (lane < 8) {
            const size_t cell = static_cast<size_t>(max(blk, 0)) * p.kv_heads + pc.head;
            sh.ks[slot][lane] = blk >= 0 ? __ldg(p.k_scale + cell) : none ? -1.f : 0.f;
            sh.vs[slot][lane] = blk >= 0 ? __ldg(p.v_scale + cell) : 0.f;
          }
          const bool any = __any_sync(0xffffffffu, none);
          if (lane == 0) sh.missing[slot] = any;
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.scale_full[slot]);
        }
        const int next = u + 1 < pc.u1 ? blocks_at(t0 + kTcKeys) : -1;
        if (step >= 2) ok = mbar_wait_warp(&sh.v_empty[s], ((step >> 1) - 1) & 1, abort_flag);
        if (!ok) break;
        store(v_sh + s * kTileBytes);
        if (lane == 0) mbar_arrive(&sh.v_full[s]);
        blk = next;
        if (u + 1 < pc.u1) load(p.k_cache, blk, t0 + kTcKeys);
      }
    }
  } else {
    // ============================================================ products
    if (lane == 0) {
      const uint32_t qk = idesc_f16(kTcKeys, false), pv = idesc_f16(DP, true);
      const uint32_t q_addr = smem_u32(q_sh), k_addr = smem_u32(k_sh), v_addr = smem_u32(v_sh);
      int step = 0, n_it[2] = {0, 0}, n_piece[2] = {0, 0};
      bool ok = true;
      auto scores = [&](int t, int s) {        // S of tile t from stage s of K
        // the weights that lie there have been used up, not only issued
        if (n_it[t] > 0 && !mbar_wait(&sh.o_done[t], (n_it[t] - 1) & 1, abort_flag)) return false;
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < kDChunks; ++c) {
          const uint64_t a = smem_desc_sw128(q_addr + t * kTileBytes + c * kChunk), b = smem_desc_sw128(k_addr + s * kTileBytes + c * kChunk);
#pragma unroll
          for (int k = 0; k < 4; ++k) umma_f16_ss(tmem + t * 128, a + 2u * k, b + 2u * k, qk, c > 0 || k > 0);
        }
        umma_commit(&sh.s_full[t]);
        return true;
      };
      while (ok && tc_next(p, st, pc)) {
        const int tiles = pc.n_rows > 128 ? 2 : 1;
        for (int t = 0; t < tiles && ok; ++t) ok = mbar_wait(&sh.q_full[t], n_piece[t]++ & 1, abort_flag);
        ok = ok && mbar_wait(&sh.k_full[step & 1], (step >> 1) & 1, abort_flag);
        for (int t = 0; t < tiles && ok; ++t) ok = scores(t, step & 1);
        if (!ok) break;
        umma_commit(&sh.k_empty[step & 1]);
        for (int u = pc.u0; u < pc.u1 && ok; ++u, ++step) {
          const int s = step & 1;
          const bool more = u + 1 < pc.u1;
          ok = mbar_wait(&sh.v_full[s], (step >> 1) & 1, abort_flag);
          for (int t = 0; t < tiles && ok; ++t) {
            ok = mbar_wait(&sh.p_full[t], n_it[t] & 1, abort_flag);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < kTcKeys / 16; ++k)
              umma_f16_ts(tmem + 256 + t * 128, tmem + t * 128 + k * 8, desc_mn(v_addr + s * kTileBytes + k * 2048), pv, u > pc.u0 || k > 0);
            umma_commit(&sh.o_done[t]);
            if (t == tiles - 1) umma_commit(&sh.v_empty[s]);
            ++n_it[t];
            if (more) {
              if (t == 0) ok = mbar_wait(&sh.k_full[s ^ 1], ((step + 1) >> 1) & 1, abort_flag);
              ok = ok && scores(t, s ^ 1);
            }
          }
          if (ok && more) umma_commit(&sh.k_empty[s ^ 1]);
        }
      }
    }
    __syncwarp();
  }

  // ------------------------------------------------------------ teardown
  tc_fence_before();
  __syncthreads();
  if (bad) p.flags[blockIdx.x] = VSCAN_ERR_INVALID_ARG;
  if (sh.abort_flag) {
    if (threadIdx.x == 0) p.flags[blockIdx.x] = VSCAN_ERR_TIMEOUT;
    for (int i = 0; i < 64; ++i) __nanosleep(2000);   // products still in flight end before their memory is given back
    __syncthreads();
  }
  if (warp == 12) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
  }
}

}  // namespace kv
}  // namespace vscan
