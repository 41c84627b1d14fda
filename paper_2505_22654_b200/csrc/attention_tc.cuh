// Attention over whole prompts for bf16 on the 5th-generation tensor cores.
//
// A CTA takes up to 256 query rows (new rows x heads of a group) of one KV head as two tiles of up to 128 and runs over its stretch of the keys,
// 128 at a time:
//   warps 0-7, 8-15  tile 0, 1: a warp 16 query rows, four threads a row.  Scores from tensor memory into registers, running maximum and sum,
//                    weights back to tensor memory as bf16, over the scores that they come from
//   warps 16-19      the results of both tiles: tensor memory to memory, while the others begin the next piece; and the values of a step
//                    that some row does not see in full (below)
//   warp 20          issues the products: S[128 x 128] = Q K^T (operands in shared memory), O[128 x d] += P V with P read from tensor
//                    memory and V, tokens down and channels across, as the MN-major operand
//   warp 21          queries, K and V by TMA; K and V in a ring of four tiles of 128 rows
//   warp 22          plans: what the next pieces of the stretch are, a few ahead of all others
// A tile of 128 rows has whole tokens of the group's heads (126 rows for groups of seven), so that TMA can bring them.
// Heads of more than 128 channels: one tile a CTA, whose sums take the tensor memory of both (warps 8-15 have nothing to do), and fewer, larger
// tiles of K and V in the ring.  4 prompts of 1,700 to 2,176 rows, 28 / 4 heads of 256, 0.20 TFLOP: 312 us; 2 x
// 9,000 to 12,200 rows: 0.91 PFLOP/s.
// The two tiles take turns: while one's weights are made, the other's products run.  A step takes the tensor cores 2,048 cycles at 128 channels
// (32 products of 64) and the exponentials, 32,768 at 16 a cycle, as many; it takes some 3,900: a tile's next scores wait for the products of
// its weights, since tensor memory is full (two tiles of scores and two of sums, 128 columns each) and the weights lie over their scores.
// The code of all roles together is more than the instruction cache holds, so what is written shorter here runs faster.
// Measured: 2 x 9,000 to 12,200 rows, 28 / 4 heads of 128, 1.78 TFLOP: 1.56 to 1.84 ms from one GPU to the next; 160 x 577 rows, 16 heads of 64, 0.22
// TFLOP: 514 to 535 us; 4 x 1,700 to 2,176 rows, 28 / 4 heads of 128: 164 to 172 us.
// Tried and slower: weights through shared memory with the next scores made ahead (2.2 ms; products whose operands all lie in shared memory
// take all of its bandwidth), the next scores ahead at 64 channels, where tensor memory has the room (760 us: more instruction cache
// misses), exponentials on the FMA pipe (by a polynomial of degree 4: 1 to 25 % slower the more of them), one thread a row (1.78 ms, 600 us).
//
// The reference that is taken off a row's scores is raised only when a score is over it by 2^kLazy, so the sums are seldom rescaled; weights
// are then up to 2^kLazy, which bf16 does not mind.  Weights are rounded to bf16: both operands of a product have one type, and V in float16
// would lose its range.  The error, up to 2^-8 of each weight and of either sign, is averaged over the keys and stays below the rounding of the
// result; their sum is taken before the rounding.  scale log2(e) is one float32 here (two in the CUDA-core kernel), so a weight and lse are off by
// 2^-24 of the score's size more.
//
// Masked weights are 0, but 0 times an infinity is not: in a step that some row does not see in full, values that are not finite are
// made 0 in shared memory before the product, and what they give to the rows that do see them is put together beside it.
// Every wait is bounded; on expiry the CTA says so in its flag word, frees its tensor memory and returns.
#pragma once

#include "attention_prompt.cuh"
#include "kv_attention_tc.cuh"
#include "tc_rows.cuh"

namespace vscan {
namespace kv {

// kPtWhole, kPtExtra: steps up to which a tile is not cut, and what its start and end weigh beside its own steps.  This kernel, us, for 4 prompts of
// 1,700 to 2,176 rows / encoder layers of 577 / 2 x 9,000 to 12,200 rows: 8 and 4: 154 / 532 / 1,559; 4 and 4: 151 / 543 and a join of 15 / 1,559;
// 16 and 4: 163 / 532 / 1,560; 8 and 0: 209 / 530 / 1,825; 8 and 2: 166 / 532 / 1,609; 8 and 8: 167 / 532 / 1,610.
constexpr int kPtThreads = 768, kPtKeys = 128, kPtWhole = 8, kPtExtra = 4;
constexpr int kPtHelper = 16, kPtIssuer = 20, kPtLoader = 21, kPtPlanner = 22;   // first warp of each role
constexpr int kPtStages = 4, kPtPlan = 4;
// Tiles of a CTA, and of K and V in the ring: what 512 columns of tensor memory and 192 KB hold
__host__ __device__ constexpr int pt_tiles(int dp) { return dp > 128 ? 1 : 2; }
__host__ __device__ constexpr int pt_stages(int dp) { return dp > 192 ? 2 : dp > 128 ? 3 : kPtStages; }
constexpr int kPtReaders = 22;       // warps that read the plan
// 768 threads start with 80 registers each: 512 x 88 + 256 x 64 = 768 x 80.
using PtShape = TileShape<kPtThreads, 0, kPtKeys, kPtWhole, kPtExtra>;

struct PtPiece {         // steps u0 .. u1 - 1 of a tile; u1 = 0: there is no more
  int b, head, tile, n_rows, first, key0, len, u0, u1, units;
  int partial;           // steps from this one on are not seen in full by some row
  int token;             // of the sequence's rows, the tile's first
  long long start;       // position of the sequence's first row
};

struct PtShared {
  uint64_t q_full[2], q_empty[2], s_full[2], p_half[2], p_full[2], o_done[2], o_free[2], stat_full[2];   // of the tiles
  uint64_t kv_full[kPtStages], kv_empty[kPtStages];
  uint64_t dirty[2], clean[2];                // of steps that are seen in part, in turn: their values are under way, and cleaned
  uint32_t tmem_base;
  int abort_flag;
  float2 stat[2][128];                        // [tile][row]: reference and sum
  uint32_t odd[2 * 128 * 8];                  // [tile][row]: channels that get +inf (a bit each) and -inf
  uint32_t found[2][4];                       // of a step that is seen in part: keys whose values are not all finite, a word of each warp
  uint64_t plan_full[kPtPlan], plan_empty[kPtPlan];
  PtPiece plan[kPtPlan];
  DivisionShared division;
};

// ---------------------------------------------------------------------------------------------- instructions
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// 16 lanes (rows) x 64 columns of tensor memory, with the wait: v[4 i + k] is row lane / 4 + 8 (k / 2), column 8 i + 2 (lane % 4) + k % 2
__device__ __forceinline__ void tmem_read_rows(uint32_t taddr, uint32_t* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x8.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
        "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
        "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
        "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(taddr)
      : "memory");
}
// The same rows x 16 columns, read and written
__device__ __forceinline__ void tmem_read_rows16(uint32_t taddr, uint32_t* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_write_rows16(uint32_t taddr, const uint32_t* v) {
  asm volatile("tcgen05.st.sync.aligned.16x256b.x2.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
// The same rows x 32 columns written: v[2 i + k] is row lane / 4 + 8 k, column 4 i + lane % 4
__device__ __forceinline__ void tmem_write_pairs(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
// The largest of three; NaN if one is
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// Bounded wait of a warp, in few instructions: this kernel's code has to stay in the instruction cache
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  bool got = tc::mbar_try_wait(bar, parity);
#pragma unroll 1
  for (uint32_t i = 0; i < tc::kSpinLimit && !got; ++i) {
    if ((i & 1023u) == 1023u && *abort_flag) break;
    got = tc::mbar_try_wait(bar, parity);
  }
  if (!got) *abort_flag = 1;
  return __all_sync(0xffffffffu, got);
}
// A wait that may last for all of a piece: the limit of the other waits, 4 s or some two million steps, is granted once more for every
// 2^17 keys that there may be.  If another role gives up, so does this wait.
__device__ __forceinline__ bool wait_piece(const PromptParams& p, uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  bool got = tc::mbar_try_wait(bar, parity);
#pragma unroll 1
  for (unsigned long long i = 0, n = static_cast<unsigned long long>((p.kv_rows >> 17) + 1) * tc::kSpinLimit; i < n && !got; ++i) {
    if ((i & 1023u) == 1023u && *abort_flag) break;
    got = tc::mbar_try_wait(bar, parity);
  }
  if (!got) *abort_flag = 1;
  return __all_sync(0xffffffffu, got);
}
// Keys that row `token` of a sequence sees
__host__ __device__ __forceinline__ int keys_seen(const PromptParams& p, const PtPiece& pc, int token) {
  if (!p.causal) return pc.len;
  return static_cast<int>(min(max(pc.start + token + 1, 0ll), static_cast<long long>(pc.len)));
}

// The pieces of a CTA's stretch one after another, by a warp whose lanes all do the same
struct PtPlanner {
  TcStretch st;
  TcSequence q;
  long long seg0;        // of the tile that the stretch is in
  int key0, head, tile;
  bool inside;

  __host__ __device__ __forceinline__ void enter(const PromptParams& p, int b) {
    st.b = b;
    q = tc_sequence_at<PtShape>(p, b);
    int keys;
    key_span(p, b, key0, keys);
  }
  __host__ __device__ __forceinline__ bool next(const PromptParams& p, PtPiece& pc, Boundary& cut) {
    const long long one = step_weight<PtShape>(p);
    while (st.begin < st.end) {
      if (!inside) {                                     // the stretch's first tile takes a search
        enter(p, st.b);
        head = static_cast<int>(quotient(st.begin - st.seq0, q.weight));
        const long long rel = st.begin - st.seq0 - head * q.weight;
        int lo = 0, hi = q.tiles;
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (tiles_before<PtShape>(p, q, mid) <= rel) lo = mid; else hi = mid;
        }
        tile = lo;
        seg0 = st.begin - (rel - tiles_before<PtShape>(p, q, lo));
        inside = true;
      } else if (tile == q.tiles) {
        tile = 0;
        if (++head == p.kv_heads) {
          head = 0;
          do enter(p, st.b + 1); while (q.tiles == 0);   // there is one: the stretch goes on
        }
      }
      const long long seg_end = seg0 + tile_weight<PtShape>(p, q, tile);
      pc.b = st.b; pc.head = head; pc.tile = tile; pc.first = q.s.first; pc.key0 = key0; pc.len = q.s.len; pc.start = q.s.start;
      const int tokens = p.tile_rows / p.group;
      pc.token = tile * tokens;
      const int n = min(q.s.n - pc.token, tokens);
      pc.n_rows = n * p.group;
      pc.units = max(1, (keys_seen(p, pc, pc.token + n - 1) + kPtKeys - 1) / kPtKeys);
      const bool starts = st.begin == seg0, ends = st.end >= seg_end, whole = pc.units <= kPtWhole;
      pc.u0 = whole || starts ? 0 : step_at<PtShape>(st.begin - seg0, one, pc.units);
      pc.u1 = whole || ends ? pc.units : step_at<PtShape>(st.end - seg0, one, pc.units);
      pc.partial = max(pc.u0, keys_seen(p, pc, pc.token) / kPtKeys);
      cut = {seg0, min(seg_end, seg0 + (pc.units + kPtExtra) * one), st.quota, st.b, head, tile, q.s.first, pc.n_rows, 0};
      ++tile;
      st.begin = seg0 = seg_end;
      if (whole ? starts : pc.u0 < pc.u1) return true;
    }
    return false;
  }
};

template <int DP>
__global__ void __launch_bounds__(kPtThreads, 1) prompt_tc_kernel(PromptParams p, const __grid_constant__ CUtensorMap q_map,
                                                                  const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  using namespace tc;
  constexpr int kDChunks = DP / 64, kTileBytes = kDChunks * kChunk, kTiles = pt_tiles(DP), kStages = pt_stages(DP), kOddWords = kTiles == 1 ? 8 : 4;
  extern __shared__ unsigned char smem_dyn[];
  __shared__ PtShared sh;
  unsigned char* base = smem_dyn + ((1024u - (smem_u32(smem_dyn) & 1023u)) & 1023u);
  unsigned char* q_sh = base;                      // [tiles]
  unsigned char* kv_sh = q_sh + kTiles * kTileBytes;    // [stages]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int D = p.head_dim;
  volatile int* abort_flag = &sh.abort_flag;

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.q_full[i], 1); mbar_init(&sh.q_empty[i], 1); mbar_init(&sh.s_full[i], 1);
      mbar_init(&sh.p_half[i], 8); mbar_init(&sh.p_full[i], 8);
      mbar_init(&sh.o_done[i], 1); mbar_init(&sh.o_free[i], 4); mbar_init(&sh.stat_full[i], 8);
      mbar_init(&sh.dirty[i], 1); mbar_init(&sh.clean[i], 4);
    }
    for (int i = 0; i < kStages; ++i) { mbar_init(&sh.kv_full[i], 1); mbar_init(&sh.kv_empty[i], 1); }
    for (int i = 0; i < kPtPlan; ++i) { mbar_init(&sh.plan_full[i], 1); mbar_init(&sh.plan_empty[i], kPtReaders); }
    sh.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kPtIssuer) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)), "n"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem_base;              // scores of tile t at column 128 t; sums at 256 + 128 t
  grid_dependency_wait();
  const TcStretch st = tc_locate<PtShape>(p, sh.division);
  if (threadIdx.x == 0) {
    if (blockIdx.x == 0) { p.status[0] = kStatusFlags | gridDim.x; p.status[1] = 0; }
    p.boundary[blockIdx.x].seg1 = 0;
    p.flags[blockIdx.x] = 0;
  }
  __syncthreads();
  PtPiece pc;
  int n_plan = 0;                                  // pieces read so far
  // The next piece of the plan; false where there is none, or another role gave up
  auto next = [&]() {
    const int slot = n_plan % kPtPlan;
    if (!wait_piece(p, &sh.plan_full[slot], (n_plan / kPtPlan) & 1, abort_flag)) return false;
    pc = sh.plan[slot];
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.plan_empty[slot]);
    ++n_plan;
    return pc.u1 > 0;
  };
  const int tokens = p.tile_rows / (kTiles * p.group), half = tokens * p.group;      // tokens and rows of a tile of 128

  if (warp < kPtHelper) {
    // ============================================================ four threads a query row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 88;");
    const int tile = warp >> 3, row0 = (warp & 3) * 32 + ((warp >> 2) & 1) * 16;
    const uint32_t lanes = static_cast<uint32_t>(row0) << 16;
    const uint32_t s_addr = tmem + lanes + tile * 128;            // these rows' scores, and their weights
    const uint32_t o_addr = tmem + lanes + 256 + tile * 128;
    const float factor = fmaxf(p.scale_log2e, 0x1p-126f);         // held above 0: a masked score stays -inf
    int n_it = 0, n_piece = 0;                                    // steps and pieces of this tile so far
    bool ok = true;
    while (ok && next()) {
      if (tile * half >= pc.n_rows) continue;
      int seen[2];                       // of rows row0 + lane / 4 and 8 on, less this lane's first column
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = row0 + (lane >> 2) + 8 * i;
        seen[i] = (r < half && tile * half + r < pc.n_rows ? keys_seen(p, pc, pc.token + tile * tokens + r / p.group) : 0) - 2 * (lane & 3);
      }
      float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};      // reference, and this thread's sum of the weights, in units of 2^m
      float minus_m[2] = {0.f, 0.f};     // what is added to a score; NaN where the reference is infinite
      const bool sees_all = pc.partial >= pc.u1;
      for (int u = pc.u0; u < pc.u1; ++u, ++n_it) {
        ok = u == pc.u0 ? wait_piece(p, &sh.s_full[tile], n_it & 1, abort_flag) : wait_warp(&sh.s_full[tile], n_it & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        uint32_t v[64];                  // v[4 i + k]: row k / 2, column 8 i + k % 2 from the lane's first
        tmem_read_rows(s_addr, v);
        tmem_read_rows(s_addr + 64, v + 32);
        if (!sees_all && u >= pc.partial) {
          const int vis[2] = {seen[0] - u * kPtKeys, seen[1] - u * kPtKeys};
#pragma unroll
          for (int k = 0; k < 64; ++k)
            if ((k >> 2) * 8 + (k & 1) >= vis[(k >> 1) & 1]) v[k] = 0xff800000u;      // -inf
        }
        float top[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          top[i][0] = __uint_as_float(v[2 * i]);
          top[i][1] = __uint_as_float(v[2 * i + 1]);
#pragma unroll
          for (int k = 4; k < 60; k += 8) {
            top[i][0] = max3_nan(top[i][0], __uint_as_float(v[2 * i + k]), __uint_as_float(v[2 * i + k + 4]));
            top[i][1] = max3_nan(top[i][1], __uint_as_float(v[2 * i + k + 1]), __uint_as_float(v[2 * i + k + 5]));
          }
          top[i][0] = max_nan(max3_nan(top[i][0], __uint_as_float(v[2 * i + 60]), __uint_as_float(v[2 * i + 61])), top[i][1]);
          top[i][0] = max_nan(top[i][0], __shfl_xor_sync(0xffffffffu, top[i][0], 1));
          top[i][0] = max_nan(top[i][0], __shfl_xor_sync(0xffffffffu, top[i][0], 2)) * factor;      // NaN where a score is
        }
        if (__any_sync(0xffffffffu, !(top[0][0] <= m[0] + kLazy) || !(top[1][0] <= m[1] + kLazy))) {
          float f[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float now = max_nan(m[i], top[i][0]);
            f[i] = now == m[i] ? 1.f : ex2(m[i] - now);
            m[i] = now;
            minus_m[i] = now == -INFINITY ? 0.f : now == INFINITY ? __uint_as_float(0x7fc00000u) : -now;
            l[i] *= f[i];
          }
          if (u > pc.u0 && __any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f)) {
            // (the products with V of the step before are done: this step's scores were issued after them)
#pragma unroll 1
            for (int c = 0; c < DP; c += 16) {
              uint32_t x[8];
              tmem_read_rows16(o_addr + c, x);
#pragma unroll
              for (int k = 0; k < 8; ++k) x[k] = __float_as_uint(__uint_as_float(x[k]) * f[(k >> 1) & 1]);
              tmem_write_rows16(o_addr + c, x);
            }
          }
        }
        const uint64_t mul = pair(factor, factor), add[2] = {pair(minus_m[0], minus_m[0]), pair(minus_m[1], minus_m[1])};
        uint64_t sums[2] = {0, 0};
        auto weigh = [&](int h) {        // 64 columns of both rows
          uint32_t w[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            const int at = h * 32 + 2 * k;
            const float2 x = unpair(fma2(pair(__uint_as_float(v[at]), __uint_as_float(v[at + 1])), mul, add[k & 1]));
            const float2 e = make_float2(ex2(x.x), ex2(x.y));
            sums[k & 1] = add2(sums[k & 1], pair(e.x, e.y));
            w[k] = pack_bf16(e.x, e.y);
          }
          tmem_write_pairs(s_addr + h * 32, w);
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
        };
        weigh(0);
        if (lane == 0) mbar_arrive(&sh.p_half[tile]);      // the products with the first half of the values begin
        weigh(1);
        if (lane == 0) mbar_arrive(&sh.p_full[tile]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float2 both = unpair(sums[i]);
          l[i] += both.x + both.y;
        }
      }
      if (!ok) break;
      // ---- reference and sum to the warps that write the results, which are done with those of the piece before
      if (n_piece > 0) ok = wait_piece(p, &sh.o_free[tile], (n_piece - 1) & 1, abort_flag);
      if (!ok) break;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
        l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
        if ((lane & 3) == 0) sh.stat[tile][row0 + (lane >> 2) + 8 * i] = make_float2(m[i], l[i]);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.stat_full[tile]);
      ++n_piece;
    }
  } else if (warp < kPtIssuer) {
    // ============================================================ results; values of steps that are seen in part
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    const int quarter = warp & 3, r = quarter * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
    const int r_token = r / p.group, r_head = r - r_token * p.group;
    int pos = 0;                 // tiles of K and V that the pieces before have taken
    int n_partial = 0, n_piece[2] = {0, 0};
    bool ok = true;
    while (ok && next()) {
      const int two = pc.n_rows > half;
      bool odd = false;          // some value is not finite; the same in all of these warps
      int seen[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) seen[t] = r < half && t * half + r < pc.n_rows ? keys_seen(p, pc, pc.token + t * tokens + r_token) : 0;
      for (int u = pc.partial; u < pc.u1 && ok; ++u, ++n_partial) {
        const int at = pos + 1 + 2 * (u - pc.u0), s = at % kStages;
        ok = wait_piece(p, &sh.dirty[n_partial & 1], (n_partial >> 1) & 1, abort_flag) &&
             wait_warp(&sh.kv_full[s], (at / kStages) & 1, abort_flag);
        if (!ok) break;
        // a row of 64 channels is 128 bytes; 16-byte pieces of a row may be in any order
        unsigned char* tile = kv_sh + s * kTileBytes;
        unsigned found = 0;                        // rows of this thread's pieces, 16 a chunk
#pragma unroll 1
        for (int c = 0; c < kDChunks; ++c)
#pragma unroll 4
          for (int i = 0; i < 8; ++i) {
            uint4* x = reinterpret_cast<uint4*>(tile + c * kChunk) + i * 128 + r;
            uint4 w = *x;
            auto bad = [](uint32_t y) { return ((y & 0x7f807f80u) + 0x00800080u) & 0x80008000u; };     // exponent all ones
            const uint32_t b0 = bad(w.x), b1 = bad(w.y), b2 = bad(w.z), b3 = bad(w.w);
            if (b0 | b1 | b2 | b3) {
              auto clear = [](uint32_t y, uint32_t b) { return y & ~((b & 0x8000u ? 0xffffu : 0u) | (b & 0x80000000u ? 0xffff0000u : 0u)); };
              *x = make_uint4(clear(w.x, b0), clear(w.y, b1), clear(w.z, b2), clear(w.w, b3));
              found |= 1u << i;
            }
          }
        // key 16 i + 4 quarter + g is bit 4 i + g of the warp's word: eight lanes have a key's pieces
        uint32_t mine = 0;
        if (__any_sync(0xffffffffu, found != 0)) {
#pragma unroll 1
          for (int i = 0; i < 8; ++i) {
            const uint32_t hits = __ballot_sync(0xffffffffu, (found >> i) & 1u);
            for (int g = 0; g < 4; ++g)
              if ((hits >> (8 * g)) & 0xffu) mine |= 1u << (4 * i + g);
          }
        }
        uint32_t (&words)[4] = sh.found[n_partial & 1];
        fence_async();
        if (lane == 0) words[quarter] = mine;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.clean[n_partial & 1]);
        ok = wait_warp(&sh.clean[n_partial & 1], (n_partial >> 1) & 1, abort_flag);    // the words of all four
        if (ok && (words[0] | words[1] | words[2] | words[3])) {   // rare: what those values give to the rows that see them, from memory
          if (!odd)
            for (int t = 0; t < kTiles; ++t)
              for (int i = 0; i < 2 * kOddWords; ++i) sh.odd[(t * 128 + r) * 2 * kOddWords + i] = 0;
          odd = true;
          const char* v = p.v + (p.padded ? pc.b * p.v_seq : pc.key0 * p.v_row) + pc.head * p.v_head;
          const int t1 = min(max(seen[0], seen[1]), (u + 1) * kPtKeys);
          for (int t = u * kPtKeys; t < t1; ++t) {
            if (!((words[(t >> 2) & 3] >> (((t >> 4) & 7) * 4 + (t & 3))) & 1u)) continue;
            for (int c = 0; c < D; ++c) {
              const float x = __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(v + t * p.v_row)[c]);
              if (x - x == 0.f) continue;
              for (int i = 0; i < kTiles; ++i) {
                if (t >= seen[i]) continue;
                uint32_t* odds = sh.odd + (i * 128 + r) * 2 * kOddWords + (c >> 5);
                if (!(x < 0.f)) odds[0] |= 1u << (c & 31);
                if (!(x > 0.f)) odds[kOddWords] |= 1u << (c & 31);
              }
            }
          }
        }
      }
      pos += 2 * (pc.u1 - pc.u0);
      const bool complete = pc.u0 == 0 && pc.u1 == pc.units;
      for (int t = 0; t <= two && ok; ++t) {
        ok = wait_piece(p, &sh.stat_full[t], n_piece[t] & 1, abort_flag) && wait_piece(p, &sh.o_done[t], n_piece[t] & 1, abort_flag);
        if (!ok) break;
        ++n_piece[t];
        tc_fence_after();
        const int in_tile = t * half + r;
        const bool on = r < half && in_tile < pc.n_rows;
        const float2 stat = sh.stat[t][r];
        const RowAt at = {pc.token + t * tokens + r_token, pc.head * p.group + r_head};
        const float mul = complete ? (stat.y == 0.f ? 0.f : 1.f / stat.y) : 1.f;
        float* part = p.partial + (static_cast<size_t>(blockIdx.x) * 2 + (pc.u0 == 0 ? 1 : 0)) * partial_floats(p.tile_rows, D);
        char* out = out_at(p, pc.b, pc.first, at);
#pragma unroll 1
        for (int c = 0; c < DP; c += 16) {
          uint32_t v[16];
          tmem_read16(tmem + lanes + 256 + t * 128 + c, v);
          if (on && c < D) {
          float x[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) x[k] = __uint_as_float(v[k]);
          if (odd) {
            const uint32_t* odds = sh.odd + (t * 128 + r) * 2 * kOddWords + (c >> 5);
            const uint32_t up = odds[0] >> (c & 31), down = odds[kOddWords] >> (c & 31);
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              if ((up >> k) & 1u) x[k] += INFINITY;
              if ((down >> k) & 1u) x[k] -= INFINITY;
            }
          }
#pragma unroll
          for (int k = 0; k < 16; k += 8) {
            if (c + k >= D) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[k + i] *= mul;
            if (complete) {
              st_16(out + (c + k) * 2, Vec16<__nv_bfloat16>::pack(x + k));
            } else {
              *reinterpret_cast<float4*>(part + static_cast<size_t>(in_tile) * D + c + k) = make_float4(x[k], x[k + 1], x[k + 2], x[k + 3]);
              *reinterpret_cast<float4*>(part + static_cast<size_t>(in_tile) * D + c + k + 4) = make_float4(x[k + 4], x[k + 5], x[k + 6], x[k + 7]);
            }
          }
          }
          __syncwarp();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.o_free[t]);
        if (on) {
          if (!complete) { part[p.tile_rows * D + in_tile] = stat.x; part[p.tile_rows * D + p.tile_rows + in_tile] = stat.y; }
          else if (p.lse) *lse_at(p, pc.b, pc.first, at) = log_sum(stat.x, stat.y);
        }
      }
    }
  } else if (warp == kPtIssuer) {
    // ============================================================ products
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    const uint32_t qk = idesc_bf16(kPtKeys, false), pv = idesc_bf16(DP, true);
    const uint32_t q_addr = smem_u32(q_sh), kv_addr = smem_u32(kv_sh);
    int pos = 0, n_partial = 0, n_it[2] = {0, 0}, n_piece[2] = {0, 0};
    bool ok = true;
    auto scores = [&](int t, int s) {        // S of tile t from stage s
      const uint64_t a = smem_desc_sw128(q_addr + t * kTileBytes), b = smem_desc_sw128(kv_addr + s * kTileBytes);
#pragma unroll
      for (int c = 0; c < kDChunks; ++c) umma_f16_ss_x4(tmem + t * 128, a + c * (kChunk >> 4), b + c * (kChunk >> 4), qk, c > 0);
    };
    auto wait_kv = [&](int at) { return wait_warp(&sh.kv_full[at % kStages], (at / kStages) & 1, abort_flag); };
    while (ok && next()) {
      const int two = pc.n_rows > half;
      for (int t = 0; t <= two && ok; ++t) ok = wait_warp(&sh.q_full[t], n_piece[t] & 1, abort_flag);
      ok = ok && wait_kv(pos);
      if (!ok) break;
      tc_fence_after();
      for (int t = 0; t <= two; ++t) {
        scores(t, pos % kStages);
        umma_commit_warp(&sh.s_full[t]);
        if (pc.u0 + 1 == pc.u1) umma_commit_warp(&sh.q_empty[t]);
      }
      umma_commit_warp(&sh.kv_empty[pos % kStages]);
      ++pos;
      for (int u = pc.u0; u < pc.u1 && ok; ++u) {
        const int vs = pos % kStages, ks = (pos + 1) % kStages;
        const bool more = u + 1 < pc.u1;
        ok = wait_kv(pos);
        if (u >= pc.partial) {
          ok = ok && wait_warp(&sh.clean[n_partial & 1], (n_partial >> 1) & 1, abort_flag);
          ++n_partial;
        }
#pragma unroll 1
        for (int t = 0; t <= two && ok; ++t) {
          if (u == pc.u0 && n_piece[t] > 0) ok = wait_piece(p, &sh.o_free[t], (n_piece[t] - 1) & 1, abort_flag);
          ok = ok && wait_warp(&sh.p_half[t], n_it[t] & 1, abort_flag);
          if (!ok) break;
          tc_fence_after();
          const uint64_t b = desc_mn(kv_addr + vs * kTileBytes);
          umma_f16_ts_x4(tmem + 256 + t * 128, tmem + t * 128, b, pv, u > pc.u0);
          ok = wait_warp(&sh.p_full[t], n_it[t] & 1, abort_flag);
          if (!ok) break;
          tc_fence_after();
          umma_f16_ts_x4(tmem + 256 + t * 128, tmem + t * 128 + 32, b + (64 * 128 >> 4), pv, true);
          if constexpr (kTiles == 1) umma_commit_warp(&sh.kv_empty[vs]);      // the next values do not wait for the scores
          if (more) {            // over the weights that the products before this one read: products run in the order of their issue
            if (t == 0) ok = wait_kv(pos + 1);
            if (!ok) break;
            tc_fence_after();
            scores(t, ks);
            umma_commit_warp(&sh.s_full[t]);
            if (u + 2 == pc.u1) umma_commit_warp(&sh.q_empty[t]);
          } else {
            umma_commit_warp(&sh.o_done[t]);
          }
          ++n_it[t];
        }
        if (!ok) break;
        if constexpr (kTiles > 1) umma_commit_warp(&sh.kv_empty[vs]);
        if (more) umma_commit_warp(&sh.kv_empty[ks]);
        pos += more ? 2 : 1;
      }
      for (int t = 0; t <= two; ++t) ++n_piece[t];
    }
    __syncwarp();
  } else if (warp == kPtLoader) {
    // ============================================================ queries, keys and values
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    int pos = 0, n_partial = 0, n_piece[2] = {0, 0};
    bool ok = true;
    while (ok && next()) {
      const int seq = p.padded ? pc.b : 0, two = pc.n_rows > half;
      for (int i = 2 * pc.u0; i < 2 * pc.u1 && ok; ++i, ++pos) {
        const int s = pos % kStages, u = i >> 1;
        if (pos >= kStages) ok = wait_warp(&sh.kv_empty[s], (pos / kStages - 1) & 1, abort_flag);
        if (!ok) break;
        if (lane == 0) {
          mbar_arrive_expect_tx(&sh.kv_full[s], kTileBytes);
#pragma unroll
          for (int c = 0; c < kDChunks; ++c)
            tma_load_4d(kv_sh + s * kTileBytes + c * kChunk, (i & 1) ? &v_map : &k_map, &sh.kv_full[s], c * 64, pc.key0 + u * kPtKeys, pc.head, seq);
          if ((i & 1) && u >= pc.partial) mbar_arrive(&sh.dirty[n_partial & 1]);
        }
        if ((i & 1) && u >= pc.partial) ++n_partial;
        if (i == 2 * pc.u0) {                                // the first keys do not wait for the queries of the piece before
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (t > two || !ok) continue;
            if (n_piece[t] > 0) ok = wait_piece(p, &sh.q_empty[t], (n_piece[t] - 1) & 1, abort_flag);
            if (!ok) continue;
            ++n_piece[t];
            if (lane == 0) {
              mbar_arrive_expect_tx(&sh.q_full[t], kDChunks * half * 128);
#pragma unroll
              for (int c = 0; c < kDChunks; ++c)
                tma_load_4d(q_sh + t * kTileBytes + c * kChunk, &q_map, &sh.q_full[t], c * 64, pc.head * p.group, pc.first + pc.token + t * tokens, seq);
            }
          }
        }
      }
    }
    __syncwarp();
  } else if (warp == kPtPlanner) {
    // ============================================================ what there is to do
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    PtPlanner plan = {st};
    bool ok = true, more = true;
    while (ok && more) {
      const int slot = n_plan % kPtPlan;
      Boundary cut;
      more = plan.next(p, pc, cut);
      if (!more) pc.u1 = 0;
      if (n_plan >= kPtPlan) ok = wait_piece(p, &sh.plan_empty[slot], (n_plan / kPtPlan - 1) & 1, abort_flag);
      if (!ok) break;
      if (lane == 0) {
        if (more && pc.u0 > 0) p.boundary[blockIdx.x] = cut;
        sh.plan[slot] = pc;
        mbar_arrive(&sh.plan_full[slot]);
      }
      __syncwarp();
      ++n_plan;
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
  }

  // ------------------------------------------------------------ teardown
  tc_fence_before();
  __syncthreads();
  if (sh.abort_flag) {
    if (threadIdx.x == 0) p.flags[blockIdx.x] = VSCAN_ERR_TIMEOUT;
    for (int i = 0; i < 64; ++i) __nanosleep(2000);   // products and copies still in flight end before their memory is given back
    __syncthreads();
  }
  if (warp == kPtIssuer) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
  }
}

}  // namespace kv
}  // namespace vscan
