// Attention of many query rows (prompts, chunks) for bf16 queries on the 5th-generation tensor cores.
//
// A CTA takes 256 query rows (new rows x heads of a group) of one KV head as two tiles of 128 and runs over its stretch of
// the keys, 128 at a time:
//   warps 0-7, 8-15  tile 0, 1: two threads a query row, 64 of the step's scores each.  Scores from tensor memory, running
//                    maximum and sum, weights back to tensor memory, over the scores that they come from; the results at the end
//   warps 16-23      K and V from codes to f16 in shared memory (128-byte swizzle), two stages each; a key that was turned
//                    once serves both tiles
//   warp 24          issues the products: S[128 x 128] = Q K^T (operands in shared memory), O[128 x d] += P V with P read
//                    from tensor memory and V, tokens down and channels across, as the MN-major operand
// The two tiles take turns: while one's weights are made, the other's products run.  Tensor memory is full: two tiles of
// scores and two of sums, 128 columns each.  (Scores of 64 keys in two buffers a tile would hide the products behind the
// weights, but a product 64 columns wide takes as long as one of 128: 70 and 65 cycles measured.)
//
// Roundings: queries exact in f16 but for a power of two; weights in f16, all else float32.  The V scale of a token's block is part of
// its weight's exponent, and a row's reference is the largest sum of score and scale that the row has seen, so what a row loses
// below the smallest step of f16 is small beside its own result, whatever the scales of blocks are that it does not see.  Behind
// a step of larger scales the reference comes down by what the scales do.  The denominator takes the scale off again.
// Per element of S: one fused multiply-add, one exponential, one add, one multiply, half a conversion; 16 exponentials a cycle and SM
// take as long as the products at the tensor cores' rate.
// Measured: 2 x 900 to 1,024 new rows x 28 heads behind 15,000 to 16,384 tokens, 448 GFLOP: 672 us, 667 TFLOP/s (tensor pipe 35 %,
// issue slots 54 %, ALU 41 % busy), and 20 us for the join.  At 72 registers a thread, what 800 threads can have, the compiler keeps
// about 40 words of a thread in local memory.
// Every wait is bounded; on expiry the CTA says so in its flag word, frees its tensor memory and returns.
#pragma once

#include "attention_division.cuh"
#include "kv_attention_mma.cuh"
#include "tc_common.cuh"

namespace vscan {
namespace kv {

constexpr int kTcThreads = 800;
constexpr int kTcConverter = 16, kTcIssuer = 24;   // first warp of each role
// 800 threads start with 72 registers each; the converters give 16 back, the 512 threads of the rows take 8 more:
// 512 x 80 + 256 x 56 + 32 x 72 = 800 x 72.
constexpr int kTcRows = 256;          // query rows of a CTA
constexpr int kTcKeys = 128;          // keys of a step
constexpr int kTcWhole = 4;           // a tile of up to this many steps is not cut: joining 256 rows takes longer than they do
using TcShape = TileShape<kTcThreads, kTcRows, kTcKeys, kTcWhole>;
constexpr int kTcRing = 4;            // steps whose scales are kept: the converters are at most three ahead of a reader
constexpr int kChunk = 128 * 128;     // bytes of [128 rows x 64 f16]

struct TcShared {
  uint64_t q_full[2], s_full[2], p_full[2], o_done[2];   // of the tiles
  uint64_t pair[2][4];                                   // of the two warps that share 32 rows
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t scale_full[kTcRing];
  uint32_t tmem_base;
  int abort_flag;
  float4 group[16][4];                    // per warp: of each of its 16-token groups {K scale, V scale's exponent in the reference,
                                          // what takes it off a sum of weights, its exponent in the weights}
  float q_scale[2][128];                  // [tile][row]: what a score is multiplied by
  float swap[2][2][2][128];               // [step parity][tile][half][row]: what the two threads of a row tell each other
  uint32_t there[kTcRing];                // of the 16-token groups of a step: a bit each, not there at all: 0
  alignas(16) float ks[kTcRing][8], vs[kTcRing][8];
  DivisionShared division;
};

// ---------------------------------------------------------------------------------------------- instructions
// The issuing warp stays converged: all lanes run its control flow and compute the descriptors, which are warp-uniform, and one
// elected lane issues.  (Inside a branch of one lane every descriptor has to go through vector registers: 100 cycles a product.)
// Four products of 16 inner elements each; the operands' descriptors advance by step_a (or columns) and step_b.
__device__ __forceinline__ void umma_f16_ss_x4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred e, p;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "add.u64 a1, %1, 2;\n\tadd.u64 a2, %1, 4;\n\tadd.u64 a3, %1, 6;\n\t"
      "add.u64 b1, %2, 2;\n\tadd.u64 b2, %2, 4;\n\tadd.u64 b3, %2, 6;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a1, b1, %3, 1;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a2, b2, %3, 1;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a3, b3, %3, 1;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(accumulate))
      : "memory");
}
// A operand in tensor memory: row i in lane i, two f16 in a column; 16 rows of 128 bytes of B a product
__device__ __forceinline__ void umma_f16_ts_x4(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred e, p;\n\t.reg .b32 a1, a2, a3;\n\t.reg .b64 b1, b2, b3;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "add.u32 a1, %1, 8;\n\tadd.u32 a2, %1, 16;\n\tadd.u32 a3, %1, 24;\n\t"
      "add.u64 b1, %2, 128;\n\tadd.u64 b2, %2, 256;\n\tadd.u64 b3, %2, 384;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a1], b1, %3, 1;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a2], b2, %3, 1;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a3], b3, %3, 1;\n\t}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(accumulate))
      : "memory");
}
// Arrives on `bar` when the products that the elected lane has issued so far are done
__device__ __forceinline__ void umma_commit_warp(uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(tc::smem_u32(bar)) : "memory");
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
// 16 bytes, or zeros: a predicated load, no branch around it
__device__ __forceinline__ uint4 ld_nc_16_if(const void* p, uint32_t on) {
  uint4 r;
  asm volatile(
      "{\n\t.reg .pred q;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "mov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
      "@q ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
      : "=&r"(r.x), "=&r"(r.y), "=&r"(r.z), "=&r"(r.w)
      : "l"(p), "r"(on));
  return r;
}
// The larger; NaN if one is
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// Two float32 operations in one instruction
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpair(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// Tensor-memory loads with their wait in one statement: between the two the compiler must not move a register, because its
// value is not there yet
__device__ __forceinline__ void tmem_read16(uint32_t taddr, uint32_t* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
        "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_read32(uint32_t taddr, uint32_t* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
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
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// The V scale of a block, in the reference of a row and in the exponent of its weights.  Tokens of a scale of 0 count in the
// denominator alone: 40 binades lower in the weights than in the reference, they are below 2^-25 and 0 in f16, and far from 0 in the
// float32 sum.  NaN stays NaN.
__device__ __forceinline__ float value_exponent(float s) { return s < 0x1p-126f ? -32.f : __log2f(s); }
__device__ __forceinline__ float weight_exponent(float s) { return (s < 0x1p-126f ? -72.f : __log2f(s)) + kWeightShift; }
// Its binade, held within what a reference follows; kNoScale where it is 0 or NaN
constexpr int kNoScale = -1000;
__device__ __forceinline__ int scale_binade(float s) {
  return s > 0.f ? min(max(static_cast<int>(__float_as_uint(s) >> 23) - 127, -30), 30) : kNoScale;
}

// A warp's wait for the first scores of a piece.  A tile that has no rows in the pieces before waits for all of those: the limit of
// the other waits, 4 s or some two million steps, is granted once more for every 2^17 tokens that a table has room for.  If another
// role gives up, so does this wait.
static __device__ __noinline__ bool wait_scores(uint64_t* bar, uint32_t parity, int more, volatile int* abort_flag) {
  bool got = false;
  for (int turn = 0; turn <= more && !got && !*abort_flag; ++turn)
    for (uint32_t i = 0; i < tc::kSpinLimit && !got; ++i) {
      got = tc::mbar_try_wait(bar, parity);
      if ((i & 1023u) == 1023u && *abort_flag) break;
    }
  if (!got) *abort_flag = 1;
  return __all_sync(0xffffffffu, got);
}

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
      mbar_init(&sh.q_full[i], 8); mbar_init(&sh.s_full[i], 1); mbar_init(&sh.p_full[i], 8); mbar_init(&sh.o_done[i], 1);
      for (int k = 0; k < 4; ++k) mbar_init(&sh.pair[i][k], 2);
      mbar_init(&sh.k_full[i], 8); mbar_init(&sh.k_empty[i], 1); mbar_init(&sh.v_full[i], 8); mbar_init(&sh.v_empty[i], 1);
    }
    for (int i = 0; i < kTcRing; ++i) mbar_init(&sh.scale_full[i], 1);
    sh.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kTcIssuer) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)), "n"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem_base;              // scores of tile t at column 128 t; sums at 256 + 128 t
  grid_dependency_wait();
  TcStretch st = tc_locate<TcShape>(p, sh.division);
  if (threadIdx.x == 0) {
    if (blockIdx.x == 0) { p.status[0] = kStatusFlags | gridDim.x; p.status[1] = 0; }
    p.boundary[blockIdx.x].seg1 = 0;
    p.flags[blockIdx.x] = 0;
  }
  __syncthreads();
  bool bad = false;
  TcPiece pc;

  if (warp < kTcConverter) {
    // ============================================================ two threads a query row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 80;");
    const int tile = warp >> 3, half = (warp >> 2) & 1, quarter = warp & 3, r = quarter * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
    const uint32_t s_addr = tmem + lanes + tile * 128 + half * 64;                      // this thread's scores, and its weights
    const uint32_t o_addr = tmem + lanes + 256 + tile * 128 + half * (DP / 2);          // its half of the sums
    int n_piece = 0;         // pieces of this tile so far
    int n_it = 0;            // steps of this tile so far
    int step = 0;            // steps of the CTA so far
    int n_swap = 0;          // exchanges with the row's other thread so far
    bool ok = true;
    // Gives x to the row's other thread and returns what that gives
    auto swap = [&](float x) {
      sh.swap[n_swap & 1][tile][half][r] = x;
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.pair[tile][quarter]);
      ok = mbar_wait_warp(&sh.pair[tile][quarter], n_swap & 1, abort_flag);
      return sh.swap[n_swap++ & 1][tile][half ^ 1][r];
    };
    while (ok && tc_next<TcShape>(p, st, pc)) {
      const int steps = pc.u1 - pc.u0;
      if (pc.u0 > 0 && threadIdx.x == 0)
        p.boundary[blockIdx.x] = {pc.seg0, pc.seg1, st.quota, pc.b, pc.head, pc.tile, pc.q.s.first, pc.n_rows, 0};
      if (tile * 128 >= pc.n_rows) { step += steps; continue; }
      if (p.kv_len[pc.b] > pc.q.s.len) bad = true;
      const int in_tile = tile * 128 + r;
      const bool on = in_tile < pc.n_rows;
      const int flat = pc.tile * kTcRows + (on ? in_tile : 0), i_row = flat / p.group;
      const RowAt at = {i_row, pc.head * p.group + flat - i_row * p.group};
      const int seen = on ? visible(p, pc.q.s, i_row) : 0;

      // ---- the tile's queries: 16 bytes a thread and pass, each row's largest element among the lanes that have the row, a
      // power of two, f16 into the swizzled tile
      {
        constexpr int kLanes = DP / 8, kPass = 256 / kLanes, kPasses = 128 / kPass;
        const int t = threadIdx.x & 255, piece = t % kLanes, row0 = t / kLanes;
        uint4 raw[kPasses];
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
          const int row = tile * 128 + row0 + i * kPass, f = pc.tile * kTcRows + row, new_row = f / p.group;
          raw[i] = make_uint4(0, 0, 0, 0);
          if (row < pc.n_rows && piece * 8 < D)
            raw[i] = ld_nc_16(q_at(p, pc.b, pc.q.s.first, RowAt{new_row, pc.head * p.group + f - new_row * p.group}) + piece * 16);
        }
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
          float f[8], top = 0.f;
          Vec16<__nv_bfloat16>::unpack(raw[i], f);
#pragma unroll
          for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(f[j]));
#pragma unroll
          for (int off = 1; off < kLanes; off <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
          const int e = max(static_cast<int>(__float_as_uint(top) >> 23) - 127, -100), row = row0 + i * kPass;
          const float up = copysignf(exp2_int(min(14 - e, 127)), p.scale_log2e);   // the factor of a score is kept positive
          if (piece == 0) sh.q_scale[tile][row] = exp2_int(max(e - 14, -126)) * fabsf(p.scale_log2e);
          const uint4 w = make_uint4(pack_f16(f[0] * up, f[1] * up), pack_f16(f[2] * up, f[3] * up), pack_f16(f[4] * up, f[5] * up),
                                     pack_f16(f[6] * up, f[7] * up));
          *reinterpret_cast<uint4*>(q_sh + tile * kTileBytes + (piece >> 3) * kChunk + row * 128 + (((piece & 7) ^ (row & 7)) << 4)) = w;
        }
        fence_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_full[tile]);
        ok = mbar_wait_warp(&sh.q_full[tile], n_piece++ & 1, abort_flag);
        // A tile that had nothing to do in the piece before may be steps ahead of the converters, and a wait tells a phase from
        // the next only: the first scores of a piece are waited for before its first scales.
        ok = ok && wait_scores(&sh.s_full[tile], n_it & 1, p.max_blocks >> (17 - p.shift), abort_flag);
        if (!ok) break;
      }
      const float cq = sh.q_scale[tile][r];

      // m: the row's reference, a score plus its V scale's logarithm; weights are 2^8 at it, l in units of 2^m
      float m = -INFINITY, l = 0.f;
      float peak = -INFINITY;  // the largest that m has been, less the scales that it stood for
      int binade = -30;        // of the V scales that m stands for
      for (int j = 0; j < steps && ok; ++j, ++n_it, ++step) {
        const int slot = step & (kTcRing - 1);
        ok = mbar_wait_warp(&sh.scale_full[slot], (step / kTcRing) & 1, abort_flag);
        if (!ok) break;
        // ---- the scales, and what follows from them for all rows alike
        const float k8 = sh.ks[slot][lane & 7], v8 = sh.vs[slot][lane & 7];
        const uint32_t there = sh.there[slot];
        const bool odd = __any_sync(0xffffffffu, k8 != k8 || v8 != v8);
        if ((lane >> 2) == half) {
          const float up = weight_exponent(v8);
          sh.group[warp][lane & 3] = make_float4(k8, value_exponent(v8), ex2(-up), up);
        }
        __syncwarp();
        if (j > 0) ok = mbar_wait_warp(&sh.s_full[tile], n_it & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        const float4* group = sh.group[warp];
        // the columns that this row sees, 32 to a word
        const int vis = seen - (pc.u0 + j) * kTcKeys - half * 64;
        const uint32_t there4 = (there >> (half * 4)) & 15u;
        const bool masked = __any_sync(0xffffffffu, vis < 64) || there4 != 15u;
        auto hide = [&](uint32_t* v, int h, uint32_t with) {
          const int n = vis - h * 32;
          const uint32_t mask = (n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u) &
                                (((there4 >> (2 * h)) & 1u ? 0xffffu : 0u) | ((there4 >> (2 * h + 1)) & 1u ? 0xffff0000u : 0u));
#pragma unroll
          for (int k = 0; k < 32; ++k)
            if (!((mask >> k) & 1u)) v[k] = with;
        };

        // ---- largest sum of a score and its V scale
        float top = -INFINITY;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t v[32];
          tmem_read32(s_addr + h * 32, v);
          if (masked) hide(v, h, 0xff800000u);   // -inf
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            float x = __uint_as_float(v[g * 16]);
#pragma unroll
            for (int k = 1; k < 15; k += 2) x = fmaxf(fmaxf(x, __uint_as_float(v[g * 16 + k])), __uint_as_float(v[g * 16 + k + 1]));
            x = fmaxf(x, __uint_as_float(v[g * 16 + 15]));
            if (x > -INFINITY) top = fmaxf(top, fmaf(x, cq * group[h * 2 + g].x, group[h * 2 + g].y));
          }
        }
        top = fmaxf(top, swap(top));
        if (!ok) break;
        // ---- the largest V scale that this row sees in the step: its groups are the first ones.  (Taken here rather than beside the other
        // scales: one register less over the scores, 682 us against 688.)
        int up_to = scale_binade(sh.vs[slot][lane & 7]);
        const int groups = min(max(seen - (pc.u0 + j) * kTcKeys + 15, 0) >> 4, 8);
        if (__all_sync(0xffffffffu, groups == 8)) {
          up_to = __reduce_max_sync(0xffffffffu, up_to);
        } else {
#pragma unroll
          for (int off = 1; off < 8; off <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, up_to, off, 8);
            if ((lane & 7) >= off) up_to = max(up_to, x);
          }
          up_to = __shfl_sync(0xffffffffu, up_to, max(groups - 1, 0));
          if (groups == 0) up_to = kNoScale;
        }
        // ---- a new reference rescales the sums, which is rare.  Both threads of a row decide alike.
        float f = 1.f;
        binade = max(binade, up_to);
        const bool down = static_cast<unsigned>(binade - up_to - kFollow - 1) < 128u;       // and there is such a scale
        if (__any_sync(0xffffffffu, top > m + kLazy || down)) {
          if (down) binade = up_to;
          const float now = fmaxf(down ? fminf(m, peak + static_cast<float>(binade)) : m, top);
          f = now == -INFINITY ? 1.f : ex2(m - now);
          peak = fmaxf(peak, now - static_cast<float>(binade));
          m = now;
          l *= f;
        }
        if (j > 0 && __any_sync(0xffffffffu, f != 1.f)) {
          // (the products with V of the step before are done: this step's scores were issued after them)
#pragma unroll 1
          for (int c = 0; c < DP / 2; c += 16) {
            uint32_t x[16];
            tmem_read16(o_addr + c, x);
#pragma unroll
            for (int k = 0; k < 16; ++k) x[k] = __float_as_uint(__uint_as_float(x[k]) * f);
            tmem_st16(o_addr + c, x);
          }
        }
        // ---- weights over the scores, read a second time (the registers hold 32): the columns that a chunk is written to have
        // been read before
        const float minus_m = m == -INFINITY ? 0.f : -m;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t v[32], w[16];
          tmem_read32(s_addr + h * 32, v);
          if (masked) hide(v, h, 0xff800000u);   // -inf, and a weight of 0: the factor is held above 0
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const float4 gr = group[h * 2 + g];
            const float fk = max_nan(cq * gr.x, 0x1p-126f), shifted = minus_m + gr.w;
            const uint64_t mul = pair(fk, fk), add = pair(shifted, shifted);
#pragma unroll
            for (int k = g * 16; k < g * 16 + 16; k += 2) {
              const float2 x = unpair(fma2(pair(__uint_as_float(v[k]), __uint_as_float(v[k + 1])), mul, add));
              v[k] = __float_as_uint(ex2(x.x));
              v[k + 1] = __float_as_uint(ex2(x.y));
            }
          }
          if (masked && odd) hide(v, h, 0u);     // scales that are NaN reach who sees them only
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            uint64_t sums = 0;
#pragma unroll
            for (int k = 0; k < 16; k += 2) {
              const float w0 = __uint_as_float(v[g * 16 + k]), w1 = __uint_as_float(v[g * 16 + k + 1]);
              sums = add2(sums, pair(w0, w1));
              w[g * 8 + k / 2] = pack_f16(w0, w1);
            }
            const float2 both = unpair(sums);
            const float sum = both.x + both.y;
            if (sum != 0.f) l = fmaf(sum, group[h * 2 + g].z, l);   // (not where nothing is seen: the factor may be NaN)
          }
          tmem_st16(s_addr + h * 16, w);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_full[tile]);
      }
      if (!ok) break;
      // ---- results
      l += swap(l);
      ok = ok && mbar_wait_warp(&sh.o_done[tile], (n_it - 1) & 1, abort_flag);
      if (!ok) break;
      tc_fence_after();
      const bool complete = pc.u0 == 0 && pc.u1 == pc.units;
      const float unit = 1.f / kWeightScale, mul = complete ? (l == 0.f ? 0.f : unit / l) : unit;
      float* part = p.partial + (static_cast<size_t>(blockIdx.x) * 2 + (pc.u0 == 0 ? 1 : 0)) * partial_floats(kTcRows, D);
      char* out = out_at(p, pc.b, pc.q.s.first, at);
#pragma unroll 1
      for (int i = 0; i < DP / 2; i += 16) {
        uint32_t v[16];
        tmem_read16(o_addr + i, v);
        const int c = half * (DP / 2) + i;
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
      if (on && half == 0) {
        if (!complete) { part[kTcRows * D + in_tile] = m; part[kTcRows * D + kTcRows + in_tile] = l; }
        else if (p.lse) *lse_at(p, pc.b, pc.q.s.first, at) = log_sum(m, l);
      }
    }
  } else if (warp < kTcIssuer) {
    // ============================================================ codes to f16
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    constexpr int kPer = DP / 16, kRowsPass = 256 / kPer, kLoads = 64 / kRowsPass;   // pieces of a token; tokens of a pass; loads of an item
    const int tid = threadIdx.x - kTcConverter * 32, piece = tid % kPer, row0 = tid / kPer;
    const bool in_dim = piece * 16 < D;
    const size_t cell_bytes = static_cast<size_t>(p.block_size) * D;
    int step = 0;
    bool ok = true;
    while (ok && tc_next<TcShape>(p, st, pc)) {
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
      // An item is 64 keys of K or of V: four a step (K, K, V, V), two of them on their way while one is turned
      uint4 raw[2][kLoads];
      const unsigned rows_mask = static_cast<unsigned>(p.block_size - 1);
      auto load = [&](uint4* raw, const uint8_t* cache, int blk, int t0, int part) {    // part: 64 keys of the step
        const uint8_t* mine = cache + piece * 16;
        const unsigned cell = static_cast<unsigned>(blk) * static_cast<unsigned>(p.kv_heads) + static_cast<unsigned>(pc.head);
        const uint8_t* at[kLoads];
        uint32_t on[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {       // the 16-token group of a load is the same for all lanes
          const int row = part * 64 + row0 + i * kRowsPass, group = part * 4 + (warp - kTcConverter) * (32 / kPer) / 16 + i * kRowsPass / 16;
          const unsigned c = __shfl_sync(0xffffffffu, cell, group);
          const int block = __shfl_sync(0xffffffffu, blk, group);      // by all lanes, whatever they load
          on[i] = in_dim && t0 + row < pc.most && block >= 0;
          at[i] = mine + static_cast<size_t>(c) * static_cast<unsigned>(cell_bytes) + ((t0 + row) & rows_mask) * static_cast<unsigned>(D);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) raw[i] = ld_nc_16_if(at[i], on[i]);
      };
      auto store = [&](const uint4* raw, unsigned char* dst, int part) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int row = part * 64 + row0 + i * kRowsPass;
          const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
          uint32_t h[8];
#pragma unroll
          for (int k = 0; k < 4; ++k) codes_to_f16<KV>(w[k], h[2 * k], h[2 * k + 1]);
          unsigned char* at = dst + (piece >> 2) * kChunk + row * 128;
          const int c16 = (piece & 3) * 2;
          *reinterpret_cast<uint4*>(at + ((c16 ^ (row & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
          *reinterpret_cast<uint4*>(at + (((c16 + 1) ^ (row & 7)) << 4)) = make_uint4(h[4], h[5], h[6], h[7]);
        }
      };
      int blk = blocks_at(pc.u0 * kTcKeys);
      load(raw[0], p.k_cache, blk, pc.u0 * kTcKeys, 0);
      load(raw[1], p.k_cache, blk, pc.u0 * kTcKeys, 1);
      int next = pc.u0 + 1 < pc.u1 ? blocks_at((pc.u0 + 1) * kTcKeys) : -1;
      for (int u = pc.u0; u < pc.u1 && ok; ++u, ++step) {
        const int s = step & 1, slot = step & (kTcRing - 1), t0 = u * kTcKeys;
        const bool more = u + 1 < pc.u1;
        if (step >= 2) ok = mbar_wait_warp(&sh.k_empty[s], ((step >> 1) - 1) & 1, abort_flag);
        if (!ok) break;
        float scale = 0.f;         // lanes 0-7 K, 8-15 V, of the first warp: on its way while the keys are turned
        const int b8 = __shfl_sync(0xffffffffu, blk, lane & 7);
        if (warp == kTcConverter) {
          const size_t cell = static_cast<size_t>(max(b8, 0)) * p.kv_heads + pc.head;
          if (lane < 16 && b8 >= 0) scale = __ldg((lane < 8 ? p.k_scale : p.v_scale) + cell);
        }
        store(raw[0], k_sh + s * kTileBytes, 0);
        load(raw[0], p.v_cache, blk, t0, 0);
        store(raw[1], k_sh + s * kTileBytes, 1);
        fence_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.k_full[s]);
        load(raw[1], p.v_cache, blk, t0, 1);
        if (warp == kTcConverter) {
          if (lane < 8) sh.ks[slot][lane] = b8 >= 0 ? scale : 1.f;      // (a group that is not there is masked; its V scale is 0)
          else if (lane < 16) sh.vs[slot][lane - 8] = scale;
          const unsigned there = __ballot_sync(0xffffffffu, blk >= 0);
          if (lane == 0) sh.there[slot] = there & 0xffu;
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.scale_full[slot]);
        }
        if (step >= 2) ok = mbar_wait_warp(&sh.v_empty[s], ((step >> 1) - 1) & 1, abort_flag);
        if (!ok) break;
        store(raw[0], v_sh + s * kTileBytes, 0);
        if (more) load(raw[0], p.k_cache, next, t0 + kTcKeys, 0);
        store(raw[1], v_sh + s * kTileBytes, 1);
        fence_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.v_full[s]);
        if (more) load(raw[1], p.k_cache, next, t0 + kTcKeys, 1);
        blk = next;
        next = u + 2 < pc.u1 ? blocks_at(t0 + 2 * kTcKeys) : -1;
      }
    }
  } else {
    // ============================================================ products
    {
      const uint32_t qk = idesc_f16(kTcKeys, false), pv = idesc_f16(DP, true);
      const uint32_t q_addr = smem_u32(q_sh), k_addr = smem_u32(k_sh), v_addr = smem_u32(v_sh);
      int step = 0, n_it[2] = {0, 0}, n_piece[2] = {0, 0};
      bool ok = true;
      auto scores = [&](int t, int s) {        // S of tile t from stage s of K
        const uint64_t a = smem_desc_sw128(q_addr + t * kTileBytes), b = smem_desc_sw128(k_addr + s * kTileBytes);
#pragma unroll
        for (int c = 0; c < kDChunks; ++c) umma_f16_ss_x4(tmem + t * 128, a + c * (kChunk >> 4), b + c * (kChunk >> 4), qk, c > 0);
        umma_commit_warp(&sh.s_full[t]);
      };
      while (ok && tc_next<TcShape>(p, st, pc)) {
        const int two = pc.n_rows > 128;
        for (int t = 0; t <= two && ok; ++t) ok = mbar_wait_warp(&sh.q_full[t], n_piece[t]++ & 1, abort_flag);
        ok = ok && mbar_wait_warp(&sh.k_full[step & 1], (step >> 1) & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        for (int t = 0; t <= two; ++t) scores(t, step & 1);
        umma_commit_warp(&sh.k_empty[step & 1]);
        for (int u = pc.u0; u < pc.u1 && ok; ++u, ++step) {
          const int s = step & 1;
          const bool more = u + 1 < pc.u1;
          ok = mbar_wait_warp(&sh.v_full[s], (step >> 1) & 1, abort_flag);
#pragma unroll 1
          for (int t = 0; t <= two && ok; ++t) {
            ok = mbar_wait_warp(&sh.p_full[t], n_it[t] & 1, abort_flag);
            if (!ok) break;
            tc_fence_after();
            const uint64_t b = desc_mn(v_addr + s * kTileBytes);
            umma_f16_ts_x4(tmem + 256 + t * 128, tmem + t * 128, b, pv, u > pc.u0);
            umma_f16_ts_x4(tmem + 256 + t * 128, tmem + t * 128 + 64, b + (64 * 128 >> 4), pv, true);
            umma_commit_warp(&sh.o_done[t]);
            if (t == two) umma_commit_warp(&sh.v_empty[s]);
            if (more) {        // the weights that lie where the next scores go have to be used up, not only issued
              if (t == 0) ok = mbar_wait_warp(&sh.k_full[s ^ 1], ((step + 1) >> 1) & 1, abort_flag);
              ok = ok && mbar_wait_warp(&sh.o_done[t], n_it[t] & 1, abort_flag);
              if (!ok) break;
              tc_fence_after();
              scores(t, s ^ 1);
              if (t == two) umma_commit_warp(&sh.k_empty[s ^ 1]);
            }
            ++n_it[t];
          }
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
  if (warp == kTcIssuer) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
  }
}

}  // namespace kv
}  // namespace vscan
