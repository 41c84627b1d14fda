// Attention of few query rows (decode steps, drafts) for bf16 queries: the products run as m16n8k16 matrix instructions with
// f16 operands and float32 sums, the tokens and channels of the cache as the 16-row side (two rows of a decode step would
// leave a 128-row tensor-memory tile empty; the cache has to come through the registers to be turned from codes anyway).
//
//   S^T [16 tokens x 8 rows] = K [16 tokens x d] q^T         O^T [16 channels x 8 rows] += V^T [16 channels x 16 tokens] P^T
//
// Which channel stands at which place of the inner dimension of the first product, and which channel at which row of the
// second, is free as long as both operands agree.  They are chosen such that a lane's codes are consecutive bytes: K and V go
// from global memory straight into the fragments, 16 bytes a load, no shared memory and no shuffle, and V is transposed by
// the byte permutes that pair two tokens' codes.  P^T comes from S^T by an 8 x 8 transpose instruction.
//
// Roundings: codes are exact in f16; a query row is scaled by a power of two to 2^14 .. 2^15 at its largest element, so that
// its f16 form is exact down to 2^-28 of it; weights are rounded to f16: 2^-11 relative, down to 2^-22 of the largest one.  The block's
// V scale is part of a weight's exponent (and is taken off again for the denominator), so that this is the largest of what adds to
// the result, not of the softmax alone.  A scale of 0 makes its codes 0.  Scores, references, denominators and sums are float32.
//
// Measured: 256 sequences of 195 to 300 tokens, 32 heads of 128, 522 MB: 115 us, 4.5 TB/s, issue slots 43 % and ALU 42 % busy; 4
// sequences of 9,000 to 16,500 tokens, 4 KV heads, 44 MB: 23 us and 5 for the join.  Four CTAs of four warps an SM, 4 KB a warp on
// their way.  Codes through shared memory, three steps deep: 139 us where each lane copies its own, 108 us by bulk copies, which
// took 10 % longer for few long sequences and 15 % for tiny ones.  Division in units of 16 tokens instead of 64: 112 us, but half
// as long again for 114 sequences of up to 9 tokens.
#pragma once

#include "kv_attention.cuh"

namespace vscan {
namespace kv {

constexpr int kMmaThreads = 128;
constexpr float kLazy = 6.f;          // a running maximum is raised when a score is over it by this many binades: weights up to 2^6 times
                                      // kWeightScale, 2^14 in f16

__device__ __forceinline__ float follow_bounds(float binade) { return fminf(fmaxf(binade, -30.f), 30.f); }

__device__ __forceinline__ void mma_f16(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Bytes 0, 1 and bytes 2, 3 of a word of codes as two f16 pairs
template <int KV>
__device__ __forceinline__ void codes_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if constexpr (KV == VSCAN_KV_E4M3) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi) : "r"(w));
  } else {
    // code + 128 as the last byte of an f16 between 1024 and 1279, less 1152
    const uint32_t u = w ^ 0x80808080u, bias = 0x64806480u;
    const uint32_t l = __byte_perm(u, 0x64646464u, 0x4140), h = __byte_perm(u, 0x64646464u, 0x4342);
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(l), "r"(bias));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(h), "r"(bias));
  }
}

__device__ __forceinline__ uint2 ld_nc_8(const void* p) {
  uint2 r;
  asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(p));
  return r;
}

// DP: head_dim rounded up to 64, 128 or 256.  NT: tiles of 8 query rows.  MT: groups of 16 tokens of a step.  FULL: head_dim is DP,
// so that where a lane's pieces lie within a block is known at compile time.
template <int KV, int DP, int NT, int MT, bool FULL>
__global__ void __launch_bounds__(kMmaThreads, DP == 256 || NT > 1 ? 2 : 4) mma_kernel(AttnParams p) {
  constexpr int R = 8 * NT, KS = DP / 16, kPieces = DP / 64, kStep = 16 * MT;
  constexpr int kVWords = DP / 32;                   // 32-bit words of V codes of a lane and token
  extern __shared__ __align__(16) float attn_smem[];
  float* o_sh = attn_smem;                           // [warps][R][DP], then maxima [warps][R], denominators [warps][R]
  float* m_sh = o_sh + 4 * R * DP;
  float* l_sh = m_sh + 4 * R;
  __shared__ ScheduleShared sched;
  __shared__ float peaks[NT][2][kMmaThreads];         // of each lane's rows: the largest that the reference has been, less the scales that it
                                                      // stood for
  __shared__ Stretch stretches[kMmaThreads / 32];     // of each warp: too much for its registers
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const int D = FULL ? DP : p.head_dim;
  grid_dependency_wait();
  if (threadIdx.x == 0) p.flags[blockIdx.x] = 0;     // before the barriers in locate(): any warp may set it behind them
  Stretch& st = stretches[threadIdx.x >> 5];
  {
    const Stretch found = locate<kMmaThreads, true>(p, sched);
    if (lane == 0) st = found;
    __syncwarp();
  }
  const int worker = st.worker;
  const bool solo = st.solo;
  if (blockIdx.x == 0 && threadIdx.x == 0) { p.status[0] = kStatusFlags | gridDim.x; p.status[1] = solo; }
  const bool writes_boundary = lane == 0 && (solo || warp == 0);
  if (writes_boundary) p.boundary[worker].seg1 = 0;
  bool bad = false;
  while (true) {
    Piece pc = {0, 0};
    __syncwarp();
    if (lane == 0) next_piece(p, st, pc);
    __syncwarp();                                     // a shuffle alone does not order what the lanes read of st
    pc.u0 = __shfl_sync(0xffffffffu, pc.u0, 0);
    pc.u1 = __shfl_sync(0xffffffffu, pc.u1, 0);
    if (pc.u1 == 0) break;
    const Sequence& s = st.s;
    const int b = st.b, head = st.head, tile = st.tile;
    const int n_rows = min(R, s.n * p.group - tile * R);
    if (pc.u0 > 0 && writes_boundary) p.boundary[worker] = {st.seg0, st.seg0 + s.units, st.quota, b, head, tile, s.first, n_rows, 0};
    if (p.kv_len[b] > s.len) bad = true;

    const int32_t* table = p.block_table + static_cast<size_t>(b) * p.max_blocks;
    const size_t cell_bytes = static_cast<size_t>(p.block_size) * D;
    const int last_row = tile * R + n_rows - 1;
    const int most = visible(p, s, last_row / p.group);
    const int stop = min(most, pc.u1 * kUnit);
    const int t_first = pc.u0 * kUnit + (solo ? 0 : warp * kStep), t_stride = solo ? kStep : 4 * kStep;

    // ---- loads of a step: block numbers, codes, scales
    int blk[MT], blk_next[MT];
    float ks[MT], vsc[MT];
    uint4 kraw[MT][2][kPieces];
    uint32_t vraw[MT][4][kVWords];
    auto load_table = [&](int t0, int* out) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int t = t0 + 16 * m;
        int x = -1;
        if (t < stop) {
          x = table[t >> p.shift];
          if (x < 0 || x >= p.num_blocks) { x = -1; bad = true; }
        }
        out[m] = x;
      }
    };
    // A step that is there in full is loaded without conditions; the last one, and one with missing blocks, piece by piece,
    // zeros for what is not there.
    auto load_k = [&](int t0) {
      bool full = FULL && t0 + kStep <= stop;
#pragma unroll
      for (int m = 0; m < MT; ++m) full = full && blk[m] >= 0;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int t = t0 + 16 * m;
        const size_t cell = static_cast<size_t>(max(blk[m], 0)) * p.kv_heads + head;
        const uint8_t* base = p.k_cache + cell * cell_bytes + ((t & (p.block_size - 1)) + g) * D + c * 16;
        if (full) {
          ks[m] = __ldg(p.k_scale + cell);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < kPieces; ++i) kraw[m][h][i] = ld_nc_16(base + h * 8 * D + i * 64);
        } else {
          ks[m] = 0.f;
          if (blk[m] >= 0) ks[m] = __ldg(p.k_scale + cell);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
              kraw[m][h][i] = make_uint4(0, 0, 0, 0);
              if (blk[m] >= 0 && t + 8 * h + g < stop && i * 64 + c * 16 < D) kraw[m][h][i] = ld_nc_16(base + h * 8 * D + i * 64);
            }
        }
      }
    };
    auto load_v = [&](int t0) {
      bool full = FULL && t0 + kStep <= stop;
#pragma unroll
      for (int m = 0; m < MT; ++m) full = full && blk[m] >= 0;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int t = t0 + 16 * m;
        const size_t cell = static_cast<size_t>(max(blk[m], 0)) * p.kv_heads + head;
        const uint8_t* base = p.v_cache + cell * cell_bytes + ((t & (p.block_size - 1)) + 2 * c) * D + g * (DP == 64 ? 8 : 16);
        vsc[m] = 0.f;
        if (full || blk[m] >= 0) vsc[m] = __ldg(p.v_scale + cell);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int tok = (k & 1) + (k >> 1) * 8;
          const bool on = full || (blk[m] >= 0 && t + 2 * c + tok < stop);
          if constexpr (DP == 64) {
            uint2 v = make_uint2(0, 0);
            if (full) v = ld_nc_8(base + tok * D);
            else if (on && g * 8 < D) v = ld_nc_8(base + tok * D);
            vraw[m][k][0] = v.x; vraw[m][k][1] = v.y;
          } else {
#pragma unroll
            for (int i = 0; i < DP / 128; ++i) {
              uint4 v = make_uint4(0, 0, 0, 0);
              if (full) v = ld_nc_16(base + tok * D + i * 128);
              else if (on && i * 128 + g * 16 < D) v = ld_nc_16(base + tok * D + i * 128);
              vraw[m][k][4 * i] = v.x; vraw[m][k][4 * i + 1] = v.y; vraw[m][k][4 * i + 2] = v.z; vraw[m][k][4 * i + 3] = v.w;
            }
          }
        }
      }
    };
    // the queries' loads first: they wait for nothing else
    uint4 q_raw[NT][kPieces][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = nt * 8 + g;
      const char* src = q_at(p, b, s.first, row_at(p, tile, head, r < n_rows ? r : 0));
#pragma unroll
      for (int i = 0; i < kPieces; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          q_raw[nt][i][k] = make_uint4(0, 0, 0, 0);
          if (r < n_rows && i * 64 + c * 16 < D) q_raw[nt][i][k] = ld_nc_16(src + (i * 64 + c * 16) * 2 + k * 16);
        }
    }
    load_table(t_first, blk);
    load_k(t_first);
    load_v(t_first);
    load_table(t_first + t_stride, blk_next);
    // Workers that are CTAs have little to do each and wait for DRAM most of the time: all their blocks (128 at most) are asked
    // into L2 at once, a thread a block.  (Not so for warps: there is enough under way, and it made them slower.)
    if (!solo) {
      const int j = (pc.u0 * kUnit >> p.shift) + threadIdx.x;
      if (static_cast<long long>(j) << p.shift < stop) {
        const int x = table[j];
        if (x >= 0 && x < p.num_blocks) {
          const size_t at = (static_cast<size_t>(x) * p.kv_heads + head) * cell_bytes;
          asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p.k_cache + at), "r"(static_cast<uint32_t>(cell_bytes)) : "memory");
          asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p.v_cache + at), "r"(static_cast<uint32_t>(cell_bytes)) : "memory");
        }
      }
    }

    // ---- queries: fragments of the rows g of each tile, scaled by a power of two; what a score is multiplied by
    uint32_t qf[KS][NT][2];
    float cq[NT][2], m[NT][2], l[NT][2];
    int seen[NT][2];
    int fewest = 0x7fffffff;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float f[8];
          Vec16<__nv_bfloat16>::unpack(q_raw[nt][i][k], f);
#pragma unroll
          for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(f[j]));
        }
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
          Vec16<__nv_bfloat16>::unpack(q_raw[nt][i][k], f);
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            qf[i * 4 + k * 2 + w][nt][0] = pack_f16(f[4 * w] * up, f[4 * w + 1] * up);
            qf[i * 4 + k * 2 + w][nt][1] = pack_f16(f[4 * w + 2] * up, f[4 * w + 3] * up);
          }
        }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int row = nt * 8 + 2 * c + k;
        cq[nt][k] = __shfl_sync(0xffffffffu, down, (2 * c + k) * 4) * p.scale_log2e;
        m[nt][k] = -INFINITY; l[nt][k] = 0.f;
        seen[nt][k] = row < n_rows ? visible(p, s, row_at(p, tile, head, row).i) : 0;
        fewest = min(fewest, row < n_rows ? seen[nt][k] : 0x7fffffff);
      }
    }
    fewest = min(fewest, __shfl_xor_sync(0xffffffffu, fewest, 1));
    fewest = min(fewest, __shfl_xor_sync(0xffffffffu, fewest, 2));
    float o[KS][NT][4];
#pragma unroll
    for (int i = 0; i < KS; ++i)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[i][nt][k] = 0.f;

#pragma unroll
    for (int nt = 0; nt < NT; ++nt) peaks[nt][0][threadIdx.x] = peaks[nt][1][threadIdx.x] = -INFINITY;
    float low = -1000.f;                // kFollow below the V scales that the references stand for; a scale of 0 is below that always

    for (int t0 = t_first; t0 < stop; t0 += t_stride) {
      // ---- scores
      float x[MT][NT][4];
      bool there[MT];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        there[mt] = blk[mt] >= 0;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int k = 0; k < 4; ++k) x[mt][nt][k] = 0.f;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          const uint32_t w0[4] = {kraw[mt][0][i].x, kraw[mt][0][i].y, kraw[mt][0][i].z, kraw[mt][0][i].w};
          const uint32_t w1[4] = {kraw[mt][1][i].x, kraw[mt][1][i].y, kraw[mt][1][i].z, kraw[mt][1][i].w};
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            uint32_t a[4];
            codes_to_f16<KV>(w0[w], a[0], a[2]);
            codes_to_f16<KV>(w1[w], a[1], a[3]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_f16(x[mt][nt], a, qf[i * 4 + w][nt][0], qf[i * 4 + w][nt][1]);
          }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float f0 = cq[nt][0] * ks[mt], f1 = cq[nt][1] * ks[mt];
          x[mt][nt][0] *= f0; x[mt][nt][1] *= f1; x[mt][nt][2] *= f0; x[mt][nt][3] *= f1;
        }
      }
      // masked: behind the row's last token, or in a block that is not there
      bool all = t0 + kStep <= fewest;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) all = all && there[mt];
      if (!all) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const int t = t0 + 16 * mt + g;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (!there[mt] || t + (k >> 1) * 8 >= seen[nt][k & 1]) x[mt][nt][k] = -INFINITY;
        }
      }
      // the next step's keys replace this one's; its values follow once this step's are used up
      float vs_now[MT];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) { blk[mt] = blk_next[mt]; vs_now[mt] = vsc[mt]; }
      const int t1 = t0 + t_stride;
      load_k(t1);
      load_table(t1 + t_stride, blk_next);

      // ---- references, largest sums of a score and its V scale's exponent: raised only when one is well over them, lowered only when
      // the scales come down, so that the sums are seldom rescaled
      float lv[MT];
      bool over = false;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        lv[mt] = __log2f(vs_now[mt]);
        low = fmaxf(low, lv[mt] - kFollow);
        over = over || lv[mt] < low;                    // (so is the scale 0)
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) over = over || fmaxf(x[mt][nt][k], x[mt][nt][k + 2]) + lv[mt] > m[nt][k] + kLazy;
      if (__any_sync(0xffffffffu, over)) {
        bool down = false;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          if (lv[mt] == -INFINITY) {      // a scale of 0: no value, whatever the codes are; the tokens count in the denominator
            lv[mt] = -48.f;
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int w = 0; w < kVWords; ++w) vraw[mt][k][w] = 0;
          }
          if (there[mt] && lv[mt] < low) {
            low = lv[mt] - kFollow;
            down = true;
          }
        }
        const float binade = follow_bounds(low + kFollow);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float& peak = peaks[nt][k][threadIdx.x];
            float top = down ? fminf(m[nt][k], peak + binade) : m[nt][k];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) top = fmaxf(top, fmaxf(x[mt][nt][k], x[mt][nt][k + 2]) + lv[mt]);
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            const float f = top == -INFINITY ? 1.f : ex2(m[nt][k] - top);
            m[nt][k] = top;
            peak = fmaxf(peak, top - binade);
            l[nt][k] *= f;
#pragma unroll
            for (int i = 0; i < KS; ++i) { o[i][nt][k] *= f; o[i][nt][k + 2] *= f; }
          }
      }
      // ---- weights, and their sums with the values
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const float up = lv[mt] + kWeightShift, down = ex2(-up);
        uint32_t pb[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float e[4];
          if (all) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              e[k] = ex2(x[mt][nt][k] + (up - m[nt][k & 1]));
              l[nt][k & 1] = fmaf(e[k], down, l[nt][k & 1]);
            }
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              // a masked score is -inf: so may be the reference of a row that has seen nothing yet, and the scale may be NaN
              const bool on = x[mt][nt][k] != -INFINITY;
              e[k] = on ? ex2(x[mt][nt][k] + (up - m[nt][k & 1])) : 0.f;
              if (on) l[nt][k & 1] = fmaf(e[k], down, l[nt][k & 1]);
            }
          }
          pb[nt][0] = transpose8x8(pack_f16(e[0], e[1]));
          pb[nt][1] = transpose8x8(pack_f16(e[2], e[3]));
        }
#pragma unroll
        for (int w = 0; w < kVWords; ++w) {
          const uint32_t t0w = vraw[mt][0][w], t1w = vraw[mt][1][w], t2w = vraw[mt][2][w], t3w = vraw[mt][3][w];
          uint32_t a[2][4];
          codes_to_f16<KV>(__byte_perm(t0w, t1w, 0x5140), a[0][0], a[0][1]);
          codes_to_f16<KV>(__byte_perm(t2w, t3w, 0x5140), a[0][2], a[0][3]);
          codes_to_f16<KV>(__byte_perm(t0w, t1w, 0x7362), a[1][0], a[1][1]);
          codes_to_f16<KV>(__byte_perm(t2w, t3w, 0x7362), a[1][2], a[1][3]);
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_f16(o[w * 2 + j][nt], a[j], pb[nt][0], pb[nt][1]);
        }
      }
      load_v(t1);
    }

    // ---- results.  Lane (g, c) has rows 2c, 2c + 1 of each tile; of the channels, word w of its values:
    // DP 64: 8 g + 4 w; else 128 (w / 4) + 16 g + 4 (w % 4); within a word o[2w][k], o[2w][k + 2], o[2w + 1][k], o[2w + 1][k + 2].
    constexpr float unit = 1.f / kWeightScale;
    const bool complete = pc.u0 == 0 && pc.u1 == s.units;
    float* part = p.partial + (static_cast<size_t>(worker) * 2 + (pc.u0 == 0 ? 1 : 0)) * partial_floats(R, D);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) l[nt][k] += __shfl_xor_sync(0xffffffffu, l[nt][k], off);
    if (solo) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int r = nt * 8 + 2 * c + k;
          if (r >= n_rows) continue;
          const RowAt at = row_at(p, tile, head, r);
          char* out = out_at(p, b, s.first, at);
          const float inv = complete ? (l[nt][k] == 0.f ? 0.f : unit / l[nt][k]) : unit;
#pragma unroll
          for (int w = 0; w < kVWords; ++w) {
            const int d = DP == 64 ? 8 * g + 4 * w : 128 * (w / 4) + 16 * g + 4 * (w % 4);
            if (d < D) {
              const float4 v = make_float4(o[2 * w][nt][k] * inv, o[2 * w][nt][k + 2] * inv, o[2 * w + 1][nt][k] * inv, o[2 * w + 1][nt][k + 2] * inv);
              if (complete) {
                const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
                *reinterpret_cast<uint2*>(out + d * 2) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
              } else {
                *reinterpret_cast<float4*>(part + r * D + d) = v;
              }
            }
          }
          if (g == 0) {
            if (!complete) { part[R * D + r] = m[nt][k]; part[R * D + R + r] = l[nt][k]; }
            else if (p.lse) *lse_at(p, b, s.first, at) = log_sum(m[nt][k], l[nt][k]);
          }
        }
    } else {
      __syncthreads();                              // the shared buffers of the piece before are done with
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int r = nt * 8 + 2 * c + k;
          if (r >= n_rows) continue;
#pragma unroll
          for (int w = 0; w < kVWords; ++w) {
            const int d = DP == 64 ? 8 * g + 4 * w : 128 * (w / 4) + 16 * g + 4 * (w % 4);
            *reinterpret_cast<float4*>(o_sh + (warp * R + r) * DP + d) =
                make_float4(o[2 * w][nt][k] * unit, o[2 * w][nt][k + 2] * unit, o[2 * w + 1][nt][k] * unit, o[2 * w + 1][nt][k + 2] * unit);
          }
          if (g == 0) { m_sh[warp * R + r] = m[nt][k]; l_sh[warp * R + r] = l[nt][k]; }
        }
      __syncthreads();
      for (int i = threadIdx.x; i < n_rows * (D / 4); i += kMmaThreads) {
        const int r = i / (D / 4), d = (i - r * (D / 4)) * 4;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, m_sh[w * R + r]);
        const float base = top == -INFINITY ? 0.f : top;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        float den = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float f = ex2(m_sh[w * R + r] - base);
          const float4 x = *reinterpret_cast<const float4*>(o_sh + (w * R + r) * DP + d);
          v.x = fmaf(f, x.x, v.x); v.y = fmaf(f, x.y, v.y); v.z = fmaf(f, x.z, v.z); v.w = fmaf(f, x.w, v.w);
          den = fmaf(f, l_sh[w * R + r], den);
        }
        if (complete) {
          const RowAt at = row_at(p, tile, head, r);
          const float inv = den == 0.f ? 0.f : 1.f / den;
          const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x * inv, v.y * inv), hi = __floats2bfloat162_rn(v.z * inv, v.w * inv);
          *reinterpret_cast<uint2*>(out_at(p, b, s.first, at) + d * 2) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
          if (d == 0 && p.lse) *lse_at(p, b, s.first, at) = log_sum(top, den);
        } else {
          *reinterpret_cast<float4*>(part + r * D + d) = v;
          if (d == 0) { part[R * D + r] = top; part[R * D + R + r] = den; }
        }
      }
    }
  }
  if (bad) p.flags[blockIdx.x] = VSCAN_ERR_INVALID_ARG;
  grid_dependency_launch();
}

}  // namespace kv
}  // namespace vscan
