// Joining the pieces of segments that the division of the work has cut.
//
// Where the stretch of worker k starts inside a segment that is cut there for the first time, the segment's rows from its
// pieces: the last piece of worker k - 1, then the first ones of k, k + 1, ... up to the segment's end.  The pieces are
// added in a fixed order, so results do not depend on timing.  Three shapes of the work:
//   few rows, workers are CTAs    a few segments in many pieces: a CTA looks at kJoinLook boundaries, its warps share the rows and
//                                 pieces of a segment that is cut there
//   few rows, workers are warps   many segments in two pieces or three: a warp takes a boundary
//   tiles of 64 to 256 rows       a CTA takes join_rows of them: their factors first, then all their channels side by side
#pragma once

#include "kv_attention.cuh"

namespace vscan {
namespace kv {

constexpr int kJoinThreads = 512;
constexpr int kJoinWarps = kJoinThreads / 32;
constexpr int kJoinRows = 128;    // of a tile of 256: two CTAs a cut, all resident at once (32 rows: 28 us for 147 cuts)
// of more than 128 channels half as many rows: a CTA holds as much
__host__ __device__ constexpr int join_rows(int head_dim) { return head_dim > 128 ? kJoinRows / 2 : kJoinRows; }
constexpr int kJoinLook = 4;      // so that all CTAs of the launch are resident at once

struct Pieces {          // of one segment
  const float* first;
  size_t stride;
  int n;
  __host__ __device__ __forceinline__ const float* at(int i) const { return first + (i == 0 ? 0 : 2 * i - 1) * stride; }
};

__host__ __device__ __forceinline__ bool cut_at(const AttnParams& p, int k, Boundary& bd, Pieces& pc) {
  if (k == 0) return false;
  bd = p.boundary[k];
  const Boundary before = p.boundary[k - 1];
  if (bd.seg1 == 0 || (before.seg1 != 0 && before.seg0 == bd.seg0)) return false;   // no cut, or not the segment's first
  pc.stride = partial_floats(p.tile_rows, p.head_dim);
  pc.n = static_cast<int>((bd.seg1 - 1) / bd.quota) - k + 2;                         // up to the worker of the segment's last unit
  pc.first = p.partial + (static_cast<size_t>(k) * 2 - 1) * pc.stride;               // slot 1 of k - 1; then slot 0 of k, ...
  return true;
}

// Row r: its largest maximum over all pieces, its denominator, and pieces i0, i0 + step, ... of its sums (lane: channels
// 4 lane .. + 3, and 128 on).  A lane has the maximum and denominator of a piece; 32 pieces at a time.
__device__ __forceinline__ float join_row(const AttnParams& p, const Pieces& pc, int r, int i0, int step, float& den, float* acc) {
  const int lane = threadIdx.x & 31, D = p.head_dim, R = p.tile_rows;
  float top = -INFINITY;
  for (int i = lane; i < pc.n; i += 32) top = fmaxf(top, pc.at(i)[R * D + r]);
  top = warp_max(top);
  const float base = top == -INFINITY ? 0.f : top;
  den = 0.f;
#pragma unroll
  for (int c = 0; c < 8; ++c) acc[c] = 0.f;
  for (int first = 0; first < pc.n; first += 32) {
    float f = 0.f;
    if (first + lane < pc.n) {
      const float* part = pc.at(first + lane);
      f = ex2(part[R * D + r] - base);
      den = fmaf(f, part[R * D + R + r], den);
    }
    const int count = min(32, pc.n - first);
    for (int half = 0; half < (D > 128 ? 2 : 1); ++half) {
      const int c = half * 128 + lane * 4;
      float4 a = make_float4(acc[0], acc[1], acc[2], acc[3]);
      if (half) a = make_float4(acc[4], acc[5], acc[6], acc[7]);
#pragma unroll 8
      for (int i = i0; i < count; i += step) {
        const float g = __shfl_sync(0xffffffffu, f, i);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c < D) o = *reinterpret_cast<const float4*>(pc.at(first + i) + r * D + c);
        a.x = fmaf(g, o.x, a.x); a.y = fmaf(g, o.y, a.y); a.z = fmaf(g, o.z, a.z); a.w = fmaf(g, o.w, a.w);
      }
      if (half) { acc[4] = a.x; acc[5] = a.y; acc[6] = a.z; acc[7] = a.w; }
      else { acc[0] = a.x; acc[1] = a.y; acc[2] = a.z; acc[3] = a.w; }
    }
  }
  den = warp_sum(den);
  return top;
}

// Pieces of bf16 queries have V scales in their references
template <typename T>
__device__ __forceinline__ float joined_log_sum(float m, float l) {
  if constexpr (sizeof(T) == 2) return log_sum(m, l);
  else return l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

template <typename T>
__global__ void __launch_bounds__(kJoinThreads, 2) join_kernel(AttnParams p, int n_ctas) {
  __shared__ float sums[kJoinWarps][256];
  grid_dependency_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = p.head_dim;
  const bool solo = p.status[1] != 0;
  Boundary bd;
  Pieces pc;
  float den, acc[8];
  auto finish = [&](int r, float top, float d, const float* x) {       // x: what this lane has of the row, as join_row gives it
    const RowAt at = row_at(p, bd.tile, bd.head, r);
    char* out = out_at(p, bd.b, bd.first, at);
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const int ch = (c / 4) * 128 + lane * 4 + c % 4;
      if (ch < D) store_out<T>(out, ch, d == 0.f ? 0.f : x[c] / d);
    }
    if (lane == 0 && p.lse) *lse_at(p, bd.b, bd.first, at) = joined_log_sum<T>(top, d);
  };
  if (solo) {
    const int k = blockIdx.x * kJoinWarps + warp;
    if (k >= n_ctas * kWorkersPerCta || !cut_at(p, k, bd, pc)) return;
    for (int r = 0; r < bd.rows; ++r) {
      const float top = join_row(p, pc, r, 0, 1, den, acc);
      finish(r, top, den, acc);
    }
    return;
  }
  if (p.tile_rows > 16) {
    constexpr int kSlabs = kJoinRows / 32, kTurns = kJoinWarps / kSlabs;   // a warp has 32 of the rows, and every kTurns-th piece
    constexpr int kBatch = 24;                                    // pieces whose factors fit beside the rows' maxima and sums
    float (*tops)[kJoinRows] = reinterpret_cast<float (*)[kJoinRows]>(&sums[0][0]);
    float (*dens)[kJoinRows] = tops + kTurns;
    float (*factor)[kJoinRows] = dens + kTurns;
    static_assert((2 * kTurns + kBatch) * kJoinRows <= kJoinWarps * 256, "fits the sums");
    if (!cut_at(p, blockIdx.x, bd, pc)) return;
    const int R = p.tile_rows, r0 = blockIdx.y * join_rows(D), n_rows = min(join_rows(D), bd.rows - r0);
    if (n_rows <= 0) return;
    const int in_slab = warp % kSlabs * 32 + lane, mine = r0 + in_slab, turn = warp / kSlabs;
    const bool on = in_slab < n_rows;
    float top = -INFINITY;
    if (on)
      for (int i = turn; i < pc.n; i += kTurns) top = fmaxf(top, pc.at(i)[R * D + mine]);
    tops[turn][in_slab] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kTurns; ++w) top = fmaxf(top, tops[w][in_slab]);
    const float base = top == -INFINITY ? 0.f : top;
    den = 0.f;
    constexpr int kEach = 8;                                      // 128 rows x 128 channels or 64 x 256, four at a time
    static_assert(kEach * kJoinThreads * 4 >= join_rows(128) * 128 && kEach * kJoinThreads * 4 >= join_rows(256) * 256, "a CTA's rows fit");
    const int per_row = D / 4, total = n_rows * per_row;
    float4 o[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) o[e] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int first = 0; first < pc.n; first += kBatch) {
      const int count = min(kBatch, pc.n - first);
      for (int i = turn; i < count; i += kTurns) {
        float f = 0.f;
        if (on) {
          const float* part = pc.at(first + i);
          f = ex2(part[R * D + mine] - base);
          den = fmaf(f, part[R * D + R + mine], den);
        }
        factor[i][in_slab] = f;
      }
      __syncthreads();
      // half of a piece's loads on their way at once
#pragma unroll
      for (int half = 0; half < kEach; half += kEach / 2) {
        for (int i = 0; i < count; ++i) {
          const float* part = pc.at(first + i) + static_cast<size_t>(r0) * D;
          float4 x[kEach / 2];
#pragma unroll
          for (int e = 0; e < kEach / 2; ++e) {
            const int idx = threadIdx.x + (half + e) * kJoinThreads;
            x[e] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (idx < total) x[e] = *reinterpret_cast<const float4*>(part + static_cast<size_t>(idx) * 4);
          }
#pragma unroll
          for (int e = 0; e < kEach / 2; ++e) {
            const int idx = threadIdx.x + (half + e) * kJoinThreads;
            if (idx < total) {
              const float f = factor[i][idx / per_row];
              float4& a = o[half + e];
              a.x = fmaf(f, x[e].x, a.x); a.y = fmaf(f, x[e].y, a.y); a.z = fmaf(f, x[e].z, a.z); a.w = fmaf(f, x[e].w, a.w);
            }
          }
        }
      }
      __syncthreads();
    }
    dens[turn][in_slab] = den;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int idx = threadIdx.x + e * kJoinThreads;
      if (idx < total) {
        const int row = idx / per_row, c = (idx - row * per_row) * 4;
        float d = 0.f;
#pragma unroll
        for (int w = 0; w < kTurns; ++w) d += dens[w][row];
        const RowAt at = row_at(p, bd.tile, bd.head, r0 + row);
        char* out = out_at(p, bd.b, bd.first, at);
        const float inv = d == 0.f ? 0.f : 1.f / d;
        if constexpr (sizeof(T) == 2) {
          const __nv_bfloat162 lo = __floats2bfloat162_rn(o[e].x * inv, o[e].y * inv), hi = __floats2bfloat162_rn(o[e].z * inv, o[e].w * inv);
          *reinterpret_cast<uint2*>(out + c * 2) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
        } else {
          *reinterpret_cast<float4*>(out + c * 4) = make_float4(o[e].x * inv, o[e].y * inv, o[e].z * inv, o[e].w * inv);
        }
      }
    }
    if (turn == 0 && on && p.lse) {
      float d = 0.f;
#pragma unroll
      for (int w = 0; w < kTurns; ++w) d += dens[w][in_slab];
      *lse_at(p, bd.b, bd.first, row_at(p, bd.tile, bd.head, mine)) = joined_log_sum<T>(top, d);
    }
    return;
  }
  const int look = blockIdx.x * kJoinLook + (lane & (kJoinLook - 1));
  unsigned found = __ballot_sync(0xffffffffu, lane < kJoinLook && look < n_ctas && cut_at(p, look, bd, pc));
  // 8 rows: two warps a row; 16: one.  At most 16 rows a tile.
  const int parts = kJoinWarps / (p.tile_rows <= 8 ? 8 : 16), r = warp / parts;
  for (; found; found &= found - 1) {
    cut_at(p, blockIdx.x * kJoinLook + __ffs(found) - 1, bd, pc);
    float top = 0.f;
    if (r < bd.rows) {
      top = join_row(p, pc, r, warp - r * parts, parts, den, acc);
#pragma unroll
      for (int c = 0; c < 8; ++c) sums[warp][(c / 4) * 128 + lane * 4 + c % 4] = acc[c];
    }
    __syncthreads();
    if (r < bd.rows && warp == r * parts) {
      for (int w = 1; w < parts; ++w) {
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[c] += sums[warp + w][(c / 4) * 128 + lane * 4 + c % 4];
      }
      finish(r, top, den, acc);
    }
    __syncthreads();
  }
}

}  // namespace kv
}  // namespace vscan
