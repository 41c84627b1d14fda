// vscan_kv_write: new rows of K and V into the paged 8-bit cache, one power-of-two scale per block of tokens and head.
//
// Every row is read once and written at a half (bf16) or a quarter (f32) of its bytes: DRAM bounds long calls, launch and
// load latency the decode steps.  A block's scale needs the maximum over all its new tokens before the first code can be
// written, so one group of threads owns a (block, head) of K or V.  Which (sequence, block) an item number stands for is
// found by a search on row_offset with an item numbering that needs no prefix sum of block counts:
//   append form   items = rows; an item acts when its row is the first new one of its block (few rows a sequence)
//   block form    sequence b's items start at floor(row_offset[b] / block_size) + 2 b: n rows touch at most
//                 floor(n / block_size) + 2 blocks, which is never more than the distance to the next sequence's start
#include "kv_common.cuh"

namespace vscan {
namespace kv {

struct WriteParams {
  const char* src[2];               // k, v
  long long seq[2], head[2], row[2];   // strides in bytes
  uint8_t* cache[2];
  float* scale[2];
  const int32_t* kv_len;
  const int32_t* row_offset;
  const int32_t* block_table;
  int batch, kv_heads, head_dim, block_size, shift, num_blocks, max_blocks, rows, padded;
};

// A sequence's new tokens: rows n from packed row `first`, positions start ..; n = 0 where nothing is to be written
struct Span { int first, n, start; };

__device__ __forceinline__ Span span_of(const WriteParams& p, int b) {
  Span s;
  long long start;
  row_span(p.row_offset, p.kv_len, b, p.rows, p.padded, s.first, s.n, start);
  s.start = static_cast<int>(start);
  if (start < 0) s.n = 0;
  return s;
}

// Largest b in [0, batch) whose items start at or before `item`; a warp looks at 32 candidates at a time.  start(b) must
// not fall with b.
template <typename Start>
__device__ __forceinline__ int find_sequence(int batch, long long item, Start start) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = batch;                     // the answer lies in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) >> 5, b = lo + lane * step;
    const bool le = lane * step < n && start(b) <= item;
    const unsigned hits = __ballot_sync(0xffffffffu, le) | 1u;
    const int k = 31 - __clz(hits);
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
}

// Elements c .. c + 15 of a source row as floats
template <typename T>
struct Chunk {
  static constexpr int kVecs = 16 / Vec16<T>::kElems;
  uint4 v[kVecs];
  __device__ __forceinline__ void load(const char* p) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) v[i] = ld_nc_16(p + 16 * i);
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) v[i] = make_uint4(0, 0, 0, 0);
  }
  // Largest magnitude as an unsigned pattern: infinities and NaN come out above every finite value.  bf16 two at a time, as
  // 16-bit patterns
  __device__ __forceinline__ uint32_t peak() const {
    if constexpr (sizeof(T) == 2) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        m = __vmaxu2(__vmaxu2(m, v[i].x & 0x7fff7fffu), v[i].y & 0x7fff7fffu);
        m = __vmaxu2(__vmaxu2(m, v[i].z & 0x7fff7fffu), v[i].w & 0x7fff7fffu);
      }
      return max(m << 16, m & 0xffff0000u);
    } else {
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(fabsf(__uint_as_float(w[j]))));
      }
      return __float_as_uint(m) & 0x7fffffffu;
    }
  }
  // NaN to 0, the rest held between -limit and limit, which T has; all to +0 where that is 0
  __device__ __forceinline__ void clean(float limit) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      float f[Vec16<T>::kElems];
      Vec16<T>::unpack(v[i], f);
#pragma unroll
      for (int j = 0; j < Vec16<T>::kElems; ++j) f[j] = f[j] == f[j] && limit > 0.f ? fminf(fmaxf(f[j], -limit), limit) : 0.f;
      v[i] = Vec16<T>::pack(f);
    }
  }
  // Codes of elements that are all finite and, times inv, not beyond the largest code
  template <int KV>
  __device__ __forceinline__ uint4 encode(float inv) const {
    float f[16];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) Vec16<T>::unpack(v[i], f + i * Vec16<T>::kElems);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (KV == VSCAN_KV_E4M3) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * i] * inv, f[4 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * i + 2] * inv, f[4 * i + 3] * inv), __NV_SATFINITE, __NV_E4M3);
        w[i] = lo | (hi << 16);
      } else {          // 1.5 x 2^23 + x: rounded to the nearest integer, ties to even, whose last byte is the code
        uint32_t c[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j] = __float_as_uint(fmaf(f[4 * i + j], inv, 12582912.f));
        w[i] = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// 16 old codes times `ratio`, coded again
template <int KV>
__device__ __forceinline__ uint4 recode(const uint4& old, float ratio) {
  const uint32_t w[4] = {old.x, old.y, old.z, old.w};
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float f[4];
    decode4<KV>(w[i], f);
    r[i] = encode4<KV>(f[0] * ratio, f[1] * ratio, f[2] * ratio, f[3] * ratio);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}

// The scale of a (block, head) from the peak of its new elements and, where it holds older tokens, its old scale
struct Scale {
  float s, inv, ratio;    // inv: what the new elements are multiplied by; ratio: what the old codes are multiplied by (1: they stay)
  bool odd;               // elements have to be cleaned first: the scale is NaN (all codes are 0 then) or ends below what they need
  float limit;
};
template <int KV>
__device__ __forceinline__ Scale new_scale(uint32_t peak, bool holds, float old) {
  Scale r;
  r.s = peak < 0x7f800000u ? exp2_int(scale_exponent<KV>(__uint_as_float(peak))) : __uint_as_float(0x7fc00000u);
  if (holds) r.s = (r.s != r.s || old != old) ? __uint_as_float(0x7fc00000u) : fmaxf(r.s, old);
  r.ratio = holds && r.s != old ? old / r.s : 1.f;
  const bool nan = r.s != r.s;
  r.limit = nan ? 0.f : (KV == VSCAN_KV_E4M3 ? 448.f : 127.f) * r.s;
  r.odd = nan || !(__uint_as_float(peak) <= r.limit);
  r.inv = nan ? 0.f : 1.f / r.s;
  return r;
}

// ---------------------------------------------------------------------------------------------- append form
// A group of G lanes (16 elements each) owns a (row, head) of K or V; groups of a warp take neighbouring heads.
constexpr int kAppendThreads = 128;

template <typename T, int KV, int G>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(WriteParams p) {
  grid_dependency_wait();
  const int row_item = blockIdx.x, which = blockIdx.z;
  const int b = find_sequence(p.batch, row_item, [&](int i) { return static_cast<long long>(p.padded ? i * static_cast<long long>(p.rows) : p.row_offset[i]); });
  const Span sp = span_of(p, b);
  const int i = row_item - (p.padded ? b * p.rows : sp.first);
  if (i < 0 || i >= sp.n) return;
  const int pos = sp.start + i, off = pos & (p.block_size - 1), col = pos >> p.shift;
  if (i > 0 && off != 0) return;                           // not the first new row of its block
  if (col >= p.max_blocks) return;
  const int block = p.block_table[static_cast<size_t>(b) * p.max_blocks + col];
  if (block < 0 || block >= p.num_blocks) return;
  const int n = min(sp.n - i, p.block_size - off);         // new rows of this block
  const int lane = threadIdx.x & 31, lig = lane & (G - 1);
  const int h = (blockIdx.y * (kAppendThreads / G)) + threadIdx.x / G;
  const bool on = h < p.kv_heads && lig * 16 < p.head_dim;
  const char* src = p.src[which] + (p.padded ? b * p.seq[which] : 0) + static_cast<long long>(sp.first + i) * p.row[which] +
                    static_cast<long long>(h) * p.head[which] + lig * 16 * static_cast<int>(sizeof(T));
  const size_t cell = static_cast<size_t>(block) * p.kv_heads + (on ? h : 0);
  const float old = off > 0 ? p.scale[which][cell] : 0.f;
  Chunk<T> first;
  first.zero();
  if (on) first.load(src);
  uint32_t peak = first.peak();
  for (int r = 1; r < n; ++r) {
    if (on) {
      Chunk<T> c;
      c.load(src + r * p.row[which]);
      peak = max(peak, c.peak());
    }
  }
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) peak = max(peak, __shfl_xor_sync(0xffffffffu, peak, o));
  if (!on) return;
  const Scale sc = new_scale<KV>(peak, off > 0, old);
  uint8_t* dst = p.cache[which] + cell * p.block_size * p.head_dim + lig * 16;
  if (sc.ratio != 1.f)
    for (int r = 0; r < off; ++r) {
      uint4* at = reinterpret_cast<uint4*>(dst + r * p.head_dim);
      *at = recode<KV>(*at, sc.ratio);
    }
  if (sc.odd) first.clean(sc.limit);
  st_16(dst + off * p.head_dim, first.template encode<KV>(sc.inv));
  for (int r = 1; r < n; ++r) {
    Chunk<T> c;
    c.load(src + r * p.row[which]);
    if (sc.odd) c.clean(sc.limit);
    st_16(dst + (off + r) * p.head_dim, c.template encode<KV>(sc.inv));
  }
  if (lig == 0) p.scale[which][cell] = sc.s;
}

// ---------------------------------------------------------------------------------------------- block form
// A CTA owns a block of tokens, a group of W warps at a time one (head, K or V) of it: chunks of 16 elements, kHeld of them a
// lane in registers between the maximum and the codes, the rest (large blocks) read a second time from L2.  What the block's
// place in sequence and table takes to find (a chain of four loads) is found once for all its heads, and where the lane's
// chunks lie once for all units.  Small CTAs, so that the chain
// of one runs beside the copies of others.  The maximum and the codes take few instructions an element (packed maxima; what
// is not finite or saturates is cleaned on a path of its own): with plain ones the ALU was busy 75 % of the time.
// 32 x 259 rows x 32 heads of 128 in bf16, 204 MB: 38 us, 5.3 TB/s (123 us with a CTA a unit, 42 us with plain instructions);
// 4 sequences of 12,000 to 16,500 rows x 4 heads of 128 in float32, 313 MB: 60 us, 5.2 TB/s (68 us).
constexpr int kHeld = 4;
__host__ __device__ constexpr int block_threads(int w) { return w == 8 ? 256 : 128; }

template <typename T, int KV, int W>
__global__ void __launch_bounds__(block_threads(W), (sizeof(T) == 2 ? 768 : 512) / block_threads(W)) block_kernel(WriteParams p, int per_cta) {
  constexpr int kThreads = block_threads(W), kGroups = kThreads / 32 / W;
  __shared__ uint32_t warp_peak[kThreads / 32];
  grid_dependency_wait();
  const int item = blockIdx.x, per = p.rows / p.block_size + 2;   // padded: items of a sequence
  const int b = p.padded ? item / per : find_sequence(p.batch, item, [&](int i) {
    return static_cast<long long>(min(max(p.row_offset[i], 0), p.rows) >> p.shift) + 2 * i; });
  const Span sp = span_of(p, b);
  if (sp.n == 0) return;
  const int j = item - (p.padded ? b * per : (sp.first >> p.shift) + 2 * b);
  const int col = (sp.start >> p.shift) + j;
  const long long col0 = static_cast<long long>(col) << p.shift;   // first position of the block
  const long long end = static_cast<long long>(sp.start) + sp.n;
  if (j < 0 || col0 >= end || col >= p.max_blocks) return;
  const int block = p.block_table[static_cast<size_t>(b) * p.max_blocks + col];
  if (block < 0 || block >= p.num_blocks) return;
  const int off = j == 0 ? sp.start & (p.block_size - 1) : 0;
  const int n = static_cast<int>(min(end - col0, static_cast<long long>(p.block_size))) - off;
  const int i0 = static_cast<int>(col0 + off - sp.start);  // first new row of this block
  const int cpr = p.head_dim / 16, total = n * cpr;        // chunks
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, group = warp / W, in_group = threadIdx.x - group * W * 32;
  const long long row0 = static_cast<long long>(sp.first) + i0;
  int held_row[kHeld], held_col[kHeld];                    // of this lane's chunks; a row below 0: none
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int c = in_group + k * 32 * W;
    held_row[k] = c < total ? c / cpr : -1;
    held_col[k] = c < total ? (c - held_row[k] * cpr) * 16 * static_cast<int>(sizeof(T)) : 0;
  }
  const int units = 2 * p.kv_heads, u0 = blockIdx.y * per_cta, u1 = min(u0 + per_cta, units);
  for (int u = u0 + group; u < u1; u += kGroups) {
    const int h = u >> 1, which = u & 1;
    const char* src = p.src[which] + (p.padded ? b * p.seq[which] : 0) + row0 * p.row[which] + static_cast<long long>(h) * p.head[which];
    const size_t cell = static_cast<size_t>(block) * p.kv_heads + h;
    Chunk<T> held[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
      held[k].zero();
      if (held_row[k] >= 0) held[k].load(src + held_row[k] * p.row[which] + held_col[k]);
    }
    const float old = off > 0 ? p.scale[which][cell] : 0.f;
    uint32_t peak = 0;
#pragma unroll
    for (int k = 0; k < kHeld; ++k) peak = max(peak, held[k].peak());
    for (int c = in_group + kHeld * 32 * W; c < total; c += 32 * W) {
      const int r = c / cpr;
      Chunk<T> x;
      x.load(src + r * p.row[which] + (c - r * cpr) * 16 * static_cast<int>(sizeof(T)));
      peak = max(peak, x.peak());
    }
    peak = __reduce_max_sync(0xffffffffu, peak);
    if constexpr (W > 1) {                                 // the groups of a CTA go their own ways: a barrier each
      if (lane == 0) warp_peak[warp] = peak;
      asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(W * 32) : "memory");
#pragma unroll
      for (int w = 0; w < W; ++w) peak = max(peak, warp_peak[group * W + w]);
    }
    const Scale sc = new_scale<KV>(peak, off > 0, old);
    uint8_t* base = p.cache[which] + cell * p.block_size * p.head_dim;
    uint8_t* dst = base + static_cast<size_t>(off) * p.head_dim;
    if (sc.ratio != 1.f)
      for (int c = in_group; c < off * cpr; c += 32 * W) {
        uint4* at = reinterpret_cast<uint4*>(base) + c;
        *at = recode<KV>(*at, sc.ratio);
      }
    if (sc.odd) {
#pragma unroll
      for (int k = 0; k < kHeld; ++k) held[k].clean(sc.limit);
    }
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
      if (held_row[k] >= 0) st_16(dst + static_cast<size_t>(in_group + k * 32 * W) * 16, held[k].template encode<KV>(sc.inv));
    for (int c = in_group + kHeld * 32 * W; c < total; c += 32 * W) {
      const int r = c / cpr;
      Chunk<T> x;
      x.load(src + r * p.row[which] + (c - r * cpr) * 16 * static_cast<int>(sizeof(T)));
      if (sc.odd) x.clean(sc.limit);
      st_16(dst + static_cast<size_t>(c) * 16, x.template encode<KV>(sc.inv));
    }
    if constexpr (W > 1) asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(W * 32) : "memory");   // old scale and maxima have been read
    if (in_group == 0) p.scale[which][cell] = sc.s;
  }
}

static vscan_status validate_write(const vscan_kv_write_desc* d) {
  if (!d) return VSCAN_ERR_INVALID_ARG;
  if (d->dtype != VSCAN_F32 && d->dtype != VSCAN_BF16) return VSCAN_ERR_INVALID_ARG;
  if (d->kv_dtype != VSCAN_KV_E4M3 && d->kv_dtype != VSCAN_KV_I8) return VSCAN_ERR_INVALID_ARG;
  if (d->batch < 0 || d->kv_heads <= 0 || d->head_dim <= 0 || d->head_dim % 16 || d->num_blocks < 0 || d->max_blocks < 0 || d->rows < 0 ||
      !block_size_ok(d->block_size))
    return VSCAN_ERR_INVALID_ARG;
  if (d->batch == 0 || d->rows == 0 || d->num_blocks == 0 || d->max_blocks == 0) return VSCAN_OK;
  if (!d->k || !d->v || !d->kv_len || !d->row_offset || !d->block_table || !d->k_cache || !d->v_cache || !d->k_scale || !d->v_scale)
    return VSCAN_ERR_INVALID_ARG;
  if (d->head_dim > 256 || d->batch > kMaxBatch || d->kv_heads > 65535 || static_cast<int64_t>(d->max_blocks) * d->block_size > 0x7fffffff ||
      (d->padded && static_cast<int64_t>(d->batch) * d->rows > 0x7fffffff))
    return VSCAN_ERR_UNSUPPORTED;
  const size_t e = dtype_bytes(d->dtype), B = d->batch, H = d->kv_heads;
  if (!strides_ok(d->k_stride, e, d->padded) || !strides_ok(d->v_stride, e, d->padded)) return VSCAN_ERR_INVALID_ARG;
  struct Rng { const void* p; size_t n; };
  const size_t pool = static_cast<size_t>(d->num_blocks) * H;
  const Rng all[] = {{d->k, rows_extent(d->k_stride, B, H, d->rows, d->head_dim, e, d->padded)},
                     {d->v, rows_extent(d->v_stride, B, H, d->rows, d->head_dim, e, d->padded)},
                     {d->kv_len, B * 4}, {d->row_offset, (B + 1) * 4}, {d->block_table, B * d->max_blocks * 4},
                     {d->k_cache, pool * d->block_size * d->head_dim}, {d->v_cache, pool * d->block_size * d->head_dim},
                     {d->k_scale, pool * 4}, {d->v_scale, pool * 4}};
  constexpr int kInputs = 5;
  for (const Rng& r : all)
    if (!aligned16(r.p)) return VSCAN_ERR_INVALID_ARG;
  for (int o = kInputs; o < 9; ++o)
    for (int i = 0; i < o; ++i)
      if (overlaps(all[o].p, all[o].n, all[i].p, all[i].n)) return VSCAN_ERR_INVALID_ARG;
  return VSCAN_OK;
}

template <typename T, int KV>
static vscan_status launch_write(const WriteParams& p, cudaStream_t stream) {
  const long long rows = p.padded ? static_cast<long long>(p.batch) * p.rows : p.rows;
  const long long items = p.padded ? static_cast<long long>(p.batch) * (p.rows / p.block_size + 2) : p.rows / p.block_size + 2ll * p.batch;
  if (rows <= items) {
    const int lanes = p.head_dim / 16;
    const unsigned per = static_cast<unsigned>(kAppendThreads / (lanes <= 4 ? 4 : lanes <= 8 ? 8 : 16));
    const dim3 grid(static_cast<unsigned>(rows), (p.kv_heads + per - 1) / per, 2);
    prof_before("kv_append", stream);
    VSCAN_CUDA_TRY(lanes <= 4 ? launch_dependent(append_kernel<T, KV, 4>, grid, dim3(kAppendThreads), 0, stream, p)
                   : lanes <= 8 ? launch_dependent(append_kernel<T, KV, 8>, grid, dim3(kAppendThreads), 0, stream, p)
                                : launch_dependent(append_kernel<T, KV, 16>, grid, dim3(kAppendThreads), 0, stream, p));
  } else {
    // as many warps to a unit as keep its chunks in registers
    const int chunks = p.block_size * p.head_dim / 16, w = chunks <= 128 ? 1 : chunks <= 256 ? 2 : chunks <= 512 ? 4 : 8;
    // a CTA takes its warps' worth of units several times over while the grid still covers the SMs sixteen times
    const long long units = 2ll * p.kv_heads, groups = block_threads(w) / 32 / w;
    long long turns = items * units / (groups * 148 * 16);
    turns = turns < 1 ? 1 : turns > 16 ? 16 : turns;
    const long long split = (units + groups * turns - 1) / (groups * turns);
    const int per_cta = static_cast<int>(((units + split - 1) / split + groups - 1) / groups * groups);
    const dim3 grid(static_cast<unsigned>(items), static_cast<unsigned>((units + per_cta - 1) / per_cta));
    prof_before("kv_write", stream);
    VSCAN_CUDA_TRY(w == 1 ? launch_dependent(block_kernel<T, KV, 1>, grid, dim3(block_threads(w)), 0, stream, p, per_cta)
                   : w == 2 ? launch_dependent(block_kernel<T, KV, 2>, grid, dim3(block_threads(w)), 0, stream, p, per_cta)
                   : w == 4 ? launch_dependent(block_kernel<T, KV, 4>, grid, dim3(block_threads(w)), 0, stream, p, per_cta)
                            : launch_dependent(block_kernel<T, KV, 8>, grid, dim3(block_threads(w)), 0, stream, p, per_cta));
  }
  prof_after(stream);
  VSCAN_AFTER_LAUNCH();
  return VSCAN_OK;
}

}  // namespace kv
}  // namespace vscan

using namespace vscan;

extern "C" vscan_status vscan_kv_write(const vscan_kv_write_desc* d, void* stream_) {
  const vscan_status st = kv::validate_write(d);
  if (st != VSCAN_OK) return st;
  if (d->batch == 0 || d->rows == 0 || d->num_blocks == 0 || d->max_blocks == 0) return VSCAN_OK;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  const long long e = static_cast<long long>(dtype_bytes(d->dtype));
  kv::WriteParams p = {};
  p.src[0] = static_cast<const char*>(d->k); p.src[1] = static_cast<const char*>(d->v);
  const int64_t* strides[2] = {d->k_stride, d->v_stride};
  for (int i = 0; i < 2; ++i) { p.seq[i] = strides[i][0] * e; p.head[i] = strides[i][1] * e; p.row[i] = strides[i][2] * e; }
  p.cache[0] = static_cast<uint8_t*>(d->k_cache); p.cache[1] = static_cast<uint8_t*>(d->v_cache);
  p.scale[0] = d->k_scale; p.scale[1] = d->v_scale;
  p.kv_len = d->kv_len; p.row_offset = d->row_offset; p.block_table = d->block_table;
  p.batch = d->batch; p.kv_heads = d->kv_heads; p.head_dim = d->head_dim; p.block_size = d->block_size;
  p.num_blocks = d->num_blocks; p.max_blocks = d->max_blocks; p.rows = d->rows; p.padded = d->padded ? 1 : 0;
  while ((1 << p.shift) < p.block_size) ++p.shift;
  if (d->dtype == VSCAN_F32)
    return d->kv_dtype == VSCAN_KV_E4M3 ? kv::launch_write<float, VSCAN_KV_E4M3>(p, stream) : kv::launch_write<float, VSCAN_KV_I8>(p, stream);
  return d->kv_dtype == VSCAN_KV_E4M3 ? kv::launch_write<__nv_bfloat16, VSCAN_KV_E4M3>(p, stream)
                                      : kv::launch_write<__nv_bfloat16, VSCAN_KV_I8>(p, stream);
}
