// What the entry points of the paged 8-bit KV cache share: host-side checks, codes and their scales.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace vscan {
namespace kv {

constexpr int kMaxBatch = 8192;
constexpr int kExpMin = -48, kExpMax = 48;   // exponents of a block's scale: sums of codes times scales stay far inside float32

inline bool block_size_ok(int bs) { return bs == 16 || bs == 32 || bs == 64 || bs == 128 || bs == 256; }

// Strides {sequence, head, row} in elements: row starts on 16-byte boundaries, offsets that fit 64 bits with room
inline bool strides_ok(const int64_t* st, size_t elem, bool padded) {
  for (int i = padded ? 0 : 1; i < 3; ++i)
    if (st[i] < 0 || st[i] > (int64_t{1} << 40) || (st[i] * static_cast<int64_t>(elem)) % 16) return false;
  return true;
}

// Bytes from the first to the last element of rows x heads x dim by strides
inline size_t rows_extent(const int64_t* st, int64_t batch, int64_t heads, int64_t rows, int64_t dim, size_t elem, bool padded) {
  if (rows <= 0 || batch <= 0) return 0;
  const int64_t last = (padded ? st[0] * (batch - 1) : 0) + st[1] * (heads - 1) + st[2] * (rows - 1) + dim;
  return static_cast<size_t>(last) * elem;
}

// The least e in [kExpMin, kExpMax] with amax <= qmax * 2^e, for a finite amax >= 0.  qmax is m * 2^k with a mantissa m
// below 2: comparing the mantissa's bits with those of m decides between two neighbouring exponents.
template <int KV>
__device__ __forceinline__ int scale_exponent(float amax) {
  constexpr uint32_t top = KV == VSCAN_KV_E4M3 ? 0x600000u : 0x7E0000u;   // 448 = 1.75 * 2^8, 127 = 1.984375 * 2^6
  constexpr int k = KV == VSCAN_KV_E4M3 ? 8 : 6;
  const uint32_t u = __float_as_uint(amax);
  const int e = static_cast<int>(u >> 23) - 127 - k + ((u & 0x7FFFFFu) > top ? 1 : 0);
  return min(max(e, kExpMin), kExpMax);   // 0 and subnormals fall below kExpMin
}
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

// Four values, already divided by their scale, to four codes in one word.  Rounded once, to nearest, ties to even;
// beyond the largest code they saturate; a NaN gives the code of 0 (its block's scale says NaN).
template <int KV>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  if constexpr (KV == VSCAN_KV_E4M3) {
    auto clean = [](float v) { return v == v ? v : 0.f; };
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(clean(a), clean(b)), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(clean(c), clean(d)), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
  } else {
    auto code = [](float v) {   // NaN: cvt gives 0
      return static_cast<uint32_t>(__float2int_rn(fminf(fmaxf(v == v ? v : 0.f, -127.f), 127.f))) & 0xFFu;
    };
    return code(a) | (code(b) << 8) | (code(c) << 16) | (code(d) << 24);
  }
}

// Four codes to float32, exactly
template <int KV>
__device__ __forceinline__ void decode4(uint32_t w, float* out) {
  if constexpr (KV == VSCAN_KV_E4M3) {
    const __half2_raw lo = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w & 0xFFFFu), __NV_E4M3);
    const __half2_raw hi = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w >> 16), __NV_E4M3);
    const float2 l = __half22float2(__half2(lo)), h = __half22float2(__half2(hi));
    out[0] = l.x; out[1] = l.y; out[2] = h.x; out[3] = h.y;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = static_cast<float>(static_cast<int8_t>(w >> (8 * i)));
  }
}

// New rows of sequence b, held inside the `rows` of the buffer: first packed row (0: padded), count, and the position of the
// first in the sequence (below zero where kv_len is less than the rows)
__host__ __device__ __forceinline__ void row_span(const int32_t* row_offset, const int32_t* kv_len, int b, int rows, bool padded,
                                         int& first, int& n, long long& start) {
  const long long lo = row_offset[b], given = max(row_offset[b + 1] - lo, 0ll);
  start = kv_len[b] - given;
  first = padded ? 0 : static_cast<int>(lo);
  const long long room = padded ? rows : lo < 0 ? 0 : max(rows - lo, 0ll);
  n = static_cast<int>(min(given, room));
}

}  // namespace kv
}  // namespace vscan
