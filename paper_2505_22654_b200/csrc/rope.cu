// vscan_rope: rotary positions with several axes on queries and keys.
//
// A pure copy with arithmetic: every element is read and written once, so DRAM bounds it (a few tokens: launch latency).
// The angle of a pair depends on the token alone, not on the head, so a CTA takes all heads of a few tokens, computes each
// (cos, sin) once into shared memory and turns every head with it.  The angle's fraction of a turn is taken in 64 bits: at
// position 1e5 a 32-bit product is off by 4e-3 rad.  Measured: 32,768 tokens x 32 heads of 80 in float32, 671 MB: 125 us, 5.4 TB/s;
// 8,704 tokens x 32 heads of 128 in bf16, 143 MB: 31 us, 4.7 TB/s; 32 tokens: 3.2 us.
#include "common.cuh"

namespace vscan {
namespace rope {

constexpr int kThreads = 256;
constexpr int kMaxTokens = 8;   // tokens of a CTA

struct Side {
  const char* in;
  char* out;
  long long in_seq, in_head, in_tok, out_seq, out_head, out_tok;   // bytes
  int heads;
};

// Division of n < 2^31 by a number that the host knows: a high product, an add and a shift (Granlund and Montgomery, "Division by
// invariant integers using multiplication", 1994)
struct Divisor {
  unsigned d, m, l;
  void set(unsigned by) {
    d = by;
    l = 0;
    while ((1ull << l) < by) ++l;
    m = static_cast<unsigned>(((1ull << 32) * ((1ull << l) - by)) / by + 1);
  }
  __device__ __forceinline__ int div(int n) const { return static_cast<int>((__umulhi(m, static_cast<unsigned>(n)) + static_cast<unsigned>(n)) >> l); }
};

struct Params {
  Side side[2];   // queries, keys
  const int32_t* pos;
  const float* inv_freq;
  const int32_t* axis;
  int tokens, seq_len, planes, half, pair_units, units, heads, tokens_per_cta;
  Divisor by_half, by_seq, by_units, by_token;
  float sign;
};

// N elements of T as one load or store of N * sizeof(T) bytes
template <int BYTES> struct Word;
template <> struct Word<2> { using type = unsigned short; };
template <> struct Word<4> { using type = unsigned int; };
template <> struct Word<8> { using type = uint2; };
template <> struct Word<16> { using type = uint4; };

template <typename T, int V>
struct Piece {
  typename Word<V * static_cast<int>(sizeof(T))>::type w;
  __device__ __forceinline__ void load(const char* p) { w = *reinterpret_cast<const decltype(w)*>(p); }
  __device__ __forceinline__ void store(char* p) const { *reinterpret_cast<decltype(w)*>(p) = w; }
  __device__ __forceinline__ float get(int i) const { return to_float<T>(reinterpret_cast<const T*>(&w)[i]); }
  __device__ __forceinline__ void set(int i, float v) {
    if constexpr (sizeof(T) == 4) reinterpret_cast<float*>(&w)[i] = v;
    else reinterpret_cast<__nv_bfloat16*>(&w)[i] = __float2bfloat16_rn(v);
  }
};

// V: elements of a piece, the widest that divides the pair layout.  A unit is two pieces: the two halves of V pairs
// (HALVES), or 2 V consecutive channels = V pairs (ADJACENT); units behind pair_units copy channels that are not turned.
// A thread's first kAhead units are on their way while the angles are made (4 x 2176 tokens x 32 heads of 128 in bf16: 30 us
// without that and with plain divisions).
constexpr int kAhead = 4;

template <typename T, int V, bool ADJACENT>
__global__ void __launch_bounds__(kThreads) rope_kernel(Params p) {
  extern __shared__ float2 cs[];   // [tokens_per_cta][half]
  grid_dependency_wait();
  constexpr int kBytes = V * static_cast<int>(sizeof(T));
  const int tok0 = blockIdx.x * p.tokens_per_cta, n_tok = min(p.tokens_per_cta, p.tokens - tok0);
  const int total = n_tok * p.heads * p.units;
  struct Unit { const char* in; char* out; int t, u, first, second; };
  auto unit_at = [&](int i) {
    Unit w;
    w.t = p.by_token.div(i);
    const int r = i - w.t * static_cast<int>(p.by_token.d);
    int h = p.by_units.div(r);
    w.u = r - h * p.units;
    const int which = h >= p.side[0].heads;
    const Side& sd = p.side[which];
    h -= which ? p.side[0].heads : 0;
    const int b = p.by_seq.div(tok0 + w.t), s = tok0 + w.t - b * p.seq_len;
    w.in = sd.in + b * sd.in_seq + h * sd.in_head + s * sd.in_tok;
    w.out = sd.out + b * sd.out_seq + h * sd.out_head + s * sd.out_tok;
    if (w.u >= p.pair_units) {
      w.first = (2 * p.half * static_cast<int>(sizeof(T))) + (w.u - p.pair_units) * 2 * kBytes;
      w.second = w.first + kBytes;
    } else {
      w.first = ADJACENT ? 2 * w.u * kBytes : w.u * kBytes;
      w.second = ADJACENT ? w.first + kBytes : w.first + p.half * static_cast<int>(sizeof(T));
    }
    return w;
  };
  auto finish = [&](const Unit& w, Piece<T, V> x, Piece<T, V> y) {
    if (w.u < p.pair_units) {
      const float2* a = cs + w.t * p.half + w.u * V;
      if constexpr (ADJACENT) {
        if constexpr (V == 1) {
          const float e = x.get(0), o = y.get(0);
          x.set(0, e * a[0].x - o * a[0].y);
          y.set(0, o * a[0].x + e * a[0].y);
        } else {
#pragma unroll
          for (int j = 0; j < V; j += 2) {
            const float2 a0 = a[j / 2], a1 = a[V / 2 + j / 2];
            const float e0 = x.get(j), o0 = x.get(j + 1), e1 = y.get(j), o1 = y.get(j + 1);
            x.set(j, e0 * a0.x - o0 * a0.y);
            x.set(j + 1, o0 * a0.x + e0 * a0.y);
            y.set(j, e1 * a1.x - o1 * a1.y);
            y.set(j + 1, o1 * a1.x + e1 * a1.y);
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float e = x.get(j), o = y.get(j);
          x.set(j, e * a[j].x - o * a[j].y);
          y.set(j, o * a[j].x + e * a[j].y);
        }
      }
    }
    x.store(w.out + w.first);
    y.store(w.out + w.second);
  };

  Piece<T, V> x[kAhead], y[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    const int i = threadIdx.x + k * kThreads;
    if (i < total) {
      const Unit w = unit_at(i);
      x[k].load(w.in + w.first);
      y[k].load(w.in + w.second);
    }
  }
  for (int i = threadIdx.x; i < n_tok * p.half; i += kThreads) {
    const int t = p.by_half.div(i), pair = i - t * p.half;
    const int ax = min(max(p.axis[pair], 0), p.planes - 1);
    const int pos = p.pos[static_cast<size_t>(ax) * p.tokens + tok0 + t];
    const double turns = static_cast<double>(pos) * static_cast<double>(p.inv_freq[pair]) * 0.15915494309189533577;
    float s, c;
    sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &s, &c);
    cs[i] = make_float2(c, p.sign * s);
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    const int i = threadIdx.x + k * kThreads;
    if (i < total) finish(unit_at(i), x[k], y[k]);
  }
#pragma unroll 2
  for (int i = threadIdx.x + kAhead * kThreads; i < total; i += kThreads) {
    const Unit w = unit_at(i);
    Piece<T, V> a, b;
    a.load(w.in + w.first);
    b.load(w.in + w.second);
    finish(w, a, b);
  }
}

struct Extent { const char* lo; size_t n; };

// Elements from the first to the last of a tensor given by strides, as offsets from its start
struct Span { int64_t lo, hi; };
static Span span(const int64_t* stride, int64_t batch, int64_t heads, int64_t tokens, int64_t dim) {
  Span r = {0, dim};
  const int64_t n[3] = {batch, heads, tokens};
  for (int i = 0; i < 3; ++i) (stride[i] < 0 ? r.lo : r.hi) += stride[i] * (n[i] - 1);
  return r;
}
static Extent extent(const void* p, const int64_t* stride, int64_t batch, int64_t heads, int64_t tokens, int64_t dim, size_t e) {
  const Span r = span(stride, batch, heads, tokens, dim);
  return {static_cast<const char*>(p) + r.lo * static_cast<int64_t>(e), static_cast<size_t>(r.hi - r.lo) * e};
}

struct Rows { const void* p; const int64_t* stride; int64_t heads; };

// Whether no element of a lies on one of b.  Extents that do not meet are apart; of those that do, the ways in which queries and
// keys are usually views of one buffer are told apart, and anything else counts as not apart:
//   with the same steps from sequence to sequence (token to token), each has its own stretch of every token (of every sequence);
//   with the same steps in all three, the distance between the two is a fourth step of one tensor
static bool apart(const Rows& a, const Rows& b, int64_t batch, int64_t tokens, int64_t dim, size_t e) {
  const Extent ea = extent(a.p, a.stride, batch, a.heads, tokens, dim, e), eb = extent(b.p, b.stride, batch, b.heads, tokens, dim, e);
  if (!overlaps(ea.lo, ea.n, eb.lo, eb.n)) return true;
  const int64_t delta = (reinterpret_cast<intptr_t>(b.p) - reinterpret_cast<intptr_t>(a.p)) / static_cast<int64_t>(e);
  if (batch > 1 && a.stride[0] != b.stride[0]) return false;
  const int64_t counts[2] = {batch, tokens}, steps[2] = {a.stride[0], a.stride[2]};
  for (int common = 1; common <= 2; ++common) {            // the sequences are common steps, then the tokens as well
    if (common == 2 && tokens > 1 && a.stride[2] != b.stride[2]) return false;
    Span own = span(a.stride, 1, a.heads, common == 2 ? 1 : tokens, dim), other = span(b.stride, 1, b.heads, common == 2 ? 1 : tokens, dim);
    other.lo += delta;
    other.hi += delta;
    const int64_t both = (own.hi > other.hi ? own.hi : other.hi) - (own.lo < other.lo ? own.lo : other.lo);
    if ((own.hi <= other.lo || other.hi <= own.lo) && strides_apart(steps, counts, common, both)) return true;
  }
  if (a.heads > 1 && b.heads > 1 && a.stride[1] != b.stride[1]) return false;
  const int64_t all[4] = {a.stride[0], a.heads > 1 ? a.stride[1] : b.stride[1], a.stride[2], delta};
  const int64_t sizes[4] = {batch, a.heads > b.heads ? a.heads : b.heads, tokens, 2};
  return strides_apart(all, sizes, 4, dim);
}

static vscan_status validate(const vscan_rope_desc* d) {
  if (!d || (!d->q && !d->k) || (d->q == nullptr) != (d->q_out == nullptr) || (d->k == nullptr) != (d->k_out == nullptr))
    return VSCAN_ERR_INVALID_ARG;
  if (!d->pos_ids || !d->inv_freq || !d->axis) return VSCAN_ERR_INVALID_ARG;
  if (d->dtype != VSCAN_F32 && d->dtype != VSCAN_BF16) return VSCAN_ERR_INVALID_ARG;
  if (d->pairing != VSCAN_ROPE_HALVES && d->pairing != VSCAN_ROPE_ADJACENT) return VSCAN_ERR_INVALID_ARG;
  if (d->batch < 0 || d->seq_len < 0 || (d->q && d->q_heads <= 0) || (d->k && d->k_heads <= 0)) return VSCAN_ERR_INVALID_ARG;
  if (d->head_dim <= 0 || d->head_dim % 8 || d->rot_dim < 2 || d->rot_dim % 2 || d->rot_dim > d->head_dim || d->pos_planes <= 0)
    return VSCAN_ERR_INVALID_ARG;
  if (d->head_dim > 512 || d->pos_planes > 16 || static_cast<int64_t>(d->batch) * d->seq_len > 0x7fffffff ||
      static_cast<int64_t>(d->q ? d->q_heads : 0) + (d->k ? d->k_heads : 0) > 65536)
    return VSCAN_ERR_UNSUPPORTED;
  const void* ptrs[] = {d->q, d->q_out, d->k, d->k_out, d->pos_ids, d->inv_freq, d->axis};
  for (const void* ptr : ptrs)
    if (ptr && !aligned16(ptr)) return VSCAN_ERR_INVALID_ARG;
  if (d->batch == 0 || d->seq_len == 0) return VSCAN_OK;
  const size_t e = dtype_bytes(d->dtype);
  const int64_t per16 = static_cast<int64_t>(16 / e);
  const int64_t* strides[] = {d->q_stride, d->q_out_stride, d->k_stride, d->k_out_stride};
  for (int i = 0; i < 4; ++i) {
    if (!(i < 2 ? d->q : d->k)) continue;
    for (int j = 0; j < 3; ++j)
      if (strides[i][j] % per16 || strides[i][j] > (int64_t{1} << 40) || strides[i][j] < -(int64_t{1} << 40)) return VSCAN_ERR_INVALID_ARG;
  }
  // outputs: apart from every input, but for the in-place form, and from each other; no two elements of one in one place
  struct Io { const void *in, *out; const int64_t *si, *so; int heads; };
  const Io io[2] = {{d->q, d->q_out, d->q_stride, d->q_out_stride, d->q_heads}, {d->k, d->k_out, d->k_stride, d->k_out_stride, d->k_heads}};
  Extent outs[2] = {};
  for (int i = 0; i < 2; ++i) {
    if (!io[i].in) continue;
    outs[i] = extent(io[i].out, io[i].so, d->batch, io[i].heads, d->seq_len, d->head_dim, e);
    const int64_t n[3] = {d->batch, io[i].heads, d->seq_len};
    if (!strides_apart(io[i].so, n, 3, d->head_dim)) return VSCAN_ERR_INVALID_ARG;
  }
  const size_t tokens = static_cast<size_t>(d->batch) * d->seq_len;
  for (int i = 0; i < 2; ++i) {
    if (!io[i].in) continue;
    bool same = io[i].in == io[i].out;
    for (int j = 0; j < 3; ++j) same = same && io[i].si[j] == io[i].so[j];
    const Extent in = extent(io[i].in, io[i].si, d->batch, io[i].heads, d->seq_len, d->head_dim, e);
    if (!same && overlaps(in.lo, in.n, outs[i].lo, outs[i].n)) return VSCAN_ERR_INVALID_ARG;
    if (overlaps(outs[i].lo, outs[i].n, d->pos_ids, static_cast<size_t>(d->pos_planes) * tokens * 4) ||
        overlaps(outs[i].lo, outs[i].n, d->inv_freq, static_cast<size_t>(d->rot_dim) * 2) ||
        overlaps(outs[i].lo, outs[i].n, d->axis, static_cast<size_t>(d->rot_dim) * 2))
      return VSCAN_ERR_INVALID_ARG;
  }
  if (d->q && d->k) {          // queries and keys may be views of one projection's output, turned in place
    const Rows q = {d->q, d->q_stride, d->q_heads}, qo = {d->q_out, d->q_out_stride, d->q_heads};
    const Rows k = {d->k, d->k_stride, d->k_heads}, ko = {d->k_out, d->k_out_stride, d->k_heads};
    if (!apart(qo, k, d->batch, d->seq_len, d->head_dim, e) || !apart(ko, q, d->batch, d->seq_len, d->head_dim, e) ||
        !apart(qo, ko, d->batch, d->seq_len, d->head_dim, e))
      return VSCAN_ERR_INVALID_ARG;
  }
  return VSCAN_OK;
}

template <typename T>
static vscan_status launch(const vscan_rope_desc* d, cudaStream_t stream) {
  Params p = {};
  const long long e = sizeof(T);
  auto side = [&](Side& s, const void* in, void* out, const int64_t* si, const int64_t* so, int heads) {
    s = {static_cast<const char*>(in), static_cast<char*>(out), si[0] * e, si[1] * e, si[2] * e, so[0] * e, so[1] * e, so[2] * e,
         in ? heads : 0};
  };
  side(p.side[0], d->q, d->q_out, d->q_stride, d->q_out_stride, d->q_heads);
  side(p.side[1], d->k, d->k_out, d->k_stride, d->k_out_stride, d->k_heads);
  p.pos = d->pos_ids; p.inv_freq = d->inv_freq; p.axis = d->axis;
  p.tokens = d->batch * d->seq_len; p.seq_len = d->seq_len; p.planes = d->pos_planes; p.half = d->rot_dim / 2;
  p.heads = p.side[0].heads + p.side[1].heads;
  p.sign = d->inverse ? -1.f : 1.f;
  // the widest piece whose units tile both the turned and the untouched channels
  const int rest = d->head_dim - d->rot_dim;
  int v = static_cast<int>(16 / e);
  while (v > 1 && (p.half % v || rest % (2 * v))) v /= 2;
  p.pair_units = p.half / v;
  p.units = p.pair_units + rest / (2 * v);
  // enough tokens in a CTA for four units a thread, as long as the grid still covers the SMs several times
  const long long per_token = static_cast<long long>(p.heads) * p.units;
  int tpc = 1;
  while (tpc < kMaxTokens && per_token * tpc < 4 * kThreads && p.tokens / (2 * tpc) >= 148 * 8) tpc *= 2;
  p.tokens_per_cta = tpc;
  p.by_half.set(p.half); p.by_seq.set(p.seq_len); p.by_units.set(p.units); p.by_token.set(static_cast<unsigned>(per_token));
  const size_t smem = static_cast<size_t>(tpc) * p.half * sizeof(float2);
  const unsigned grid = static_cast<unsigned>((p.tokens + tpc - 1) / tpc);
#define VSCAN_ROPE_CASE(V)                                                                                        \
  if (v == V) {                                                                                                   \
    prof_before("rope", stream);                                                                                  \
    VSCAN_CUDA_TRY(d->pairing == VSCAN_ROPE_ADJACENT                                                              \
                       ? launch_dependent(rope_kernel<T, V, true>, dim3(grid), dim3(kThreads), smem, stream, p)   \
                       : launch_dependent(rope_kernel<T, V, false>, dim3(grid), dim3(kThreads), smem, stream, p)); \
    prof_after(stream);                                                                                           \
    VSCAN_AFTER_LAUNCH();                                                                                         \
    return VSCAN_OK;                                                                                              \
  }
  if constexpr (sizeof(T) == 2) { VSCAN_ROPE_CASE(8) }
  VSCAN_ROPE_CASE(4)
  VSCAN_ROPE_CASE(2)
  VSCAN_ROPE_CASE(1)
#undef VSCAN_ROPE_CASE
  return VSCAN_ERR_UNSUPPORTED;
}

}  // namespace rope
}  // namespace vscan

using namespace vscan;

extern "C" vscan_status vscan_rope(const vscan_rope_desc* d, void* stream) {
  const vscan_status st = rope::validate(d);
  if (st != VSCAN_OK) return st;
  if (d->batch == 0 || d->seq_len == 0) return VSCAN_OK;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return d->dtype == VSCAN_F32 ? rope::launch<float>(d, s) : rope::launch<__nv_bfloat16>(d, s);
}
