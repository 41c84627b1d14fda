// vscan_kv_evict: the tokens that gathered least weight leave the paged 8-bit cache.
//
// Two launches.  rank_kernel: a CTA a (sequence, head), or a sequence where all heads keep the same tokens, finds the threshold of
// the weights by an exact radix select and writes the places of the tokens that stay, ascending.  Then the codes of each block of the
// result are gathered from where they lie and written in place.  Token j of the result comes from place src(j) >= j, so
//   sweep_kernel   a warp takes a head's K or V from the first block on: what it writes nobody reads any more.  Where there are enough
//                  heads and sequences to fill the GPU with warps
//   move_kernel    a group of warps a block.  A unit holds all codes of its block in registers, says so in a flag, and writes once every
//                  unit in front of it that reads from the block it will write has said so too.  Those units have begun before it
//                  (units are handed out by a counter) and wait for nobody before they have read, so the waits end
#include "kv_attention_mma.cuh"
#include "topk.cuh"

namespace vscan {
namespace kv {

constexpr int64_t kMostTokens = 0x7ffff000;
constexpr unsigned kEvictPolls = 1u << 22;   // of about 100 ns

struct EvictParams {
  const int32_t* kv_len;
  const int32_t* budget;
  const int32_t* block_table;
  const float* weight;
  float* weight_out;
  uint8_t* cache[2];
  float* scale[2];
  int32_t* kept;          // the caller's, or in the workspace
  int32_t* delta;
  uint32_t* status;
  uint32_t* bad;          // [batch] vscan_status of a sequence
  int2* stay;             // [batch] tokens that stay, -1: left alone; 1 where some leave
  uint32_t* next;         // units handed out so far
  uint32_t* read;         // [batch][kv_heads][2][columns] a unit has read its codes
  uint32_t* keys;         // [batch][heads][max_blocks * block_size] where shared memory does not hold them
  int batch, kv_heads, heads, head_dim, block_size, shift, num_blocks, max_blocks, max_keep, keep_first, keep_last, columns, held;
};

// ---------------------------------------------------------------------------------------------- which tokens stay
// Reads 4 bytes a token and head, once; everything after that is the latency of five passes over keys in shared memory.  8 sequences of 12,000
// to 16,400 tokens, 8 heads of their own (64 CTAs): 25 us, of which a copy of the weights would be one.
__device__ __forceinline__ uint32_t rank_key(float w) { return float_to_key(w == w ? w : -INFINITY); }
constexpr uint32_t kProtected = 0xffffffffu;        // above the key of an infinite weight, or of a sum over the heads that is

__global__ void __launch_bounds__(1024) rank_kernel(EvictParams p) {
  extern __shared__ uint32_t rank_smem[];
  __shared__ SelectScratch sc;
  const int b = blockIdx.y, head = blockIdx.x;
  grid_dependency_wait();
  const int room = p.max_blocks << p.shift, len = p.kv_len[b];
  const int most = min(max(p.budget[b], 0), p.max_keep);
  const int32_t* table = p.block_table + static_cast<size_t>(b) * p.max_blocks;
  const int used = len > 0 && len <= room ? ((len - 1) >> p.shift) + 1 : 0;
  bool wrong = len < 0 || len > room;
  for (int j = threadIdx.x; j < used; j += blockDim.x) wrong = wrong || table[j] < 0 || table[j] >= p.num_blocks;
  wrong = __syncthreads_or(wrong);
  const int n = wrong ? -1 : min(most, len);
  if (head == 0 && threadIdx.x == 0) {
    if (b == 0) { p.status[0] = kStatusFlags | static_cast<uint32_t>(p.batch); *p.next = 0; }
    p.bad[b] = wrong ? VSCAN_ERR_INVALID_ARG : 0;
    p.stay[b] = make_int2(n, n >= 0 && n < len);
    p.delta[b] = wrong ? 0 : n - len;
  }
  // the flags of the heads that this CTA speaks for
  const int each = p.heads == 1 ? p.kv_heads : 1, flags = each * 2 * p.columns;
  uint32_t* read = p.read + (static_cast<size_t>(b) * p.kv_heads + (p.heads == 1 ? 0 : head)) * 2 * p.columns;
  for (int i = threadIdx.x; i < flags; i += blockDim.x) read[i] = 0;
  int32_t* out = p.kept + (static_cast<size_t>(b) * p.heads + head) * p.max_keep;
  if (n <= 0) return;
  if (n == len) {
    for (int i = threadIdx.x; i < n; i += blockDim.x) out[i] = i;
    return;
  }
  uint32_t* keys = p.held >= len ? rank_smem : p.keys + (static_cast<size_t>(b) * p.heads + head) * room;
  constexpr int kAhead = 4;                          // tokens of a thread whose loads are on their way at once
  const bool one_head = p.heads > 1 || p.kv_heads == 1;
  for (long long t0 = threadIdx.x; t0 < len; t0 += kAhead * blockDim.x) {
    const float* w[kAhead];
    float rank[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int t = static_cast<int>(min(t0 + u * static_cast<long long>(blockDim.x), static_cast<long long>(len) - 1));
      w[u] = p.weight + (static_cast<size_t>(table[t >> p.shift]) * p.kv_heads << p.shift) + (t & (p.block_size - 1));
    }
    if (one_head) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) rank[u] = __ldg(w[u] + (static_cast<size_t>(head) << p.shift));
    } else {
      double sum[kAhead] = {};
      for (int h = 0; h < p.kv_heads; ++h)
#pragma unroll
        for (int u = 0; u < kAhead; ++u) sum[u] += __ldg(w[u] + (static_cast<size_t>(h) << p.shift));
#pragma unroll
      for (int u = 0; u < kAhead; ++u) rank[u] = static_cast<float>(sum[u]);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const long long t = t0 + u * static_cast<long long>(blockDim.x);
      if (t < len) keys[t] = t < p.keep_first || t >= static_cast<long long>(len) - p.keep_last ? kProtected : rank_key(rank[u]);
    }
  }
  __syncthreads();
  uint32_t threshold;
  int need;
  block_radix_select(keys, nullptr, len, n, sc, threshold, need);
  // each warp a run of the tokens: how many are over the threshold and on it, then their places behind those of the runs in front
  __shared__ int over_of[32], on_of[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int run = ((len + warps - 1) / warps + 31) & ~31, begin = static_cast<int>(min(static_cast<long long>(warp) * run, static_cast<long long>(len)));
  const int end = static_cast<int>(min(static_cast<long long>(begin) + run, static_cast<long long>(len)));
  int over = 0, on = 0;
  for (int t0 = begin; t0 < end; t0 += 32) {
    const uint32_t key = t0 + lane < end ? keys[t0 + lane] : 0u;
    over += __popc(__ballot_sync(0xffffffffu, t0 + lane < end && key > threshold));
    on += __popc(__ballot_sync(0xffffffffu, t0 + lane < end && key == threshold));
  }
  if (lane == 0) { over_of[warp] = over; on_of[warp] = on; }
  __syncthreads();
  int above = __reduce_add_sync(0xffffffffu, lane < warp ? over_of[lane] : 0), equal = __reduce_add_sync(0xffffffffu, lane < warp ? on_of[lane] : 0);
  for (int t0 = begin; t0 < end; t0 += 32) {
    const uint32_t key = t0 + lane < end ? keys[t0 + lane] : 0u, before = (1u << lane) - 1u;
    const unsigned overs = __ballot_sync(0xffffffffu, t0 + lane < end && key > threshold);
    const unsigned ons = __ballot_sync(0xffffffffu, t0 + lane < end && key == threshold);
    const int e = equal + __popc(ons & before);
    if (((overs >> lane) & 1u) || (((ons >> lane) & 1u) && e < need)) out[above + __popc(overs & before) + min(e, need)] = t0 + lane;
    above += __popc(overs);
    equal += __popc(ons);
  }
}

// Tables of up to 512 tokens: a warp a (sequence, head), 16 keys a lane in registers, the threshold bit by bit, until n
// keys, no more, reach it.  8,192 of 256 tokens: 26 us (53 with CTAs of 128 threads), of 512: 41 (65).  (For the larger tables of a CTA, whose every bit is a
// barrier, the passes of the radix select take no longer.)
constexpr int kRankThreads = 128, kRankKeys = 16;

__global__ void __launch_bounds__(kRankThreads) rank_warp_kernel(EvictParams p) {
  grid_dependency_wait();
  const int lane = threadIdx.x & 31, unit = blockIdx.x * (kRankThreads / 32) + (threadIdx.x >> 5);
  const int b = unit / p.heads, head = unit - b * p.heads;
  if (b >= p.batch) return;
  const int room = p.max_blocks << p.shift, len = p.kv_len[b], most = min(max(p.budget[b], 0), p.max_keep);
  const int used = len > 0 && len <= room ? ((len - 1) >> p.shift) + 1 : 0;      // at most 32
  int mine = 0;
  if (lane < used) mine = p.block_table[static_cast<size_t>(b) * p.max_blocks + lane];
  const bool wrong = __any_sync(0xffffffffu, len < 0 || len > room || mine < 0 || (lane < used && mine >= p.num_blocks));
  const int n = wrong ? -1 : min(most, len);
  if (head == 0 && lane == 0) {
    if (b == 0) { p.status[0] = kStatusFlags | static_cast<uint32_t>(p.batch); *p.next = 0; }
    p.bad[b] = wrong ? VSCAN_ERR_INVALID_ARG : 0;
    p.stay[b] = make_int2(n, n >= 0 && n < len);
    p.delta[b] = wrong ? 0 : n - len;
  }
  const int each = p.heads == 1 ? p.kv_heads : 1, flags = each * 2 * p.columns;
  uint32_t* read = p.read + (static_cast<size_t>(b) * p.kv_heads + (p.heads == 1 ? 0 : head)) * 2 * p.columns;
  for (int i = lane; i < flags; i += 32) read[i] = 0;
  int32_t* out = p.kept + (static_cast<size_t>(b) * p.heads + head) * p.max_keep;
  if (n <= 0) return;
  if (n == len) {
    for (int i = lane; i < n; i += 32) out[i] = i;
    return;
  }
  uint32_t key[kRankKeys], any = 0, all = 0xffffffffu;
#pragma unroll
  for (int i = 0; i < kRankKeys; ++i) {
    const int t = i * 32 + lane, block = __shfl_sync(0xffffffffu, mine, t >> p.shift & 31);
    key[i] = 0;                                      // less than any rank
    if (t < len) {
      const float* w = p.weight + (static_cast<size_t>(block) * p.kv_heads << p.shift) + (t & (p.block_size - 1));
      if (t < p.keep_first || t >= static_cast<long long>(len) - p.keep_last) {
        key[i] = kProtected;
      } else if (p.heads > 1 || p.kv_heads == 1) {
        key[i] = rank_key(__ldg(w + (static_cast<size_t>(head) << p.shift)));
      } else {
        double sum = 0.;
        for (int h = 0; h < p.kv_heads; ++h) sum += __ldg(w + (static_cast<size_t>(h) << p.shift));
        key[i] = rank_key(static_cast<float>(sum));
      }
      any |= key[i];
      all &= key[i];
    }
  }
  any = __reduce_or_sync(0xffffffffu, any);
  all = __reduce_and_sync(0xffffffffu, all);
  // the n-th largest key, from the first bit down: those that all keys share need no count
  uint32_t threshold = 0;
  for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
    const uint32_t with = threshold | bit;
    if (!((any ^ all) & bit)) { threshold |= all & bit; continue; }
    int count = 0;
#pragma unroll
    for (int i = 0; i < kRankKeys; ++i) count += key[i] >= with;
    const int reach = __reduce_add_sync(0xffffffffu, count);
    if (reach == n) { threshold = with - 1; break; }   // the n that reach it are over this
    if (reach > n) threshold = with;
  }
  int over = 0;
#pragma unroll
  for (int i = 0; i < kRankKeys; ++i) over += key[i] > threshold;
  const int need = n - __reduce_add_sync(0xffffffffu, over);
  int above = 0, equal = 0;
  const uint32_t before = (1u << lane) - 1u;
#pragma unroll
  for (int i = 0; i < kRankKeys; ++i) {
    const unsigned overs = __ballot_sync(0xffffffffu, key[i] > threshold), ons = __ballot_sync(0xffffffffu, key[i] == threshold);
    const int e = equal + __popc(ons & before);
    if (((overs >> lane) & 1u) || (((ons >> lane) & 1u) && e < need)) out[above + __popc(overs & before) + min(e, need)] = i * 32 + lane;
    above += __popc(overs);
    equal += __popc(ons);
  }
}

// ---------------------------------------------------------------------------------------------- moving them
// Bytes bound both kernels: codes that stay, in and out, once.  A block's new scale needs all of its codes before the first is written, so
// they are held in registers; codes whose scale stays are copied, the others recoded in f16 (no value is rounded before its one rounding).
// Largest magnitude among 16 codes, as a code (a byte whose order is that of the magnitudes)
template <int KV>
__device__ __forceinline__ uint32_t peak_code(const uint4& v) {
  uint32_t m;
  if constexpr (KV == VSCAN_KV_E4M3)
    m = __vmaxu4(__vmaxu4(v.x & 0x7f7f7f7fu, v.y & 0x7f7f7f7fu), __vmaxu4(v.z & 0x7f7f7f7fu, v.w & 0x7f7f7f7fu));
  else
    m = __vmaxu4(__vmaxu4(__vabs4(v.x), __vabs4(v.y)), __vmaxu4(__vabs4(v.z), __vabs4(v.w)));
  m = __vmaxu4(m, m >> 16);
  return max(m & 0xffu, (m >> 8) & 0xffu);
}
template <int KV>
__device__ __forceinline__ float code_magnitude(uint32_t code) {
  if constexpr (KV == VSCAN_KV_E4M3) {
    float f[4];
    decode4<KV>(code, f);
    return f[0];                                     // the code of NaN gives NaN
  } else {
    return static_cast<float>(code);                 // 128 where the code is -128
  }
}
// 16 codes times a power of two between 2^-14 and 2^14 that fit the type afterwards, as codes: two at a time in f16.  Codes are exact there; so is the
// product as far as a code's last bit goes; one rounding, to nearest, ties to even (I8: 1.5 x 2^10 + x is rounded to a whole number, whose
// last byte is the code).
template <int KV>
__device__ __forceinline__ uint4 recode_half(const uint4& old, uint32_t ratio) {
  const uint32_t w[4] = {old.x, old.y, old.z, old.w};
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t lo, hi;
    codes_to_f16<KV>(w[i], lo, hi);
    if constexpr (KV == VSCAN_KV_E4M3) {
      asm("{\n\t.reg .b16 a, b;\n\t.reg .b32 x, y;\n\t"
          "mul.rn.f16x2 x, %1, %3;\n\tmul.rn.f16x2 y, %2, %3;\n\t"
          "cvt.rn.satfinite.e4m3x2.f16x2 a, x;\n\tcvt.rn.satfinite.e4m3x2.f16x2 b, y;\n\t"
          "mov.b32 %0, {a, b};\n\t}"
          : "=r"(r[i]) : "r"(lo), "r"(hi), "r"(ratio));
    } else {
      asm("fma.rn.f16x2 %0, %0, %2, %3;\n\tfma.rn.f16x2 %1, %1, %2, %3;" : "+r"(lo), "+r"(hi) : "r"(ratio), "r"(0x66006600u));
      r[i] = __byte_perm(lo, hi, 0x6420);
    }
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}
// 16 codes of one scale as codes of another: the value, then its code
template <int KV>
__device__ __forceinline__ uint4 recode(const uint4& old, float scale, float inv) {
  const uint32_t w[4] = {old.x, old.y, old.z, old.w};
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float f[4];
    decode4<KV>(w[i], f);
    r[i] = encode4<KV>(f[0] * scale * inv, f[1] * scale * inv, f[2] * scale * inv, f[3] * scale * inv);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}

// The scale of a block from its peak, and its codes
struct Fresh { float s, inv; bool nan, fits; };   // fits: no element is beyond the largest code
template <int KV>
__device__ __forceinline__ Fresh fresh_scale(uint32_t peak) {
  const int e = scale_exponent<KV>(__uint_as_float(peak));
  const bool nan = peak >= 0x7f800000u;
  return {nan ? __uint_as_float(0x7fc00000u) : exp2_int(e), nan ? 0.f : exp2_int(-e), nan, e < kExpMax};
}
template <int KV>
__device__ __forceinline__ uint4 moved(const uint4& old, float scale, const Fresh& f) {
  if (f.nan) return make_uint4(0, 0, 0, 0);
  if (scale == f.s) return old;
  const uint32_t ratio = __float_as_uint(scale * f.inv), e = ratio >> 23;
  if (!(ratio & 0x7fffffu) && e >= 127 - 14 && e <= 127 + 14 && f.fits) return recode_half<KV>(old, (e - 127 + 15) * 0x04000400u);
  return recode<KV>(old, scale, f.inv);
}

// A load that stands where it is written
__device__ __forceinline__ int load_now(const int32_t* at) {
  int v;
  asm volatile("ld.global.s32 %0, [%1];" : "=r"(v) : "l"(at) : "memory");
  return v;
}

// Few sequences: a unit a block, so that all blocks of a sequence move at once.  As many warps a unit as hold its codes in a few registers a
// thread, no more: blocks of 64 tokens of 128 channels move in 28 us with four warps a unit, 40 with eight (8 x 2,048 tokens, 8 heads).
__host__ __device__ constexpr int move_threads(int w) { return w == 8 ? 256 : 128; }

template <int KV, int W, int HELD>
__global__ void __launch_bounds__(move_threads(W)) move_kernel(EvictParams p) {
  constexpr int kThreads = move_threads(W), kGroups = kThreads / 32 / W, kWeights = 8 / W;   // weights of a lane: 256 a block at most
  __shared__ uint32_t peaks[kThreads / 32];
  __shared__ uint32_t ticket;
  __shared__ int quit;
  grid_dependency_wait();
  if (threadIdx.x == 0) { ticket = atomicAdd(p.next, 1u); quit = 0; }
  __syncthreads();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, group = warp / W, in_group = threadIdx.x - group * W * 32;
  const long long unit = static_cast<long long>(ticket) * kGroups + group;
  const int which = static_cast<int>(unit & 1);
  long long rest = unit >> 1;
  const int h = static_cast<int>(rest % p.kv_heads);
  rest /= p.kv_heads;
  const int b = static_cast<int>(rest % p.batch), j = static_cast<int>(rest / p.batch);
  if (j >= p.columns) return;                        // (a group of several warps is its whole CTA)
  const int32_t* table = p.block_table + static_cast<size_t>(b) * p.max_blocks;
  const int32_t* src = p.kept + (static_cast<size_t>(b) * p.heads + (p.heads > 1 ? h : 0)) * p.max_keep;
  const int first = j << p.shift, mask = p.block_size - 1, cpr = p.head_dim / 16;
  // places of this thread's pieces, as far as the list goes, beside the loads that say how far it counts
  int from[HELD];
#pragma unroll
  for (int k = 0; k < HELD; ++k) {
    const int r = (in_group + k * 32 * W) / cpr;
    from[k] = load_now(src + min(first + min(r, mask), p.max_keep - 1));
  }
  const int ahead = j - 1 - lane >= 0 ? load_now(src + ((j - 1 - lane) << p.shift) + mask) : -1;   // last token of a unit in front
  const int2 stay = p.stay[b];
  const int n = min(stay.x - first, p.block_size);
  if (n <= 0) return;
  const bool moves_weights = which == 0 && p.weight_out && (stay.y || p.weight_out != p.weight);
  if (!stay.y && !moves_weights) return;
  const size_t to = static_cast<size_t>(table[j]) * p.kv_heads + h;
  const int last = src[first + n - 1];
  const bool stays = last == first + n - 1;          // places ascend and none is below its number: then all of the block's tokens stay

  float w[kWeights];
  if (moves_weights) {
#pragma unroll
    for (int k = 0; k < kWeights; ++k) {
      const int r = in_group + k * 32 * W;
      if (r < n) {
        const int t = src[first + r];
        w[k] = p.weight[((static_cast<size_t>(table[t >> p.shift]) * p.kv_heads + h) << p.shift) + (t & mask)];
      }
    }
  }
  auto store_weights = [&]() {
    if (moves_weights) {
#pragma unroll
      for (int k = 0; k < kWeights; ++k) {
        const int r = in_group + k * 32 * W;
        if (r < n) p.weight_out[(to << p.shift) + r] = w[k];
      }
    }
  };
  if (stays) {                                       // nothing moves, and nobody waits for this unit
    if (p.weight_out != p.weight) store_weights();
    return;
  }

  const int total = n * cpr;
  const uint8_t* codes = p.cache[which];
  uint4 held[HELD];
  float scale[HELD];
  float top = 0.f;
#pragma unroll
  for (int k = 0; k < HELD; ++k) {
    const int c = in_group + k * 32 * W;
    held[k] = make_uint4(0, 0, 0, 0);
    scale[k] = 0.f;
    if (c < total) {
      const int r = c / cpr, t = from[k];
      const size_t cell = static_cast<size_t>(table[t >> p.shift]) * p.kv_heads + h;
      scale[k] = p.scale[which][cell];
      held[k] = *reinterpret_cast<const uint4*>(codes + ((cell << p.shift) + (t & mask)) * p.head_dim + (c - r * cpr) * 16);
    }
  }
#pragma unroll
  for (int k = 0; k < HELD; ++k) {
    const float m = code_magnitude<KV>(peak_code<KV>(held[k])) * scale[k];
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(fabsf(m)));
  }
  uint32_t peak = __reduce_max_sync(0xffffffffu, __float_as_uint(top) & 0x7fffffffu);
  if constexpr (W > 1) {
    if (lane == 0) peaks[warp] = peak;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) peak = max(peak, peaks[i]);
  } else {
    __syncwarp();
  }
  // ---- all of the group's reads are done: say so, then wait for the units in front that read from the block to be written
  uint32_t* read = p.read + ((static_cast<size_t>(b) * p.kv_heads + h) * 2 + which) * p.columns;
  bool ok = true;
  if (W == 1 || warp == 0) {
    if (lane == 0) asm volatile("st.release.gpu.global.u32 [%0], 1;" ::"l"(read + j) : "memory");
    for (int c0 = j - 1; c0 >= 0; c0 -= 32) {
      const int c = c0 - lane;
      // its last token comes from this block or from behind it
      const bool reads = c >= 0 && (c0 == j - 1 ? ahead : src[(c << p.shift) + mask]) >= first;
      unsigned polls = 0;
      uint32_t done = !reads;
      while (!done && polls < kEvictPolls) {
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(done) : "l"(read + c) : "memory");
        if (!done) { __nanosleep(100); ++polls; }
      }
      ok = __all_sync(0xffffffffu, done != 0) && ok;
      if (!ok || !__all_sync(0xffffffffu, reads)) break;                    // units further in front read from further in front
    }
    if constexpr (W > 1) { if (!ok && lane == 0) quit = 1; }
  }
  if constexpr (W > 1) {
    __syncthreads();
    ok = quit == 0;
  }
  if (!ok) {
    if (in_group == 0) p.bad[b] = VSCAN_ERR_TIMEOUT;
    return;
  }
  const Fresh f = fresh_scale<KV>(peak);
  uint8_t* dst = p.cache[which] + (to << p.shift) * p.head_dim;
#pragma unroll
  for (int k = 0; k < HELD; ++k) {
    const int c = in_group + k * 32 * W;
    if (c < total) st_16(dst + static_cast<size_t>(c) * 16, moved<KV>(held[k], scale[k], f));
  }
  if (in_group == 0) p.scale[which][to] = f.s;
  store_weights();
}

// ---------------------------------------------------------------------------------------------- a warp a head's K or V
// The next block's codes are on their way while one is coded and written.  Bound by DRAM, which reads and writes the same blocks in turn: 256 x
// 224 tokens, 32 heads of 128, 940 MB: 237 us, 4.0 TB/s (216 us if the codes were only copied).
constexpr int kSweepThreads = 128;

template <int KV, int HELD>
__global__ void __launch_bounds__(kSweepThreads, HELD > 4 ? 4 : 5) sweep_kernel(EvictParams p) {
  constexpr int kWeights = 8;
  grid_dependency_wait();
  const int lane = threadIdx.x & 31;
  const long long unit = static_cast<long long>(blockIdx.x) * (kSweepThreads / 32) + (threadIdx.x >> 5);
  const int which = static_cast<int>(unit & 1);
  const long long rest = unit >> 1;
  const int h = static_cast<int>(rest % p.kv_heads);
  if (rest / p.kv_heads >= p.batch) return;
  const int b = static_cast<int>(rest / p.kv_heads);
  const int2 stay = p.stay[b];
  const bool moves_weights = which == 0 && p.weight_out && (stay.y || p.weight_out != p.weight);
  if (stay.x <= 0 || (!stay.y && !moves_weights)) return;
  const int32_t* table = p.block_table + static_cast<size_t>(b) * p.max_blocks;
  const int32_t* src = p.kept + (static_cast<size_t>(b) * p.heads + (p.heads > 1 ? h : 0)) * p.max_keep;
  const int mask = p.block_size - 1, cpr = p.head_dim / 16;
  const uint8_t* codes = p.cache[which];
  int row[HELD];                                     // of this lane's pieces within a block, and their bytes within a row
  int col[HELD];
#pragma unroll
  for (int k = 0; k < HELD; ++k) {
    const int c = lane + k * 32;
    row[k] = c / cpr;
    col[k] = (c - row[k] * cpr) * 16;
  }
  const int columns = ((stay.x - 1) >> p.shift) + 1;
  uint4 held[HELD], next[HELD];
  float scale[HELD], next_scale[HELD];
  bool moves = false, next_moves;                    // a block of which some token does not stay in its place
  auto load = [&](int j, uint4* v, float* sc) {
    const int first = j << p.shift, n = min(stay.x - first, p.block_size);
    const bool some = n > 0 && stay.y && src[first + max(n, 1) - 1] != first + n - 1;
#pragma unroll
    for (int k = 0; k < HELD; ++k) {
      v[k] = make_uint4(0, 0, 0, 0);
      sc[k] = 0.f;
      if (some && row[k] < n) {
        const int t = src[first + row[k]];
        const size_t from = static_cast<size_t>(table[t >> p.shift]) * p.kv_heads + h;
        sc[k] = p.scale[which][from];
        v[k] = *reinterpret_cast<const uint4*>(codes + ((from << p.shift) + (t & mask)) * p.head_dim + col[k]);
      }
    }
    return some;
  };
  moves = load(0, held, scale);
  for (int j = 0; j < columns; ++j) {
    const int first = j << p.shift, n = min(stay.x - first, p.block_size);
    const size_t to = static_cast<size_t>(table[j]) * p.kv_heads + h;
    next_moves = j + 1 < columns && load(j + 1, next, next_scale);
    if (moves_weights && (moves || p.weight_out != p.weight)) {
      float w[kWeights];
#pragma unroll
      for (int k = 0; k < kWeights; ++k) {
        const int r = lane + k * 32;
        if (r < n) {
          const int t = src[first + r];
          w[k] = p.weight[((static_cast<size_t>(table[t >> p.shift]) * p.kv_heads + h) << p.shift) + (t & mask)];
        }
      }
      __syncwarp();                                  // all of them are read before one is written
#pragma unroll
      for (int k = 0; k < kWeights; ++k) {
        const int r = lane + k * 32;
        if (r < n) p.weight_out[(to << p.shift) + r] = w[k];
      }
    }
    if (moves) {
      float top = 0.f;
#pragma unroll
      for (int k = 0; k < HELD; ++k) {
        const float m = code_magnitude<KV>(peak_code<KV>(held[k])) * scale[k];
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(fabsf(m)));
      }
      const uint32_t peak = __reduce_max_sync(0xffffffffu, __float_as_uint(top) & 0x7fffffffu);
      __syncwarp();                                  // all lanes' codes are read before one is written
      const Fresh f = fresh_scale<KV>(peak);
      uint8_t* dst = p.cache[which] + (to << p.shift) * p.head_dim;
#pragma unroll
      for (int k = 0; k < HELD; ++k)
        if (row[k] < n) st_16(dst + static_cast<size_t>(lane + k * 32) * 16, moved<KV>(held[k], scale[k], f));
      if (lane == 0) p.scale[which][to] = f.s;
    }
    __syncwarp();
    moves = next_moves;
#pragma unroll
    for (int k = 0; k < HELD; ++k) { held[k] = next[k]; scale[k] = next_scale[k]; }
  }
}

// ---------------------------------------------------------------------------------------------- host side
static vscan_status validate_evict(const vscan_kv_evict_desc* d) {
  if (!d) return VSCAN_ERR_INVALID_ARG;
  if (d->kv_dtype != VSCAN_KV_E4M3 && d->kv_dtype != VSCAN_KV_I8) return VSCAN_ERR_INVALID_ARG;
  if (d->batch < 0 || d->kv_heads <= 0 || d->head_dim <= 0 || d->head_dim % 16 || d->num_blocks < 0 || d->max_blocks < 0 || d->max_keep < 0 ||
      d->keep_first < 0 || d->keep_last < 0 || !block_size_ok(d->block_size))
    return VSCAN_ERR_INVALID_ARG;
  if (d->batch == 0) return VSCAN_OK;
  if (!d->kv_len || !d->budget || !d->delta) return VSCAN_ERR_INVALID_ARG;
  if ((d->max_blocks > 0 && !d->block_table) ||
      (d->num_blocks > 0 && d->max_blocks > 0 && (!d->weight || !d->k_cache || !d->v_cache || !d->k_scale || !d->v_scale)))
    return VSCAN_ERR_INVALID_ARG;
  if (d->head_dim > 256 || d->batch > kMaxBatch || d->kv_heads > 65535 || static_cast<int64_t>(d->max_blocks) * d->block_size > kMostTokens ||
      static_cast<int64_t>(d->batch) * d->kv_heads * (d->max_keep / d->block_size + 1) > (int64_t{1} << 28))
    return VSCAN_ERR_UNSUPPORTED;
  struct Rng { const void* p; size_t n; };
  const size_t B = d->batch, H = d->kv_heads, pool = static_cast<size_t>(d->num_blocks) * H, bs = d->block_size;
  const Rng all[] = {{d->kv_len, B * 4}, {d->budget, B * 4}, {d->block_table, B * d->max_blocks * 4}, {d->weight, pool * bs * 4},
                     {d->weight_out == d->weight ? nullptr : d->weight_out, pool * bs * 4},
                     {d->k_cache, pool * bs * d->head_dim}, {d->v_cache, pool * bs * d->head_dim}, {d->k_scale, pool * 4}, {d->v_scale, pool * 4},
                     {d->kept, B * (d->per_head ? H : 1) * d->max_keep * 4}, {d->delta, B * 4}};
  constexpr int kInputs = 4, kAll = 11;
  for (const Rng& r : all)
    if (r.p && !aligned16(r.p)) return VSCAN_ERR_INVALID_ARG;
  for (int o = kInputs; o < kAll; ++o)
    for (int i = 0; i < o; ++i)
      if (overlaps(all[o].p, all[o].n, all[i].p, all[i].n)) return VSCAN_ERR_INVALID_ARG;
  return VSCAN_OK;
}

// workspace: status word | a word per sequence | tokens that stay | counter | flags of the units | kept, if the caller wants none | keys
constexpr size_t kHeldKeys = 16384;      // in shared memory, 64 KB: beyond that they pass through L2
struct EvictLayout {
  size_t bad, stay, next, read, kept, keys, bytes;
  int columns, heads;
};
static EvictLayout layout_of(const vscan_kv_evict_desc* d) {
  EvictLayout l;
  const size_t B = d->batch, H = d->kv_heads, room = static_cast<size_t>(d->max_blocks) * d->block_size;
  l.columns = static_cast<int>((static_cast<int64_t>(d->max_keep) + d->block_size - 1) / d->block_size);
  l.heads = d->per_head ? d->kv_heads : 1;
  l.bad = kStatusBytes;
  l.stay = l.bad + round_up(B * 4, 256);
  l.next = l.stay + round_up(B * 8, 256);
  l.read = l.next + 256;
  l.kept = l.read + round_up(B * H * 2 * l.columns * 4, 256);
  // (counted whether or not the caller has a buffer for them, so that the size depends on sizes only)
  l.keys = l.kept + round_up(B * l.heads * static_cast<size_t>(d->max_keep) * 4, 256);
  l.bytes = l.keys + (room > kHeldKeys ? round_up(B * l.heads * room * 4, 256) : 0);
  return l;
}

// As many warps as the sweep needs to keep DRAM busy (14 an SM).  With 16,384 of them: 237 us, 354 by blocks and flags; fewer than that, and each
// warp's chain of blocks is longer than the time that all of them need side by side.
constexpr int64_t kSweeps = 148 * 14;

template <int KV>
static vscan_status launch_moves(const EvictParams& p, cudaStream_t stream) {
  if (p.columns == 0) return VSCAN_OK;
  const int chunks = p.block_size * p.head_dim / 16;
  const int64_t sweeps = static_cast<int64_t>(p.batch) * p.kv_heads * 2;
  if (chunks <= 256 && sweeps >= kSweeps) {
    const dim3 grid(static_cast<unsigned>((sweeps + kSweepThreads / 32 - 1) / (kSweepThreads / 32)));
    prof_before("kv_evict_sweep", stream);
    VSCAN_CUDA_TRY(chunks <= 128 ? launch_dependent(sweep_kernel<KV, 4>, grid, dim3(kSweepThreads), 0, stream, p)
                                 : launch_dependent(sweep_kernel<KV, 8>, grid, dim3(kSweepThreads), 0, stream, p));
    prof_after(stream);
    VSCAN_AFTER_LAUNCH();
    return VSCAN_OK;
  }
  // as many warps to a unit as keep its codes in registers
  const int w = chunks <= 256 ? 1 : chunks <= 512 ? 4 : 8, groups = move_threads(w) / 32 / w;
  const int64_t units = static_cast<int64_t>(p.batch) * p.kv_heads * 2 * p.columns;
  const dim3 grid(static_cast<unsigned>((units + groups - 1) / groups));
  prof_before("kv_evict_move", stream);
  VSCAN_CUDA_TRY(chunks <= 128 ? launch_dependent(move_kernel<KV, 1, 4>, grid, dim3(move_threads(1)), 0, stream, p)
                 : chunks <= 256 ? launch_dependent(move_kernel<KV, 1, 8>, grid, dim3(move_threads(1)), 0, stream, p)
                 : chunks <= 512 ? launch_dependent(move_kernel<KV, 4, 4>, grid, dim3(move_threads(4)), 0, stream, p)
                 : chunks <= 1024 ? launch_dependent(move_kernel<KV, 8, 4>, grid, dim3(move_threads(8)), 0, stream, p)
                 : chunks <= 2048 ? launch_dependent(move_kernel<KV, 8, 8>, grid, dim3(move_threads(8)), 0, stream, p)
                                  : launch_dependent(move_kernel<KV, 8, 16>, grid, dim3(move_threads(8)), 0, stream, p));
  prof_after(stream);
  VSCAN_AFTER_LAUNCH();
  return VSCAN_OK;
}

template <int KV>
static vscan_status launch_evict(const EvictParams& p, cudaStream_t stream) {
  const int64_t room = static_cast<int64_t>(p.max_blocks) * p.block_size;
  // Where there are no more ranks than two CTAs an SM, the chain of passes counts: as many threads as there is work for.  Where there are more, small
  // CTAs, several an SM, whose barriers hold up fewer.  Microseconds with 128 / 256 / 512 / 1,024 threads: 64 ranks of 1,000 tokens 12 / 10 / 10 / 11, of
  // 2,000 18 / 14 / 12 / 12, of 4,000 28 / 18 / 14 / 14, of 16,000 87 / 51 / 33 / 26; 8,192 of 1,000 94 / 121 / 198 / 381, of 2,000 153 / 180 /
  // 244 / 436, of 4,000 272 / 297 / 364 / 528, of 8,000 598 / 530 / 602 / 786; 1,024 of 2,000 26 / 28 / 37 / 59, of 16,000 312 / 178 / 149 / 168.
  const bool few = static_cast<int64_t>(p.heads) * p.batch <= 2 * 148;
  const int threads = room <= 512 ? 256 : room <= 1024 ? (few ? 512 : 128) : room <= 4096 ? (few ? 1024 : 256) : few ? 1024 : 512;
  const int64_t ranks = static_cast<int64_t>(p.heads) * p.batch;
  if (room <= 32 * kRankKeys && !few) {
    prof_before("kv_evict_rank", stream);
    VSCAN_CUDA_TRY(launch_dependent(rank_warp_kernel, dim3(static_cast<unsigned>((ranks + kRankThreads / 32 - 1) / (kRankThreads / 32))), dim3(kRankThreads), 0,
                                    stream, p));
    prof_after(stream);
    VSCAN_AFTER_LAUNCH();
    return launch_moves<KV>(p, stream);
  }
  const size_t smem = static_cast<size_t>(p.held) * 4;
  VSCAN_CUDA_TRY(allow_smem(rank_kernel, smem));
  prof_before("kv_evict_rank", stream);
  VSCAN_CUDA_TRY(launch_dependent(rank_kernel, dim3(p.heads, p.batch), dim3(threads), smem, stream, p));
  prof_after(stream);
  VSCAN_AFTER_LAUNCH();
  return launch_moves<KV>(p, stream);
}

}  // namespace kv
}  // namespace vscan

using namespace vscan;

extern "C" size_t vscan_kv_evict_workspace_bytes(const vscan_kv_evict_desc* d) {
  if (!d || d->batch <= 0 || d->kv_heads <= 0 || d->max_blocks < 0 || d->max_keep < 0 || !kv::block_size_ok(d->block_size)) return kStatusBytes;
  return kv::layout_of(d).bytes;
}

extern "C" vscan_status vscan_kv_evict(const vscan_kv_evict_desc* d, void* workspace, size_t workspace_bytes, void* stream_) {
  const vscan_status st = kv::validate_evict(d);
  if (st != VSCAN_OK) return st;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  if (!workspace || !aligned256(workspace) || workspace_bytes < vscan_kv_evict_workspace_bytes(d)) return VSCAN_ERR_WORKSPACE;
  if (d->batch == 0) {
    VSCAN_CUDA_TRY(cudaMemsetAsync(workspace, 0, sizeof(uint32_t), stream));
    return VSCAN_OK;
  }
  const kv::EvictLayout l = kv::layout_of(d);
  char* ws = static_cast<char*>(workspace);
  kv::EvictParams p = {};
  p.kv_len = d->kv_len; p.budget = d->budget; p.block_table = d->block_table; p.weight = d->weight; p.weight_out = d->weight_out;
  p.cache[0] = static_cast<uint8_t*>(d->k_cache); p.cache[1] = static_cast<uint8_t*>(d->v_cache);
  p.scale[0] = d->k_scale; p.scale[1] = d->v_scale;
  p.kept = d->kept ? d->kept : reinterpret_cast<int32_t*>(ws + l.kept);
  p.delta = d->delta;
  p.status = reinterpret_cast<uint32_t*>(ws); p.bad = reinterpret_cast<uint32_t*>(ws + l.bad); p.stay = reinterpret_cast<int2*>(ws + l.stay);
  p.next = reinterpret_cast<uint32_t*>(ws + l.next); p.read = reinterpret_cast<uint32_t*>(ws + l.read); p.keys = reinterpret_cast<uint32_t*>(ws + l.keys);
  p.batch = d->batch; p.kv_heads = d->kv_heads; p.heads = l.heads; p.head_dim = d->head_dim; p.block_size = d->block_size;
  p.num_blocks = d->num_blocks; p.max_blocks = d->max_blocks; p.max_keep = d->max_keep; p.keep_first = d->keep_first; p.keep_last = d->keep_last;
  p.columns = l.columns;
  const int64_t room = static_cast<int64_t>(d->max_blocks) * d->block_size;
  p.held = static_cast<int>(room < static_cast<int64_t>(kv::kHeldKeys) ? room : kv::kHeldKeys);
  while ((1 << p.shift) < p.block_size) ++p.shift;
  return d->kv_dtype == VSCAN_KV_E4M3 ? kv::launch_evict<VSCAN_KV_E4M3>(p, stream) : kv::launch_evict<VSCAN_KV_I8>(p, stream);
}
