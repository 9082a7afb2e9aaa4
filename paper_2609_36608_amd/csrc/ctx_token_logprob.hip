// ctx_token_logprob.hip -- log probabilities of given tokens, entropy, top alternatives
// and their gradient for gfx950 (MI355X), behind the C ABI declared in
// include/ctx_token_logprob.h.
//
// A row of V logits is read once: bound by HBM for many rows, by latency for a few.  Over
// 151,936 bf16 logits: 4,301 rows of which 0.8 count 177 us, 6.0 TB/s (up to 253 in the first
// milliseconds of load, while the clock falls: bound by exps as much); 8 rows with 20 alternatives 12.3 us and 6.6
// for the merge; 2,057 rows and their gradient 286 us, 6.1 TB/s.
//
//   * logprob_kernel: a workgroup of 4 waves per row, or per share of a row where there
//     are few.  Every lane keeps a running maximum m and, with d = (z - m) scale log2 e,
//     s = sum 2^d and t = sum 2^d d, rescaled once per tile of 4 loads: raising m so
//     that every d falls by r makes them 2^-r s and 2^-r (t - r s).  Then
//     log sum exp x = scale m + ln2 log2 s, and the entropy is ln2 (log2 s - t / s).
//     d counts from the rounded product of m, up to 2^24, as do all that use s and t.
//   * Alternatives: a wave holds the best `top` it has met as 64-bit keys, the value's
//     order above the complement of the column, so that keys differ and the larger key
//     is the better alternative.  A chunk enters the search only if one of its values
//     passes the wave's threshold, its top-th best value so far; that starts at the
//     top-th largest of the lanes' maxima over the first tile, which as many values
//     reach.  Values that pass are collected, up to 128 keys, and cut back to the best
//     by counting for each how many are larger.
//   * logprob_merge_kernel joins the shares of a row, by the same counting.
//   * logprob_grad_kernel: one pass, reading and writing each row once; the given
//     tokens' entries are written over afterwards by one thread each.

#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <type_traits>

#include "ctx_token_logprob.h"

// the library's per-thread last-error message (defined with the attention entry points)
__attribute__((visibility("hidden"))) int ctx_report_error(int code, const char* msg);
__attribute__((visibility("hidden"))) void ctx_clear_error();

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kTileLoads = 4;                      // 16-byte chunks per lane and tile
constexpr int kTileChunks = 64 * kTileLoads;       // of a wave
constexpr int kMostTop = CTX_LOGPROB_MAX_TOP;
constexpr int kMostTokens = CTX_LOGPROB_MAX_TOKENS;
constexpr int kHeldKeys = 128;                     // of a wave: the best and up to 64 more
constexpr int kMostSplits = 64;
constexpr int32_t kMostVocab = 1 << 28;
constexpr int32_t kMostGroups = 0xffffffffu / kThreads;  // of a launch, whose threads are counted in 32 bits
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kFloor = -1e38f;  // logits up to here are masked
// 2^kLeast is 0 in fp32, and a finite product with it is too (0 times -inf would be NaN)
constexpr float kLeast = -200.f;

template <typename T>
constexpr int kChunkOf = 16 / sizeof(T);  // elements of a 16-byte chunk

struct RowsArgs {
  const void* logits;
  int64_t stride;
  int32_t vocab, rows, splits;
  const int32_t* tokens;
  int32_t num_tokens;
  const uint8_t* mask;
  float scale, factor;  // of a logit, also in log2 units
  int32_t top;
  float *token_logp, *entropy, *stats, *top_logp;
  int32_t* top_tokens;
  float4* part;    // [rows, splits]
  uint64_t* keys;  // [rows, splits, top]
};

template <int kBy>
__device__ __forceinline__ float row_rotate(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x120 + kBy, 0xf, 0xf, false));
}

// Reduction over the wave, in a fixed order; every lane ends with the result.
template <typename Op>
__device__ __forceinline__ float wave_reduce(float x, Op op) {
  x = op(x, __shfl_xor(x, 32));
  x = op(x, __shfl_xor(x, 16));
  x = op(x, row_rotate<8>(x));
  x = op(x, row_rotate<4>(x));
  x = op(x, row_rotate<2>(x));
  return op(x, row_rotate<1>(x));
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
// keeps a NaN
__device__ __forceinline__ float max_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float wave_max(float x) {
  return wave_reduce(x, [](float a, float b) { return max_of(a, b); });
}
__device__ __forceinline__ float wave_sum(float x) {
  return wave_reduce(x, [](float a, float b) { return a + b; });
}

template <typename T>
__device__ __forceinline__ void unpack(u32x4 x, float (&z)[kChunkOf<T>]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      z[2 * i] = __uint_as_float(x[i] << 16);
      z[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
    } else {
      z[i] = __uint_as_float(x[i]);
    }
  }
}

template <typename T>
__device__ __forceinline__ float value(const void* row, int64_t at) {
  if constexpr (sizeof(T) == 2)
    return __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(row)[at] << 16);
  else
    return reinterpret_cast<const float*>(row)[at];
}

// Buffer resource over `bytes` bytes from a wave-uniform base: loads past the end return zeros.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_rsrc(const void* base, uint32_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(base);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(((uint64_t)hi << 32) | lo), (short)0,
                                           (int)__builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}

constexpr int kNonTemporal = 2;  // buffer cache-policy bits: streamed once

__device__ __forceinline__ u32x4 load_chunk(__amdgpu_buffer_rsrc_t r, int offset) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, offset, 0, kNonTemporal));
}

// bytes of a row that loads may touch: whole words, so that the last of an odd count of
// bf16 is among them
template <typename T>
__device__ __forceinline__ uint32_t row_bytes(int32_t vocab) {
  return ((uint32_t)vocab * (uint32_t)sizeof(T) + 3u) & ~3u;
}

// the wave's own LDS accesses execute in order; the compiler must not move them
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

// A value's order as an unsigned number (-0 is +0), and back.
__device__ __forceinline__ uint32_t order_of(float z) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t order) {
  return __uint_as_float(order ^ (((order >> 31) - 1u) | 0x80000000u));
}
__device__ __forceinline__ uint64_t key_of(float z, int32_t column) {
  return (uint64_t)order_of(z) << 32 | (uint32_t)~column;
}

// How many of keys[0 .. n) are larger than each of two; n a multiple of 8, keys 16-byte aligned,
// zeros behind the last.
__device__ __forceinline__ void ranks_of(uint64_t k0, uint64_t k1, const uint64_t* keys, int n, int& r0, int& r1) {
  typedef unsigned long long u64x2 __attribute__((ext_vector_type(2)));
  r0 = r1 = 0;
  for (int i = 0; i < n; i += 8) {
    u64x2 k[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) k[j] = *reinterpret_cast<const u64x2*>(keys + i + 2 * j);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      r0 += (k[j].x > k0 ? 1 : 0) + (k[j].y > k0 ? 1 : 0);
      r1 += (k[j].x > k1 ? 1 : 0) + (k[j].y > k1 ? 1 : 0);
    }
  }
}

constexpr int round8(int n) { return (n + 7) & -8; }

// A wave's alternatives: keys[0 .. count), of which any may be among the best `top`, and a
// key that others must pass to be.  A wave goes through its columns in rising order from one
// chunk to the next, so there a value must pass the key's; within a chunk it does not.
struct Best {
  uint64_t* keys;
  int count;
  uint64_t key;
  __device__ __forceinline__ float least() const { return value_of((uint32_t)(key >> 32)); }
};

// cuts the keys back to the best `top`, the best first
__device__ __forceinline__ void cut(Best& b, int top, int lane) {
  wave_lds_fence();
  const uint64_t k0 = lane < b.count ? b.keys[lane] : 0, k1 = lane + 64 < b.count ? b.keys[lane + 64] : 0;
  const int n = (b.count + 7) & -8;
  if (lane < n - b.count) b.keys[b.count + lane] = 0;
  wave_lds_fence();
  int r0, r1;
  ranks_of(k0, k1, b.keys, n, r0, r1);
  wave_lds_fence();
  if (lane < b.count && r0 < top) b.keys[r0] = k0;
  if (lane + 64 < b.count && r1 < top) b.keys[r1] = k1;
  wave_lds_fence();
  if (b.count >= top) {
    b.count = top;
    b.key = b.keys[top - 1];
  }
}

__device__ __forceinline__ void offer(Best& b, float z, int32_t column, int top, int lane) {
  const uint64_t key = key_of(z, column);
  if (!__any(key > b.key)) return;
  if (b.count > kHeldKeys - 64) cut(b, top, lane);
  const bool passes = key > b.key;
  const unsigned long long who = __ballot(passes);
  const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u));
  if (passes) b.keys[b.count + before] = key;
  b.count += __builtin_popcountll(who);
}

// a little below the `top`-th largest of the lanes' values; keys: 64 of scratch
__device__ __forceinline__ uint64_t first_key(float z, uint64_t* keys, int top, int lane) {
  const uint64_t key = key_of(z, lane);
  keys[lane] = key;
  wave_lds_fence();
  int r, none;
  ranks_of(key, ~0ull, keys, 64, r, none);
  wave_lds_fence();
  const unsigned long long who = __ballot(r == top - 1);
  const float at = __shfl(z, __builtin_ctzll(who));
  const float below = at - fmaxf(fabsf(at) * 1e-6f, 1e-30f);
  return key_of(below > kFloor ? below : kFloor, 0);  // kFloor also where `at` is NaN
}

// What is known of a row: m, s and t as above; m is at least kFloor.
struct Sums {
  float m, s, t;
};

// What differences to m count from, log2 units: d = (z - a) factor - b.  With a = 0 and b the rounded product of
// m with the factor, d is one FMA of the logit; what the rounding adds to every d alike cancels, since the
// sums, what is taken from them and the gradient count from the same number.  Past 2^24 it may be more than
// 1 / 2, and a is m, b 0.
struct Origin {
  float a, b;
  __device__ __forceinline__ bool large() const { return a != 0.f; }  // true for a NaN too
  // below kLeast for a masked logit unless large()
  __device__ __forceinline__ float to(float z, float factor) const { return fmaf(z - a, factor, -b); }
  // how far it is past m's product itself, exact: what a row's sum in memory no longer has
  __device__ __forceinline__ float past(float m, float factor) const { return fmaf(a - m, factor, b); }
};
constexpr float kLargeProduct = 16777216.f;

__device__ __forceinline__ Origin origin_of(float m, float factor) {
  float p = m * factor;
  // Rounded here: of a difference of two such products the compiler would make one product and an FMA with
  // the other unrounded, for an unchanged maximum not 0 but the product's rounding error, by which the
  // sums would drift with every tile.
  asm("" : "+v"(p));
  return fabsf(p) < kLargeProduct ? Origin{0.f, p} : Origin{m, 0.f};
}

// Counts the sums, so far from `at`, from a maximum m on.
__device__ __forceinline__ void raise(Sums& a, Origin& at, float m, float factor) {
  const Origin to = origin_of(m, factor);
  const float d = fminf(fmaf(to.a - at.a, factor, to.b - at.b), -kLeast);
  const float c = exp2_of(-d);
  a.t = c * fmaf(-d, a.s, a.t);
  a.s *= c;
  a.m = m;
  at = to;
}

__device__ __forceinline__ void raise(Sums& a, float m, float factor) {
  Origin at = origin_of(a.m, factor);
  raise(a, at, m, factor);
}

__device__ __forceinline__ Sums wave_join(Sums a, float factor) {
  raise(a, wave_max(a.m), factor);
  a.s = wave_sum(a.s);
  a.t = wave_sum(a.t);
  return a;
}

// whether a row's results are NaN, and whether it has nothing but masked logits
__device__ __forceinline__ bool is_broken(const Sums& a) { return !(a.m < INFINITY); }
__device__ __forceinline__ bool is_empty(const Sums& a) { return a.m <= kFloor; }

__device__ __forceinline__ float log_prob(const RowsArgs& a, float z, const Sums& sums, float log_s) {
  const float d = origin_of(sums.m, a.factor).to(z, a.factor);
  // differences past fp32's range in log2 units alone
  return d > -1e37f ? (d - log_s) * kLn2 : (z - sums.m) * a.scale;
}

// The row's outputs but for the alternatives; every thread has the sums.
template <typename T>
__device__ __forceinline__ void write_row(const RowsArgs& a, int row, const Sums& sums, int tid) {
  const bool broken = is_broken(sums), empty = is_empty(sums);
  const float log_s = __log2f(sums.s);
  if (tid < a.num_tokens) {
    const int32_t tok = a.tokens[(int64_t)row * a.num_tokens + tid];
    float lp = 0.f;
    if (tok >= a.vocab) {
      lp = NAN;
    } else if (tok >= 0) {
      const float z = value<T>(reinterpret_cast<const T*>(a.logits) + (int64_t)row * a.stride, tok);
      lp = broken ? NAN : empty || z <= kFloor ? -INFINITY : log_prob(a, z, sums, log_s);
    }
    a.token_logp[(int64_t)row * a.num_tokens + tid] = lp;
  }
  if (tid == 0) {
    if (a.entropy != nullptr)
      a.entropy[row] = broken ? NAN : empty ? 0.f : kLn2 * (log_s - sums.t / sums.s);
    if (a.stats != nullptr) {
      const float s = sums.s * exp2_of(origin_of(sums.m, a.factor).past(sums.m, a.factor));
      reinterpret_cast<float2*>(a.stats)[row] = broken ? make_float2(NAN, NAN) : make_float2(sums.m, empty ? 0.f : s);
    }
  }
}

// The alternatives among keys[0 .. n) in LDS, n a multiple of 8; 0 is none.  Places past the
// last alternative have been filled by fill_top.
__device__ __forceinline__ void write_top(const RowsArgs& a, int row, const Sums& sums, const uint64_t* keys, int n,
                                          int tid) {
  if (is_broken(sums)) return;
  const float log_s = __log2f(sums.s);
  const int64_t at = (int64_t)row * a.top;
  for (int i = tid; i < n; i += 2 * kThreads) {
    const uint64_t k0 = keys[i], k1 = i + kThreads < n ? keys[i + kThreads] : 0;
    int r0, r1;
    ranks_of(k0, k1, keys, n, r0, r1);
    auto put = [&](uint64_t key, int r) {
      if (key == 0 || r >= a.top) return;
      a.top_tokens[at + r] = (int32_t) ~(uint32_t)key;
      a.top_logp[at + r] = log_prob(a, value_of((uint32_t)(key >> 32)), sums, log_s);
    };
    put(k0, r0);
    put(k1, r1);
  }
}

// the places that `there` alternatives leave
__device__ __forceinline__ void fill_top(const RowsArgs& a, int row, const Sums& sums, int there, int tid) {
  const bool broken = is_broken(sums);
  if (broken) there = 0;
  if (tid >= there && tid < a.top) {
    a.top_tokens[(int64_t)row * a.top + tid] = -1;
    a.top_logp[(int64_t)row * a.top + tid] = broken ? NAN : -INFINITY;
  }
}

__device__ __forceinline__ void write_masked(const RowsArgs& a, int row, int tid) {
  if (tid < a.num_tokens) a.token_logp[(int64_t)row * a.num_tokens + tid] = 0.f;
  if (tid < a.top) {
    a.top_tokens[(int64_t)row * a.top + tid] = -1;
    a.top_logp[(int64_t)row * a.top + tid] = 0.f;
  }
  if (tid == 0) {
    if (a.entropy != nullptr) a.entropy[row] = 0.f;
    if (a.stats != nullptr) reinterpret_cast<float2*>(a.stats)[row] = make_float2(0.f, 0.f);
  }
}

template <typename T, bool kTop, bool kEntropy>
__global__ __launch_bounds__(kThreads) void logprob_kernel(RowsArgs a) {
  constexpr int kElems = kChunkOf<T>;
  __shared__ Sums lds_sums[kWaves];
  __shared__ __attribute__((aligned(16))) uint64_t lds_keys[kTop ? kWaves * kHeldKeys : 1];
  __shared__ __attribute__((aligned(16))) uint64_t lds_best[kTop ? kWaves * kMostTop : 1];
  __shared__ int lds_there[kWaves];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = (int)blockIdx.x / a.splits;
  const int split = (int)blockIdx.x - row * a.splits;
  if (a.mask != nullptr && a.mask[row] == 0) {
    if (a.splits == 1) write_masked(a, row, tid);
    return;
  }
  const float factor = a.factor;
  // the row's chunks in shares of whole tiles
  const int chunks = (a.vocab + kElems - 1) / kElems;
  const int tiles = (chunks + kTileChunks - 1) / kTileChunks;
  const int per = (tiles + a.splits - 1) / a.splits;
  const int until = split * per + per < tiles ? split * per + per : tiles;
  const __amdgpu_buffer_rsrc_t rsrc =
      row_rsrc(reinterpret_cast<const T*>(a.logits) + (int64_t)row * a.stride, row_bytes<T>(a.vocab));

  Sums sums{kFloor, 0.f, 0.f};
  Origin at = origin_of(kFloor, factor);
  Best best{lds_keys + (kTop ? wave * kHeldKeys : 0), 0, 0};
  bool fresh = true;
  u32x4 next[kTileLoads];
  auto fetch = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < kTileLoads; ++r) next[r] = load_chunk(rsrc, (tile * kTileChunks + r * 64 + lane) * 16);
  };
  int tile = split * per + wave;
  if (tile < until) fetch(tile);
  for (; tile < until; tile += kWaves) {
    u32x4 x[kTileLoads];
#pragma unroll
    for (int r = 0; r < kTileLoads; ++r) x[r] = next[r];
    if (tile + kWaves < until) fetch(tile + kWaves);
    const int first = tile * kTileChunks * kElems;
    if (first + kTileChunks * kElems > a.vocab) {  // past the vocabulary: masked
#pragma unroll
      for (int r = 0; r < kTileLoads; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c = first + (r * 64 + lane) * kElems + i * (kElems / 4);
          if constexpr (sizeof(T) == 2) {
            if (c >= a.vocab) x[r][i] = 0xff80ff80u;
            else if (c + 1 >= a.vocab) x[r][i] = (x[r][i] & 0xffffu) | 0xff800000u;
          } else {
            if (c >= a.vocab) x[r][i] = 0xff800000u;
          }
        }
    }
    float most[kTileLoads];
#pragma unroll
    for (int r = 0; r < kTileLoads; ++r) {
      float z[kElems];
      unpack<T>(x[r], z);
      most[r] = z[0];
#pragma unroll
      for (int e = 1; e < kElems; ++e) most[r] = max_of(most[r], z[e]);
    }
    const float top = max_of(max_of(most[0], most[1]), max_of(most[2], most[3]));
    raise(sums, at, max_of(sums.m, top), factor);
    if constexpr (kTop) {
      if (fresh) best.key = first_key(top, best.keys, a.top, lane);
      fresh = false;
      const bool some = __any(top > best.least());
#pragma unroll
      for (int r = 0; r < kTileLoads; ++r) {
        if (!some || !__any(most[r] > best.least())) continue;
        float z[kElems];
        unpack<T>(x[r], z);
        const int c = first + (r * 64 + lane) * kElems;
#pragma unroll
        for (int e = 0; e < kElems; ++e) offer(best, z[e], c + e, a.top, lane);
      }
    }
    // The sums of a tile.  A masked logit's d of -inf would make t NaN, which the lanes of such
    // tiles have and take the sums again with d bounded; the others save a bound per logit (4,301 whole rows
    // 211 us, 262 with one in 64 masked, 207 either way without the entropy).  In waves with a lane whose
    // product is large, as of one that has met masked logits alone, each takes its own differences.
    auto add = [&](auto large, auto bounded, float& s, float& t) __attribute__((always_inline)) {
#pragma unroll
      for (int r = 0; r < kTileLoads; ++r) {
        float z[kElems];
        unpack<T>(x[r], z);
#pragma unroll
        for (int e = 0; e < kElems; ++e) {
          float d = large ? at.to(z[e], factor) : fmaf(z[e], factor, -at.b);
          if (bounded) d = fmaxf(d, kLeast);
          if (large) d = z[e] <= kFloor ? kLeast : d;
          const float w = exp2_of(d);
          s += w;
          if (kEntropy) t = fmaf(w, d, t);
        }
      }
    };
    float s = 0.f, t = 0.f;
    const std::true_type yes;
    const std::false_type no;
    if (!__any(at.large())) {
      add(no, no, s, t);
      if (kEntropy && __any(t != t)) {
        s = t = 0.f;
        add(no, yes, s, t);
      }
    } else {
      add(yes, yes, s, t);
    }
    sums.s += s;
    sums.t += t;
  }

  sums = wave_join(sums, factor);
  if (lane == 0) lds_sums[wave] = sums;
  if constexpr (kTop) {
    cut(best, a.top, lane);
    if (lane < round8(a.top)) lds_best[wave * round8(a.top) + lane] = lane < best.count ? best.keys[lane] : 0;
    if (lane == 0) lds_there[wave] = best.count;
  }
  __syncthreads();
  float m = lds_sums[0].m;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) m = max_of(m, lds_sums[w].m);
  Sums all{m, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    Sums one = lds_sums[w];
    raise(one, m, factor);
    all.s += one.s;
    all.t += one.t;
  }
  if (a.splits == 1) {
    write_row<T>(a, row, all, tid);
    if constexpr (kTop) {
      int there = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) there += lds_there[w];
      fill_top(a, row, all, there, tid);
      write_top(a, row, all, lds_best, kWaves * round8(a.top), tid);
    }
    return;
  }
  if (tid == 0) a.part[(int64_t)row * a.splits + split] = make_float4(all.m, all.s, all.t, 0.f);
  if constexpr (kTop) {
    // the share's best, in order
    uint64_t* const out = a.keys + ((int64_t)row * a.splits + split) * a.top;
    int there = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) there += lds_there[w];
    if (tid >= there && tid < a.top) out[tid] = 0;
    const int n = kWaves * round8(a.top);  // up to a key per thread
    const uint64_t key = tid < n ? lds_best[tid] : 0;
    int r, none;
    ranks_of(key, ~0ull, lds_best, n, r, none);
    if (key != 0 && r < a.top) out[r] = key;
  }
}

// Joins a row's shares: one workgroup per row, a share per lane.  Of the shares' alternatives, each
// share's in order, only those are compared with each other that reach a key which `top` of
// them reach: with p = ceil(top / shares), the least of the shares' p-th ones, or the largest of
// their last.
template <typename T, bool kTop>
__global__ __launch_bounds__(kThreads) void logprob_merge_kernel(RowsArgs a) {
  __shared__ __attribute__((aligned(16))) uint64_t lds_best[kTop ? kMostSplits * kMostTop + 8 : 1];
  __shared__ int lds_count;
  const int tid = threadIdx.x, lane = tid & 63;
  const int row = blockIdx.x;
  if (a.mask != nullptr && a.mask[row] == 0) return write_masked(a, row, tid);
  const int64_t at = (int64_t)row * a.splits;
  Sums sums{kFloor, 0.f, 0.f};
  uint64_t enough = 0, last = 0;
  if (lane < a.splits) {
    const float4 p = a.part[at + lane];
    sums = Sums{p.x, p.y, p.z};
    if constexpr (kTop) {
      const uint64_t* const keys = a.keys + (at + lane) * a.top;
      enough = keys[(a.top + a.splits - 1) / a.splits - 1];
      last = keys[a.top - 1];
    }
  }
  sums = wave_join(sums, a.factor);
  write_row<T>(a, row, sums, tid);
  if constexpr (kTop) {
    if (lane >= a.splits) enough = ~0ull;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
      const uint64_t e = __shfl_xor(enough, off), l = __shfl_xor(last, off);
      enough = e < enough ? e : enough;
      last = l > last ? l : last;
    }
    const uint64_t least = enough > last ? enough : last;
    if (tid == 0) lds_count = 0;
    __syncthreads();
    const int n = a.splits * a.top;
    for (int base = 0; base < n; base += kThreads) {
      const uint64_t key = base + tid < n ? a.keys[at * a.top + base + tid] : 0;
      if (key != 0 && key >= least) lds_best[atomicAdd(&lds_count, 1)] = key;  // in any order
    }
    __syncthreads();
    const int there = lds_count;
    if (tid < 8) lds_best[there + tid] = 0;
    __syncthreads();
    fill_top(a, row, sums, there, tid);
    write_top(a, row, sums, lds_best, (there + 7) & -8, tid);
  }
}

// ------------------------------------------------------------------ gradient

struct GradArgs {
  const void* logits;
  void* grad;
  int64_t stride, grad_stride;
  int32_t vocab, splits;
  const int32_t* tokens;
  int32_t num_tokens;
  const uint8_t* mask;
  float factor, scale;
  const float *stats, *entropy, *grad_logp, *grad_entropy;
};

__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
  bf16x2 v = {(__bf16)a, (__bf16)b};  // round to nearest even
  return __builtin_bit_cast(uint32_t, v);
}

template <typename T, bool kEntropy>
__global__ __launch_bounds__(kThreads) void logprob_grad_kernel(GradArgs a) {
  constexpr int kElems = kChunkOf<T>;
  __shared__ int32_t lds_tokens[kMostTokens];
  __shared__ float lds_by[kMostTokens];
  const int tid = threadIdx.x;
  const int row = (int)blockIdx.x / a.splits;
  const int split = (int)blockIdx.x - row * a.splits;
  const int whole = a.vocab / kElems;
  const int chunks = (a.vocab + kElems - 1) / kElems;
  const int per = (chunks + a.splits - 1) / a.splits;
  const int from = split * per, until = from + per < chunks ? from + per : chunks;
  const T* const src = reinterpret_cast<const T*>(a.logits) + (int64_t)row * a.stride;
  T* const dst = reinterpret_cast<T*>(a.grad) + (int64_t)row * a.grad_stride;
  const bool live = a.mask == nullptr || a.mask[row] != 0;
  float2 st = make_float2(0.f, 0.f);
  float by = 0.f, by_h = 0.f, any = 0.f;
  if (live) {
    st = reinterpret_cast<const float2*>(a.stats)[row];
    if (tid < a.num_tokens) {
      const int32_t tok = a.tokens[(int64_t)row * a.num_tokens + tid];
      const bool given = tok >= 0 && tok < a.vocab;
      lds_tokens[tid] = given ? tok : -1;
      lds_by[tid] = given ? a.grad_logp[(int64_t)row * a.num_tokens + tid] : 0.f;
    }
    if (kEntropy) by_h = a.grad_entropy[row];
    __syncthreads();
    for (int i = 0; i < a.num_tokens; ++i) {
      by += lds_by[i];
      any = lds_by[i] != 0.f ? 1.f : any;  // a NaN too
    }
  }
  // p (c0 + c1 log2 p) with log2 p = d - log2 s:  -scale p (by + by_h (ln p + entropy))
  const Origin at = origin_of(st.x, a.factor);
  const bool large = at.large();
  const float log_s = __log2f(st.y) - at.past(st.x, a.factor);
  const float h = kEntropy && live ? a.entropy[row] : 0.f;
  const float c0 = st.x == st.x ? -a.scale * (kEntropy ? fmaf(by_h, h, by) : by) : NAN;
  const float c1 = kEntropy ? -a.scale * by_h * kLn2 : 0.f;
  // log2 of a probability
  auto log2_p = [&](float z) __attribute__((always_inline)) {
    if (large) return z <= kFloor ? kLeast : fmaxf(at.to(z, a.factor) - log_s, kLeast);
    return fmaxf(fmaf(z, a.factor, -at.b) - log_s, kLeast);
  };
  auto weight = [&](float z) __attribute__((always_inline)) {
    const float d = log2_p(z);
    return exp2_of(d) * (kEntropy ? fmaf(c1, d, c0) : c0);
  };
  const bool zero = !live || st.y == 0.f || (any == 0.f && by_h == 0.f);
  const __amdgpu_buffer_rsrc_t rs = row_rsrc(src, zero ? 0u : row_bytes<T>(a.vocab));
  const __amdgpu_buffer_rsrc_t rd = row_rsrc(dst, (uint32_t)whole * 16u);
  for (int c0i = from; c0i < until; c0i += kTileLoads * kThreads) {
    u32x4 x[kTileLoads];
#pragma unroll
    for (int r = 0; r < kTileLoads; ++r) x[r] = load_chunk(rs, (c0i + r * kThreads + tid) * 16);
#pragma unroll
    for (int r = 0; r < kTileLoads; ++r) {
      const int c = c0i + r * kThreads + tid;
      u32x4 o = {0u, 0u, 0u, 0u};
      if (!zero) {
        float z[kElems];
        unpack<T>(x[r], z);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (sizeof(T) == 2)
            o[i] = pack_bf16x2(weight(z[2 * i]), weight(z[2 * i + 1]));
          else
            o[i] = __float_as_uint(weight(z[i]));
        }
      }
      if (c >= until) continue;
      if (c < whole) {
        __builtin_amdgcn_raw_buffer_store_b128(o, rd, c * 16, 0, kNonTemporal);
      } else {  // the partial chunk: its columns below vocab
        for (int e = 0; e < a.vocab - whole * kElems; ++e) {
          if constexpr (sizeof(T) == 2)
            dst[(int64_t)whole * kElems + e] = (T)(e & 1 ? o[e >> 1] >> 16 : o[e >> 1] & 0xffffu);
          else
            dst[(int64_t)whole * kElems + e] = __uint_as_float(o[e]);
        }
      }
    }
  }
  if (zero || a.num_tokens == 0) return;
  // the given tokens of this share: their entries written again, after the share's stores have arrived
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  if (tid < a.num_tokens) {
    const int32_t tok = lds_tokens[tid];
    if (tok >= 0 && tok / kElems >= from && tok / kElems < until) {
      float own = 0.f;  // of every place that names the token; each of their threads writes the same
      for (int i = 0; i < a.num_tokens; ++i) own += lds_tokens[i] == tok ? lds_by[i] : 0.f;
      const float g = fmaf(a.scale, own, weight(value<T>(src, tok)));
      if constexpr (sizeof(T) == 2)
        dst[tok] = (T)(pack_bf16x2(g, g) & 0xffffu);
      else
        dst[tok] = g;
    }
  }
}

// ------------------------------------------------------------------ host

int fail(int code, const char* fmt, ...) {
  char msg[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(msg, sizeof msg, fmt, ap);
  va_end(ap);
  return ctx_report_error(code, msg);
}

bool aligned16(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0; }

int chunk_of(ctx_dtype dtype) { return dtype == CTX_DTYPE_BF16 ? kChunkOf<uint16_t> : kChunkOf<float>; }

int check_shape(ctx_dtype dtype, int32_t vocab, int32_t num_rows) {
  if (dtype != CTX_DTYPE_BF16 && dtype != CTX_DTYPE_F32) return fail(CTX_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
  if (vocab <= 0) return fail(CTX_ERR_INVALID_ARG, "vocab %d <= 0", vocab);
  if (vocab > kMostVocab) return fail(CTX_ERR_UNSUPPORTED, "vocab %d > %d", vocab, kMostVocab);
  if (num_rows < 0) return fail(CTX_ERR_INVALID_ARG, "num_rows %d < 0", num_rows);
  if (num_rows > kMostGroups) return fail(CTX_ERR_UNSUPPORTED, "num_rows %d > %d", num_rows, kMostGroups);
  return CTX_OK;
}

int check_top(int32_t top) {
  if (top < 0) return fail(CTX_ERR_INVALID_ARG, "top %d < 0", top);
  if (top > kMostTop) return fail(CTX_ERR_UNSUPPORTED, "top %d > %d", top, kMostTop);
  return CTX_OK;
}

int check_rows(const char* name, ctx_dtype dtype, int64_t stride, int32_t vocab) {
  if (stride < vocab || stride % chunk_of(dtype) != 0)
    return fail(CTX_ERR_INVALID_ARG, "%s %lld must be >= vocab and a multiple of %d", name, (long long)stride,
                chunk_of(dtype));
  return CTX_OK;
}

int check_tokens(const int32_t* tokens, int32_t num_tokens) {
  if (num_tokens < 0) return fail(CTX_ERR_INVALID_ARG, "num_tokens %d < 0", num_tokens);
  if (num_tokens > kMostTokens) return fail(CTX_ERR_UNSUPPORTED, "num_tokens %d > %d", num_tokens, kMostTokens);
  if ((num_tokens > 0) != (tokens != nullptr))
    return fail(CTX_ERR_INVALID_ARG, "tokens and a positive num_tokens go together");
  return CTX_OK;
}

// Whether two arrays of rows of `width` bytes share any: rows of equal strides may lie between each
// other's.
bool rows_overlap(const void* p, int64_t p_stride, const void* q, int64_t q_stride, int64_t width, int64_t rows) {
  const int64_t a = (int64_t)reinterpret_cast<uintptr_t>(p), b = (int64_t)reinterpret_cast<uintptr_t>(q);
  if (a + (rows - 1) * p_stride + width <= b || b + (rows - 1) * q_stride + width <= a) return false;
  if (p_stride != q_stride || rows == 1) return true;
  const int64_t off = ((b - a) % p_stride + p_stride) % p_stride;
  return off < width || off + width > p_stride;
}

int check_scale(float scale) {
  if (!(scale >= 1e-30f && scale <= 1e30f)) return fail(CTX_ERR_INVALID_ARG, "scale must be in [1e-30, 1e30]");
  return CTX_OK;
}

int query_cus(int* cus) {
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e == hipSuccess) e = hipDeviceGetAttribute(cus, hipDeviceAttributeMultiprocessorCount, device);
  if (e != hipSuccess) return fail(CTX_ERR_HIP, "device query: %s", hipGetErrorString(e));
  return CTX_OK;
}

// Workgroups that share a row: kPerCu of them per CU in all, a tile per wave at least.
constexpr int kPerCu = 8;

int32_t splits_of(ctx_dtype dtype, int32_t vocab, int32_t rows, int cus) {
  const int64_t tiles = ((int64_t)vocab + chunk_of(dtype) * kTileChunks - 1) / (chunk_of(dtype) * kTileChunks);
  const int64_t want = (kPerCu * (int64_t)cus + rows - 1) / rows;
  int64_t s = tiles / kWaves;
  s = s < want ? s : want;
  s = s < kMostSplits ? s : kMostSplits;
  return s < 1 ? 1 : (int32_t)s;
}

size_t workspace_of(int32_t rows, int32_t splits, int32_t top) {
  return splits == 1 ? 0 : (size_t)rows * splits * (sizeof(float4) + sizeof(uint64_t) * (size_t)top);
}

template <typename T, bool kTop>
void launch_rows(const RowsArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.rows * (unsigned)a.splits), block(kThreads);
  if (a.entropy != nullptr)
    hipLaunchKernelGGL((logprob_kernel<T, kTop, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((logprob_kernel<T, kTop, false>), grid, block, 0, s, a);
  if (a.splits > 1) hipLaunchKernelGGL((logprob_merge_kernel<T, kTop>), dim3((unsigned)a.rows), block, 0, s, a);
}

}  // namespace

extern "C" int ctx_token_logprob_workspace(ctx_dtype dtype, int32_t vocab, int32_t num_rows, int32_t top,
                                           size_t* bytes) {
  ctx_clear_error();
  if (bytes == nullptr) return fail(CTX_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = 0;
  int rc = check_shape(dtype, vocab, num_rows);
  if (rc == CTX_OK) rc = check_top(top);
  if (rc != CTX_OK || num_rows == 0) return rc;
  int cus = 0;
  if ((rc = query_cus(&cus)) != CTX_OK) return rc;
  *bytes = workspace_of(num_rows, splits_of(dtype, vocab, num_rows, cus), top);
  return CTX_OK;
}

extern "C" int ctx_token_logprob_run(const void* logits, ctx_dtype dtype, int64_t row_stride, int32_t vocab,
                                     const int32_t* tokens, int32_t num_tokens, const uint8_t* mask, int32_t num_rows,
                                     float scale, int32_t top, float* token_logp, float* entropy, float* stats,
                                     int32_t* top_tokens, float* top_logp, void* workspace, size_t workspace_bytes,
                                     void* stream) {
  ctx_clear_error();
  int rc = check_shape(dtype, vocab, num_rows);
  if (rc == CTX_OK) rc = check_top(top);
  if (rc == CTX_OK) rc = check_rows("row_stride", dtype, row_stride, vocab);
  if (rc == CTX_OK) rc = check_scale(scale);
  if (rc != CTX_OK) return rc;
  if (num_rows == 0) return CTX_OK;
  if ((rc = check_tokens(tokens, num_tokens)) != CTX_OK) return rc;
  if (logits == nullptr) return fail(CTX_ERR_INVALID_ARG, "logits is NULL");
  if ((num_tokens > 0) != (token_logp != nullptr))
    return fail(CTX_ERR_INVALID_ARG, "token_logp and a positive num_tokens go together");
  if ((top > 0) != (top_tokens != nullptr) || (top > 0) != (top_logp != nullptr))
    return fail(CTX_ERR_INVALID_ARG, "top_tokens, top_logp and a positive top go together");
  if (!aligned16(logits) || !aligned16(workspace))
    return fail(CTX_ERR_ALIGNMENT, "logits and workspace must be 16-byte aligned");
  int cus = 0;
  if ((rc = query_cus(&cus)) != CTX_OK) return rc;
  const int32_t splits = splits_of(dtype, vocab, num_rows, cus);
  const size_t need = workspace_of(num_rows, splits, top);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need))
    return fail(CTX_ERR_CAPACITY, "workspace of %zu bytes, %zu needed", workspace == nullptr ? 0 : workspace_bytes, need);
  RowsArgs a{};
  a.logits = logits;
  a.stride = row_stride;
  a.vocab = vocab;
  a.rows = num_rows;
  a.splits = splits;
  a.tokens = tokens;
  a.num_tokens = num_tokens;
  a.mask = mask;
  a.scale = scale;
  a.factor = (float)((double)scale * 1.4426950408889634);
  a.top = top;
  a.token_logp = token_logp;
  a.entropy = entropy;
  a.stats = stats;
  a.top_tokens = top_tokens;
  a.top_logp = top_logp;
  a.part = static_cast<float4*>(workspace);
  a.keys = reinterpret_cast<uint64_t*>(a.part + (size_t)num_rows * splits);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (dtype == CTX_DTYPE_BF16)
    top > 0 ? launch_rows<uint16_t, true>(a, s) : launch_rows<uint16_t, false>(a, s);
  else
    top > 0 ? launch_rows<float, true>(a, s) : launch_rows<float, false>(a, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(CTX_ERR_HIP, "kernel launch: %s", hipGetErrorString(e));
  return CTX_OK;
}

extern "C" int ctx_token_logprob_grad_run(const void* logits, ctx_dtype dtype, int64_t row_stride, int32_t vocab,
                                          const int32_t* tokens, int32_t num_tokens, const uint8_t* mask,
                                          int32_t num_rows, float scale, const float* stats, const float* entropy,
                                          const float* grad_logp, const float* grad_entropy, void* grad_logits,
                                          int64_t grad_row_stride, void* stream) {
  ctx_clear_error();
  int rc = check_shape(dtype, vocab, num_rows);
  if (rc == CTX_OK) rc = check_rows("row_stride", dtype, row_stride, vocab);
  if (rc == CTX_OK) rc = check_rows("grad_row_stride", dtype, grad_row_stride, vocab);
  if (rc == CTX_OK) rc = check_scale(scale);
  if (rc != CTX_OK) return rc;
  if (num_rows == 0) return CTX_OK;
  if ((rc = check_tokens(tokens, num_tokens)) != CTX_OK) return rc;
  if (logits == nullptr || stats == nullptr || grad_logits == nullptr)
    return fail(CTX_ERR_INVALID_ARG, "NULL logits, stats or grad_logits");
  if ((num_tokens > 0) != (grad_logp != nullptr))
    return fail(CTX_ERR_INVALID_ARG, "grad_logp and a positive num_tokens go together");
  if ((grad_entropy != nullptr) != (entropy != nullptr))
    return fail(CTX_ERR_INVALID_ARG, "entropy and grad_entropy must both be given or both be NULL");
  if (!aligned16(logits) || !aligned16(grad_logits))
    return fail(CTX_ERR_ALIGNMENT, "logits and grad_logits must be 16-byte aligned");
  const int64_t size = 16 / chunk_of(dtype);
  if (rows_overlap(logits, row_stride * size, grad_logits, grad_row_stride * size, vocab * size, num_rows))
    return fail(CTX_ERR_INVALID_ARG, "grad_logits overlaps the logits");
  GradArgs a{};
  a.logits = logits;
  a.grad = grad_logits;
  a.stride = row_stride;
  a.grad_stride = grad_row_stride;
  a.vocab = vocab;
  a.tokens = tokens;
  a.num_tokens = num_tokens;
  a.mask = mask;
  a.factor = (float)((double)scale * 1.4426950408889634);
  a.scale = scale;
  a.stats = stats;
  a.entropy = entropy;
  a.grad_logp = grad_logp;
  a.grad_entropy = grad_entropy;
  // A workgroup per tile of a row: all of them at work at once read and write near each other, as
  // a copy does (2,057 rows of 151,936 bf16 logits 195 us, with 4 workgroups per row 250; smaller
  // tiles gain nothing: half 203).
  const int64_t chunks = (vocab + chunk_of(dtype) - 1) / chunk_of(dtype);
  const int64_t tiles = (chunks + kTileLoads * kThreads - 1) / (kTileLoads * kThreads);
  const int64_t most = kMostGroups / num_rows;
  a.splits = (int32_t)(tiles < most ? tiles : most);
  const dim3 grid((unsigned)num_rows * (unsigned)a.splits), block(kThreads);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (dtype == CTX_DTYPE_BF16) {
    if (grad_entropy != nullptr)
      hipLaunchKernelGGL((logprob_grad_kernel<uint16_t, true>), grid, block, 0, s, a);
    else
      hipLaunchKernelGGL((logprob_grad_kernel<uint16_t, false>), grid, block, 0, s, a);
  } else {
    if (grad_entropy != nullptr)
      hipLaunchKernelGGL((logprob_grad_kernel<float, true>), grid, block, 0, s, a);
    else
      hipLaunchKernelGGL((logprob_grad_kernel<float, false>), grid, block, 0, s, a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(CTX_ERR_HIP, "kernel launch: %s", hipGetErrorString(e));
  return CTX_OK;
}
