// ctx_paged_common.h -- device helpers shared by the attention over paged caches whose blocks
// go straight from memory into LDS (causal prefill in ctx_prefill_paged.hip, drafted trees in
// ctx_tree_attn.hip).  Internal: not part of the C ABI.
#ifndef CTX_PAGED_COMMON_H_
#define CTX_PAGED_COMMON_H_

#include "ctx_attn_common.h"

namespace {

typedef __attribute__((address_space(3))) void lds_void;

// s_waitcnt vmcnt(n) with expcnt and lgkmcnt left open
constexpr int wait_vmcnt(int n) { return 0x0F70 | (n & 15) | ((n >> 4) << 14); }

// Quotients of 0 <= x < 2^31 by d > 0, exact: with 2^(shift - 1) < d <= 2^shift the factor's
// excess over 2^(31 + shift) / d is less than 1, which x / 2^31 of cannot carry the
// quotient over the next whole number.  (Three instructions where a division takes 30, and
// a workgroup has a dozen before its first block.)
struct Divisor {
  int32_t d;
  uint32_t factor;
  int32_t shift;
  Divisor() = default;
  explicit Divisor(int32_t by) : d(by), shift(0) {
    while (((int64_t)1 << shift) < by) ++shift;
    factor = (uint32_t)((((uint64_t)1 << (31 + shift)) + by - 1) / by);
  }
  __device__ __forceinline__ int of(int x) const { return (int)(__umulhi((uint32_t)x << 1, factor) >> shift); }
};

// Workgroup barrier with no memory fence: the caller has already waited for its own
// loads into LDS that the other waves will read, and a fence would also wait for the
// loads of later blocks still in flight.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_barrier" ::: "memory"); }

// 16 bytes per lane from voff in r straight to LDS base + 16 * lane
template <int kPolicy>
__device__ __forceinline__ void load16_to_lds(__amdgpu_buffer_rsrc_t r, uint16_t* base, int voff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)base, 16, voff, 0, 0, kPolicy);
}

// NaN-propagating maximum of 8, which gfx950 has as a three-input instruction
__device__ __forceinline__ float max8(f32x4 a, f32x4 b) {
  const auto mx = [](float x, float y) { return __builtin_elementwise_maximum(x, y); };
  return mx(mx(mx(mx(a[0], a[1]), a[2]), mx(mx(a[3], b[0]), b[1])), mx(b[2], b[3]));
}

// the largest of a column, whose tokens are spread over the 4 rows of 16 lanes
__device__ __forceinline__ float column_max(float x) {
  const uint32_t a = __float_as_uint(x);
  const auto rows = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  const uint32_t b = __float_as_uint(fmaxf(__uint_as_float(rows[0]), __uint_as_float(rows[1])));
  const auto halves = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return fmaxf(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
}

}  // namespace

#endif  // CTX_PAGED_COMMON_H_
