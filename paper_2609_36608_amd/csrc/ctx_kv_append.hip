// ctx_kv_append.hip -- append of new keys and values to paged caches for gfx950
// (MI355X), with the head norm and the rotation of positions on the way, behind
// ctx_kv_append_run_paged in the C ABI declared in include/ctx_paged_attn.h.
//
// Per packed row (one new token): Hq query, Hkv key and Hkv value heads of 128
// bf16 are read once and written once, so the work is bound by HBM for many rows
// (30,629 rows of 32/8 heads 136 us, 5.5 TB/s: the copy rate) and by latency for a
// few (4 rows of 16/8 heads 4.0 us, 256 of 32/8 5.6).
//
//   * 16 lanes hold one head, 8 dimensions (16 bytes) each; a wave instruction
//     moves 4 heads.  A row's heads are numbered queries, keys, values; which of
//     the three a lane has only chooses its addresses and its weights.
//   * Norm: sum of squares over the 16 lanes by rotations of the row of lanes.
//   * Rotation: pairs (i, i + R/2) are R/16 lanes apart (R a multiple of 16), one
//     lane move per word; interleaved pairs are in the lane.  The angles of a row
//     are its position times inv_freq for all heads: lane i of the wave finds
//     angle i, in turns and reduced to half a turn in fp64 (the product's 55 bits
//     would lose a far position's angle in fp32), and passes cosine and sine on
//     through the wave's piece of LDS.
//   * All arithmetic between is fp32; one rounding to bf16 (nearest even).

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "ctx_attn_common.h"
#include "ctx_paged_attn.h"

namespace {

constexpr int kWaves = 4;         // per workgroup
constexpr int kLaneDims = 8;      // dimensions per lane
constexpr int kHeadLanes = kHeadDim / kLaneDims;
constexpr int kPassHeads = 64 / kHeadLanes;
constexpr int kAngles = kHeadDim / 2;  // most per row

struct AppendArgs {
  const uint16_t *q, *k, *v;  // q null: keys and values alone
  int64_t q_stride, k_stride, v_stride;
  uint16_t *k_pages, *v_pages, *q_out;
  const int32_t *block_tables, *lens, *q_starts, *q_lens;  // q_starts null: row b is sequence b's
  const int32_t* positions;
  const float* inv_freq;
  const uint16_t *q_norm, *k_norm;
  int32_t num_pages, max_pages, page_tokens;
  int32_t num_seqs, rows;
  int32_t hq, hkv;
  int32_t rotary_dim;
  float norm_eps;
};

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

__device__ __forceinline__ void unpack8(u32x4 x, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = bf16_lo(x[i]);
    f[2 * i + 1] = bf16_hi(x[i]);
  }
}

// x of the lane kBy further round in the row of 16
template <int kBy>
__device__ __forceinline__ float row_rotate(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x120 + kBy, 0xf, 0xf, false));
}

// Sequence b whose new rows hold row j (wave-uniform); -1 if none does.
__device__ __forceinline__ int row_sequence(const AppendArgs& a, int j, int lane) {
  for (int base = 0; base < a.num_seqs; base += 64) {
    const int i = base + lane;
    const int64_t first = i < a.num_seqs ? a.q_starts[i] : 0;
    const int64_t n = i < a.num_seqs ? a.q_lens[i] : 0;
    const unsigned long long hit = __ballot(first <= j && j < first + n);
    if (hit) return base + __builtin_ctzll(hit);
  }
  return -1;
}

// How a call's rows pass the caches: as they are, written past them, or read past them too.
enum Stream { kCached, kStreamOut, kStreamBoth };

// kRowWaves waves share the heads of a row.
template <int kRowWaves, int kStream, bool kNorm, bool kInterleaved>
__global__ __launch_bounds__(64 * kWaves) void kv_append_kernel(AppendArgs a) {
  __shared__ __attribute__((aligned(16))) float2 lds_turn[kWaves][kAngles];  // cosine, sine
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int j = (int)blockIdx.x * (kWaves / kRowWaves) + wave / kRowWaves;
  if (j >= a.rows) return;
  int b, p;
  if (a.q_starts == nullptr) {
    b = j;
    p = max(a.lens[b], 0) - 1;
  } else {
    b = row_sequence(a, j, lane);
    if (b < 0) return;
    p = max(a.lens[b], 0) - a.q_lens[b] + (j - a.q_starts[b]);
  }
  if (p < 0) return;
  // the token's cache row, -1 outside the cache
  int64_t slot = -1;
  {
    const int pj = p / a.page_tokens;
    if (pj < a.max_pages) {
      const int page = a.block_tables[(size_t)b * a.max_pages + pj];
      if (page >= 0 && page < a.num_pages) slot = (int64_t)page * a.page_tokens + (p - pj * a.page_tokens);
    }
  }

  const int hl = lane & (kHeadLanes - 1);  // lane of the head
  const int rot_lanes = a.rotary_dim / kLaneDims;
  const int half_lanes = rot_lanes / 2;
  // this lane's cosines and sines, sine negative where the lane holds the pair's first
  float turn_c[kLaneDims], turn_s[kLaneDims];
  int partner = lane;
  if (rot_lanes > 0) {
    if (lane < a.rotary_dim / 2) {
      const int pos = a.positions != nullptr ? a.positions[j] : p;
      const double turns = (double)pos * (double)a.inv_freq[lane] * 0.15915494309189533577;
      float s, c;
      sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
      lds_turn[wave][lane] = make_float2(c, s);
    }
    // the wave's own LDS accesses execute in order
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
    if (kInterleaved) {
#pragma unroll
      for (int e = 0; e < kLaneDims; e += 2) {
        const float2 cs = lds_turn[wave][(hl < rot_lanes ? hl : 0) * (kLaneDims / 2) + e / 2];
        turn_c[e] = turn_c[e + 1] = cs.x;
        turn_s[e] = -cs.y;
        turn_s[e + 1] = cs.y;
      }
    } else {
      const bool second = hl >= half_lanes;
      const int at = hl < rot_lanes ? (second ? hl - half_lanes : hl) * kLaneDims : 0;
#pragma unroll
      for (int e = 0; e < kLaneDims; ++e) {
        const float2 cs = lds_turn[wave][at + e];
        turn_c[e] = cs.x;
        turn_s[e] = second ? cs.y : -cs.y;
      }
      if (hl < rot_lanes) partner = second ? lane - half_lanes : lane + half_lanes;
    }
  }

  u32x4 wq = {0u, 0u, 0u, 0u}, wk = wq;  // norm weights of this lane's dimensions
  if (kNorm) {
    if (a.q_norm != nullptr) wq = *reinterpret_cast<const u32x4*>(a.q_norm + hl * kLaneDims);
    if (a.k_norm != nullptr) wk = *reinterpret_cast<const u32x4*>(a.k_norm + hl * kLaneDims);
  }

  const int heads = a.hq + 2 * a.hkv;
  const int first = a.q != nullptr ? 0 : a.hq;
  for (int h0 = first + (wave % kRowWaves) * kPassHeads; h0 < heads; h0 += kRowWaves * kPassHeads) {
    const int h = h0 + lane / kHeadLanes;
    const bool is_q = h < a.hq, is_k = !is_q && h < a.hq + a.hkv;
    const uint16_t* src;
    uint16_t* dst;
    if (is_q) {
      src = a.q + (int64_t)j * a.q_stride + (int64_t)h * kHeadDim;
      dst = a.q_out + ((int64_t)j * a.hq + h) * kHeadDim;
    } else {
      const int kv = is_k ? h - a.hq : h - a.hq - a.hkv;
      src = (is_k ? a.k + (int64_t)j * a.k_stride : a.v + (int64_t)j * a.v_stride) + (int64_t)kv * kHeadDim;
      dst = (is_k ? a.k_pages : a.v_pages) + (slot * a.hkv + kv) * kHeadDim;
    }
    const bool live = h < heads && (is_q || slot >= 0);
    u32x4 x = {0u, 0u, 0u, 0u};
    if (live)
      x = kStream == kStreamBoth ? load16(src + hl * kLaneDims) : *reinterpret_cast<const u32x4*>(src + hl * kLaneDims);
    float f[kLaneDims];
    unpack8(x, f);
    if (kNorm) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < kLaneDims; ++e) sum = fmaf(f[e], f[e], sum);
      sum += row_rotate<8>(sum);
      sum += row_rotate<4>(sum);
      sum += row_rotate<2>(sum);
      sum += row_rotate<1>(sum);
      const float r = rsqrtf(fmaf(sum, 1.0f / kHeadDim, a.norm_eps));
      if (is_q ? a.q_norm != nullptr : a.k_norm != nullptr) {
        float w[kLaneDims];
        unpack8(is_q ? wq : wk, w);
#pragma unroll
        for (int e = 0; e < kLaneDims; ++e) f[e] = f[e] * r * w[e];
      }
    }
    float o[kLaneDims];
    if (kInterleaved) {
#pragma unroll
      for (int e = 0; e < kLaneDims; ++e) o[e] = fmaf(f[e], turn_c[e], f[e ^ 1] * turn_s[e]);
    } else {
#pragma unroll
      for (int e = 0; e < kLaneDims; ++e) {
        const float other = rot_lanes > 0 ? __shfl(f[e], partner) : 0.f;
        o[e] = fmaf(f[e], turn_c[e], other * turn_s[e]);
      }
    }
    u32x4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      y[i] = hl < rot_lanes ? pack_bf16x2(o[2 * i], o[2 * i + 1]) : pack_bf16x2(f[2 * i], f[2 * i + 1]);
    if (!is_q && !is_k) y = x;
    if (live) {
      if constexpr (kStream != kCached)
        __builtin_nontemporal_store(y, reinterpret_cast<u32x4*>(dst + hl * kLaneDims));
      else
        *reinterpret_cast<u32x4*>(dst + hl * kLaneDims) = y;
    }
  }
}

template <int kRowWaves, int kStream>
void launch_append(const AppendArgs& a, bool norm, bool interleaved, hipStream_t s) {
  constexpr int kRows = kWaves / kRowWaves;
  const dim3 grid((unsigned)((a.rows + kRows - 1) / kRows)), block(64 * kWaves);
  if (norm && interleaved)
    hipLaunchKernelGGL((kv_append_kernel<kRowWaves, kStream, true, true>), grid, block, 0, s, a);
  else if (norm)
    hipLaunchKernelGGL((kv_append_kernel<kRowWaves, kStream, true, false>), grid, block, 0, s, a);
  else if (interleaved)
    hipLaunchKernelGGL((kv_append_kernel<kRowWaves, kStream, false, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((kv_append_kernel<kRowWaves, kStream, false, false>), grid, block, 0, s, a);
}

int check_stride(const char* name, int64_t stride, int64_t heads) {
  if (stride < heads * kHeadDim || stride % 8 != 0)
    return fail(CTX_ERR_INVALID_ARG, "%s_stride %lld must be a multiple of 8 and at least %lld", name,
                (long long)stride, (long long)(heads * kHeadDim));
  return CTX_OK;
}

}  // namespace

extern "C" int ctx_kv_append_run_paged(ctx_decode_attn* h, const void* q, int64_t q_stride, const void* k,
                                       int64_t k_stride, const void* v, int64_t v_stride, void* k_pages,
                                       void* v_pages, int32_t num_pages, const int32_t* block_tables,
                                       int32_t max_pages_per_seq, const int32_t* seq_lens, const int32_t* q_starts,
                                       const int32_t* q_lens, int32_t num_seqs, int32_t total_q,
                                       const ctx_rotary* rotary, void* q_out, void* stream) {
  int rc = check_common(h, num_seqs, 1.0f);
  if (rc != CTX_OK) return rc;
  const ctx_decode_attn_desc& d = h->desc;
  if (d.page_tokens <= 0) return fail(CTX_ERR_UNSUPPORTED, "the handle was created without page_tokens");
  if (total_q < 0) return fail(CTX_ERR_INVALID_ARG, "total_q %d < 0", total_q);
  if (num_pages < 0 || max_pages_per_seq <= 0)
    return fail(CTX_ERR_INVALID_ARG, "num_pages must not be negative and max_pages_per_seq must be positive");
  if ((q_starts == nullptr) != (q_lens == nullptr))
    return fail(CTX_ERR_INVALID_ARG, "q_starts and q_lens must both be given or both be NULL");
  if (q_starts == nullptr && total_q != num_seqs)
    return fail(CTX_ERR_INVALID_ARG, "without q_starts total_q %d must be num_seqs %d", total_q, num_seqs);
  if ((q == nullptr) != (q_out == nullptr))
    return fail(CTX_ERR_INVALID_ARG, "q and q_out must both be given or both be NULL");
  ctx_rotary r{};
  if (rotary != nullptr) r = *rotary;
  if ((r.flags & ~CTX_ROTARY_INTERLEAVED) != 0) return fail(CTX_ERR_INVALID_ARG, "unknown rotary flags 0x%x", r.flags);
  if (r.rotary_dim < 0) return fail(CTX_ERR_INVALID_ARG, "rotary_dim %d < 0", r.rotary_dim);
  if (r.rotary_dim > kHeadDim || r.rotary_dim % 16 != 0)
    return fail(CTX_ERR_UNSUPPORTED, "rotary_dim %d must be a multiple of 16 up to %d", r.rotary_dim, kHeadDim);
  if ((r.rotary_dim > 0) != (r.inv_freq != nullptr))
    return fail(CTX_ERR_INVALID_ARG, "inv_freq and a positive rotary_dim go together");
  if ((r.q_norm != nullptr || r.k_norm != nullptr) && !(std::isfinite(r.norm_eps) && r.norm_eps >= 0.f))
    return fail(CTX_ERR_INVALID_ARG, "norm_eps must be finite and >= 0");
  if (num_seqs == 0 || total_q == 0) return CTX_OK;
  if (k == nullptr || v == nullptr || k_pages == nullptr || v_pages == nullptr || block_tables == nullptr ||
      seq_lens == nullptr)
    return fail(CTX_ERR_INVALID_ARG, "NULL data pointer");
  if (q != nullptr && (rc = check_stride("q", q_stride, d.num_q_heads)) != CTX_OK) return rc;
  if ((rc = check_stride("k", k_stride, d.num_kv_heads)) != CTX_OK) return rc;
  if ((rc = check_stride("v", v_stride, d.num_kv_heads)) != CTX_OK) return rc;
  if (q_out == q && q != nullptr && q_stride != (int64_t)d.num_q_heads * kHeadDim)
    return fail(CTX_ERR_INVALID_ARG, "q_out may be q only if q's rows are contiguous");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(k_pages) || !aligned16(v_pages) ||
      !aligned16(q_out) || !aligned16(r.q_norm) || !aligned16(r.k_norm))
    return fail(CTX_ERR_ALIGNMENT, "q, k, v, k_pages, v_pages, q_out and norm weights must be 16-byte aligned");
  rc = check_device(h);
  if (rc != CTX_OK) return rc;
  AppendArgs a{};
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.k_pages = static_cast<uint16_t*>(k_pages);
  a.v_pages = static_cast<uint16_t*>(v_pages);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.block_tables = block_tables;
  a.lens = seq_lens;
  a.q_starts = q_starts;
  a.q_lens = q_lens;
  a.positions = r.positions;
  a.inv_freq = r.inv_freq;
  a.q_norm = static_cast<const uint16_t*>(r.q_norm);
  a.k_norm = static_cast<const uint16_t*>(r.k_norm);
  a.num_pages = num_pages;
  a.max_pages = max_pages_per_seq;
  a.page_tokens = d.page_tokens;
  a.num_seqs = num_seqs;
  a.rows = total_q;
  a.hq = d.num_q_heads;
  a.hkv = d.num_kv_heads;
  a.rotary_dim = r.rotary_dim;
  a.norm_eps = r.norm_eps;
  const bool norm = r.q_norm != nullptr || r.k_norm != nullptr;
  const bool interleaved = (r.flags & CTX_ROTARY_INTERLEAVED) != 0;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  // A row per wave once that fills the chip; before, its heads are shared by the 4 waves of
  // a workgroup.  In a graph, 4 waves and 1 per row of 32/8 heads: 64 rows 4.6 and 10.0 us,
  // 1,000 8.7 and 13.6, 2,500 14.0 and 15.4, 3,000 15.4 and 15.8, 3,500 20.2 and 17.7, 4,100
  // 24.0 and 19.4; of 16/8 heads 3,000 12.6 and 12.3.  Large calls write past the caches, and
  // those that move more than the 256 MiB last-level cache read past them too: 30,629 rows
  // of 32/8 heads 154 us with neither, 145 with the first, 136 with both; 20,479 of 28/4 77,
  // 74 and 70.  (Smaller calls find in it what the projection
  // has just written: 9,600 rows and their prefill 192 us, 206 with both.)
  const int64_t moved = (int64_t)a.rows * ((a.q != nullptr ? a.hq : 0) + 2 * a.hkv) * kHeadDim * 2 * 2;
  if ((int64_t)a.rows < 11 * (int64_t)h->num_cus)
    launch_append<kWaves, kCached>(a, norm, interleaved, s);
  else if (moved <= (int64_t)256 << 20)
    launch_append<1, kStreamOut>(a, norm, interleaved, s);
  else
    launch_append<1, kStreamBoth>(a, norm, interleaved, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "kernel launch");
  return CTX_OK;
}
