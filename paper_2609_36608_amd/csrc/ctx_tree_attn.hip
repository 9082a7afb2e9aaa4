// ctx_tree_attn.hip -- attention of drafted trees over paged caches for gfx950 (MI355X),
// behind ctx_tree_attn_run_paged in the C ABI declared in include/ctx_tree_attn.h.
//
// As in the causal prefill, the columns of the 16-column MFMA tiles are the consecutive
// (draft, head) pairs of one KV group, S^T = K Q^T and O^T += V^T P^T.  Here all drafts
// of a sequence see nearly the same long context, so one pass over it serves all columns:
// bound by HBM up to about 128 columns per KV head, beyond by vector and matrix work.
//
//   * Work: an item is a (sequence, tile of columns, KV head), as long as the sequence has
//     blocks of 32 tokens.  The items' blocks, one after another, are cut into equal ranges,
//     one per workgroup; a workgroup finds its own from the lengths.  An item that lies
//     within a range gets its outputs at once; of the others each workgroup writes a partial
//     one, at most two, and tree_join_kernel joins them in order.
//   * A workgroup has 8 waves on a CU of its own.  With up to 128 columns four waves hold the
//     columns and the two fours take one of two neighbouring blocks each, joined
//     through LDS at the item's end; with more, all eight hold columns.  The blocks
//     pass through four stages of LDS tiles, loaded three steps ahead by all waves; waves
//     without columns only load.  32 query heads on 8, bf16: 64 contexts of 2,048..8,191 with
//     12..31 drafts 286 us, 4.9 TB/s; 32 of 512..32,767 with 64 drafts 427 us, 650 TFLOP/s (two-term
//     weights 320 and 495).  In the first milliseconds of load, while the clock falls, up to 371 and 539.
//     With 4 waves and two workgroups per CU 308 and 511 us; with the next block's keys read
//     ahead, which spills registers for fp32 outputs, 308 and 380 (290 and 425 at that time).
//   * Trees: the ancestors of every draft, as a mask of bits, by doubling: with the ancestors up
//     to 2^k steps up known, those up to 2^(k+1) are these and those of the one 2^k up.
//     They are needed for the blocks that hold drafts, and elsewhere only for the drafts'
//     depths, where a window or slopes ask for positions; blocks without drafts are on their
//     way meanwhile.
//   * Blocks that no draft sees (between the prefix and the window) are left out, as in the
//     prefill: tokens are numbered flattened, as v, and token v + skip is meant from v = hole on.
//   * Scores are kept relative to the running maximum (log2 units), which moves when a column
//     passes it by 2^8.

#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "ctx_attn_common.h"
#include "ctx_paged_common.h"
#include "ctx_tree_attn.h"

namespace {

constexpr int kBlock = 32;  // tokens
constexpr int kHalf = 16;   // tokens of half a block: on one page
constexpr int kBlockElems = kBlock * kHeadDim;
constexpr int kNowhere = 0x7ffffff0;  // a byte offset past every range
constexpr int kHeld = 64;             // half blocks whose cache rows a wave holds
constexpr int kMostDrafts = CTX_TREE_MAX_DRAFTS;
constexpr int kLeastBlocks = 4;       // of a range (4 contexts of up to 1,024 tokens 21.7 us; 2: 22.0, 8: 23.0)

// what a kernel changes of the scores
enum Change { kPlain, kBias, kCap, kCapBias };

struct TreePlan {
  const int32_t *block_tables, *lens, *q_starts, *q_lens, *parents;
  const int32_t* prefix_lens;  // or null
  const float* slopes;         // or null
  int32_t window;              // or 0
  int32_t max_pages, num_pages;
  Divisor page_tokens;
  int32_t total_q, max_q_len, num_seqs;
  int32_t hq, hkv;
  Divisor group;
  int32_t ranges;
  float* o_ws;      // partial outputs [ranges, 2, columns of a workgroup, D] and
  float2* ml_ws;    // their (maximum, sum) pairs
  int64_t* before;  // blocks before each sequence's, and of a range
  float factor;     // of the product in log2 units, without a cap
  float cap_in, cap_out;  // scale / cap and cap in log2 units
};

// What a sequence's drafts see: the tokens before prefix, and from low on.
struct Seen {
  int drafts, hist, end;  // drafts, tokens before them, tokens with them (that the table can name)
  int prefix, low;
  int hole, skip;
  int blocks;
};

__device__ __forceinline__ Seen seen_of(const TreePlan& pp, int b) {
  Seen s;
  const int len = pp.lens[b] < 0 ? 0 : pp.lens[b];
  const int given = pp.q_lens[b] < 0 ? 0 : pp.q_lens[b] < len ? pp.q_lens[b] : len;
  s.drafts = given < pp.max_q_len ? given : pp.max_q_len;
  s.hist = len - given;
  const int64_t named = (int64_t)pp.max_pages * pp.page_tokens.d;
  const int64_t end = (int64_t)s.hist + s.drafts < named ? (int64_t)s.hist + s.drafts : named;
  s.end = end < kMostTokens ? (int)end : kMostTokens;
  int prefix = pp.prefix_lens != nullptr ? pp.prefix_lens[b] : 0;
  prefix = prefix < s.hist ? prefix : s.hist;
  prefix = prefix < s.end ? prefix : s.end;
  s.prefix = prefix < 0 ? 0 : prefix;
  int low = pp.window > 0 && s.hist >= pp.window ? s.hist - pp.window + 1 : 0;
  s.low = low < s.end ? low : s.end;
  s.hole = (s.prefix + kBlock - 1) & -kBlock;
  s.skip = (s.low & -kBlock) > s.hole ? (s.low & -kBlock) - s.hole : 0;
  const int blocks = (s.end - s.skip + kBlock - 1) / kBlock;
  s.blocks = blocks > 0 ? blocks : 1;
  return s;
}

template <int kCols>
__device__ __forceinline__ int tiles_of(const TreePlan& pp, int drafts) {
  return (drafts * pp.group.d + kCols - 1) / kCols;
}

// x, which all lanes hold, as a scalar
__device__ __forceinline__ int64_t uniform(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)x >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}

__device__ __forceinline__ int64_t quota_of(int64_t total, int ranges) {
  const int64_t even = (total + ranges - 1) / ranges;
  return even > kLeastBlocks ? even : kLeastBlocks;
}

// A barrier after which the waves see each other's LDS writes.  Loads into LDS stay in flight.
__device__ __forceinline__ void lds_sync() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

constexpr int kWaves = 8;
constexpr int kStages = 4;  // of a step's blocks in LDS

// Column waves (the others take other blocks) and 16-column tiles per wave.
template <int kColWaves, int kTiles>
constexpr int kColsOf = kColWaves* kTiles * 16;

// kTerms: bf16 terms of each softmax weight, 1, 2 (16 bits) or 3 (24).  With bf16 outputs one, as in the other
// attention calls, unless asked: their own rounding is 0.0017 of the result (2-norm), with one term
// the whole is 0.0018 to 0.0023, and two cost 12 to 16% of the time (64 contexts 320 us for 286).
template <typename OutT, int kTerms, int kChange, int kColWaves, int kTiles>
__global__ __launch_bounds__(64 * kWaves) void tree_attn_kernel(const uint16_t* __restrict__ q,
                                                                const uint16_t* __restrict__ kc,
                                                                const uint16_t* __restrict__ vc, TreePlan pp,
                                                                OutT* __restrict__ out) {
  constexpr bool kHasBias = (kChange & 1) != 0;
  constexpr bool kHasCap = kChange >= kCap;
  constexpr int kCols = kColsOf<kColWaves, kTiles>;
  constexpr int kNodes = kCols < kMostDrafts ? kCols : kMostDrafts;  // most drafts of a sequence
  constexpr int kWords = kNodes / 32;
  constexpr int kStep = kWaves / kColWaves;  // blocks of a step; also loads per thread of its K, and of its V
  constexpr int kLoads = 2 * kStep;
  constexpr int kStageElems = kStep * kBlockElems;
  static_assert(kWaves * 4 == kBlock, "a wave loads four tokens of every block");
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col_wave = wave % kColWaves;
  const int part_wave = wave / kColWaves;  // which block of a step
  const int n = lane & 15;
  const int c = lane >> 4;
  const int g = pp.group.d;

  // stages of K and V, distinct arrays named at compile time, so that the compiler's waits before
  // the reads cover only their own stage's loads
  __shared__ __attribute__((aligned(16))) uint16_t lds_k0[kStageElems], lds_v0[kStageElems];
  __shared__ __attribute__((aligned(16))) uint16_t lds_k1[kStageElems], lds_v1[kStageElems];
  __shared__ __attribute__((aligned(16))) uint16_t lds_k2[kStageElems], lds_v2[kStageElems];
  __shared__ __attribute__((aligned(16))) uint16_t lds_k3[kStageElems], lds_v3[kStageElems];
  __shared__ uint32_t lds_mask[kNodes][kWords];  // bit a of draft i: it sees draft a
  __shared__ int16_t lds_depth[kNodes];          // -1: padding
  __shared__ int16_t lds_up[kNodes];

  // this workgroup's range
  int64_t blocks = 0, sum = 0;  // of the lane's sequence, and up to it among the wave's
  auto count = [&](int base) __attribute__((always_inline)) {
    const int b = base + lane;
    blocks = 0;
    if (b < pp.num_seqs) {
      const Seen s = seen_of(pp, b);
      blocks = (int64_t)s.blocks * tiles_of<kCols>(pp, s.drafts) * pp.hkv;
    }
    sum = blocks;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int64_t y = __shfl_up(sum, off);
      if (lane >= off) sum += y;
    }
  };
  int64_t total = 0;
  for (int base = 0; base < pp.num_seqs; base += 64) {
    count(base);
    if (blockIdx.x == 0 && wave == 0 && base + lane < pp.num_seqs) pp.before[base + lane] = total + sum - blocks;
    total += uniform(__shfl(sum, 63));
  }
  const int64_t quota = quota_of(total, pp.ranges);
  if (blockIdx.x == 0 && tid == 0) pp.before[pp.num_seqs] = quota;
  const int64_t begin = (int64_t)blockIdx.x * quota;
  int64_t from = begin;
  const int64_t to = begin + quota < total ? begin + quota : total;
  if (from >= to) return;
  // the sequence that it starts in
  int b = 0;
  int64_t at = 0;  // blocks before it
  for (int base = 0; base < pp.num_seqs; base += 64) {
    if (pp.num_seqs > 64) count(base);
    const unsigned long long after = __ballot(at + sum > from);
    if (after != 0) {
      const int first = __builtin_ctzll(after);
      b = base + first;
      at += uniform(__shfl(sum - blocks, first));
      break;
    }
    at += uniform(__shfl(sum, 63));
  }
  b = __builtin_amdgcn_readfirstlane(b);

  const size_t row_elems = (size_t)pp.hkv * kHeadDim;
  const int row_bytes = (int)(row_elems * 2);
  // per-lane LDS offsets of the operand reads within a 16-token half block
  int k_off[4];
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) k_off[kk] = n * kHeadDim + (((4 * kk + c) ^ tile_swizzle(n)) << 3);
  const int v_tok = 4 * c + (n >> 2);
  const int v_row = v_tok * kHeadDim + 4 * (n & 1);
  const int v_swz = tile_swizzle(v_tok);
  const int v_ch = (n & 3) >> 1;
  // A block load writes lane L's 16 bytes at LDS base + 16 L: a wave fills the slots of four tokens
  // of a half block, and each lane fetches the chunk that the swizzle puts at its slot.
  const int load_tok = (wave & 3) * 4 + (lane >> 4);  // within the half
  const int load_off = load_tok * row_bytes + (((lane & 15) ^ tile_swizzle(load_tok)) << 4);
  const int load_half = wave >> 2;

  int tree_of = -1;  // the sequence whose tree is in LDS
  for (; from < to; ++b) {
    const Seen s = seen_of(pp, b);
    const int64_t items = (int64_t)tiles_of<kCols>(pp, s.drafts) * pp.hkv;
    const int64_t behind = at + items * s.blocks;
    while (from < to && from < behind) {
      const int64_t item = (from - at) / s.blocks;
      const int first_block = (int)(from - at - item * s.blocks);
      const int last_block = s.blocks - first_block < to - from ? s.blocks : first_block + (int)(to - from);
      const int tile = __builtin_amdgcn_readfirstlane((int)(item / pp.hkv));
      const int kv = __builtin_amdgcn_readfirstlane((int)(item - (int64_t)tile * pp.hkv));
      const bool whole_item = first_block == 0 && last_block == s.blocks;
      const int64_t slot = 2 * (int64_t)blockIdx.x + (from == begin ? 0 : 1);
      from += last_block - first_block;

      const int row0 = pp.q_starts[b];
      // the tree, for blocks with drafts and where positions are asked for; the item's last
      // workgroup has it in any case, to know the padding
      const bool has_drafts = last_block == s.blocks || last_block * kBlock + s.skip > s.hist;
      const bool need_tree = tree_of != b && (has_drafts || pp.window > 0 || kHasBias);
      int up = -2;  // the ancestor 2^k above; -1: none, -2: padding
      if (need_tree && tid < s.drafts) {
        const int64_t row = (int64_t)row0 + tid;
        const int parent = row >= 0 && row < pp.total_q ? pp.parents[row] : -2;
        up = parent >= -1 && parent < tid ? parent : -2;
      }
      // this lane's columns
      auto row_at = [&](int ct) -> int64_t {  // first element of its query (and output) row, -1 without one
        const int col = tile * kCols + (ct * kColWaves + col_wave) * 16 + n;
        const int qi = pp.group.of(col);
        const int64_t row = (int64_t)row0 + qi;
        return qi < s.drafts && row >= 0 && row < pp.total_q ? (row * pp.hq + kv * g + (col - qi * g)) * kHeadDim : -1;
      };
      auto head_at = [&](int ct) {
        const int col = tile * kCols + (ct * kColWaves + col_wave) * 16 + n;
        return kv * g + (col - pp.group.of(col) * g);
      };
      bf16x8 qb[kTiles][4];
      float slope[kTiles];
#pragma unroll
      for (int ct = 0; ct < kTiles; ++ct) {
        const int64_t row = row_at(ct);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          qb[ct][kk] = as_bf16x8(row >= 0 ? load16(q + row + 8 * c + 32 * kk) : u32x4{0u, 0u, 0u, 0u});
        slope[ct] = kHasBias && row >= 0 ? pp.slopes[head_at(ct)] * 1.4426950408889634f : 0.f;
      }
      int draft[kTiles];  // -1 without one
      int low[kTiles], pos[kTiles];
      bool padding[kTiles];
      int all_low = 0;  // what every column of the wave sees past the prefix
      const bool busy = pp.group.of(tile * kCols + col_wave * 16) < s.drafts;  // wave-uniform

      Softmax st[kTiles];
      int unset = (1 << kTiles) - 1;  // bit ct: the column has seen no token yet
      f32x4 o[kTiles][8];
#pragma unroll
      for (int ct = 0; ct < kTiles; ++ct) {
        st[ct] = Softmax{0.f, 0.f};
#pragma unroll
        for (int nb = 0; nb < 8; ++nb) o[ct][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
      }

      const uint16_t* const khead = kc + (size_t)kv * kHeadDim;
      const uint16_t* const vhead = vc + (size_t)kv * kHeadDim;
      auto token = [&](int v) { return v < s.hole ? v : v + s.skip; };
      // Of the halves of the next kHeld / 2 blocks, from `held` on, one per lane: its first cache
      // row / 16, whether it may have tokens that no draft sees (kEdge), and its tokens
      // before the end; 0 outside the cache and past the end.
      constexpr uint32_t kEdge = 32;
      int held = 0;
      uint32_t halves = 0;
      auto look_up = [&](int u) __attribute__((always_inline)) {
        held = u;
        halves = 0;
        int half = lane;
        asm volatile("" : "+v"(half));  // nothing of this is kept in a register for the next time
        const int block = u + (half >> 1);
        const int t = token(block * kBlock + (half & 1) * kHalf);
        if (block < last_block && t < s.end) {
          const int j = pp.page_tokens.of(t);
          if (j < pp.max_pages) {
            const int page = pp.block_tables[(size_t)b * pp.max_pages + j];
            if (page >= 0 && page < pp.num_pages) {
              const int row = page * pp.page_tokens.d + (t - j * pp.page_tokens.d);
              const uint32_t edge = (t < s.low && t + kHalf > s.prefix) || t + kHalf > s.hist ? kEdge : 0u;
              halves = (uint32_t)(row / kHalf) << 6 | edge | (uint32_t)(s.end - t < kHalf ? s.end - t : kHalf);
            }
          }
        }
      };
      uint32_t absent = 0;  // a byte per step, the next one's lowest: bit h where half h is on no page
      // the loads of the blocks u .. u + kStep - 1 into a stage
      auto issue = [&](int u, uint16_t* dk, uint16_t* dv, int ahead) __attribute__((always_inline)) {
        if (u - held >= kHeld / 2) look_up(u);
#pragma unroll
        for (int r = 0; r < kStep; ++r) {
          const int lane0 = (u - held + r) * 2;
          const uint32_t w0 = (uint32_t)__builtin_amdgcn_readlane((int)halves, lane0);
          const uint32_t w1 = (uint32_t)__builtin_amdgcn_readlane((int)halves, lane0 + 1);
          const uint32_t gone = ((w0 & 31) == 0 ? 1u : 0u) | ((w1 & 31) == 0 ? 2u : 0u);
          if (r == part_wave) absent |= gone << (8 * ahead);
          const uint32_t w = load_half == 0 ? w0 : w1;
          const uint64_t first = (uint64_t)(w >> 6) * (uint32_t)(kHalf * row_bytes);
          const uint32_t bytes = (w & 31) * (uint32_t)row_bytes;
          const int to_lds = r * kBlockElems + (load_half * kHalf + (wave & 3) * 4) * kHeadDim;
          int off = load_off;
          load16_to_lds<kLoadAux>(
              make_rsrc(reinterpret_cast<const uint16_t*>(reinterpret_cast<const char*>(khead) + first), bytes),
              dk + to_lds, off);
          if (w & kEdge) {  // values that no draft sees may hold anything: zeros
            int at_tok = load_tok;
            asm volatile("" : "+v"(at_tok));
            const int t = token((u + r) * kBlock + load_half * kHalf) + at_tok;
            const bool hidden = t < s.hist ? t >= s.prefix && t < s.low : t < s.end && lds_depth[t - s.hist] < 0;
            if (hidden) off = kNowhere;
          }
          load16_to_lds<kLoadAux>(
              make_rsrc(reinterpret_cast<const uint16_t*>(reinterpret_cast<const char*>(vhead) + first), bytes),
              dv + to_lds, off);
        }
      };

      // S^T of a staged block: tokens 16 h + 4c + i (i < 4) for every column tile
      auto scores = [&](const uint16_t* kt, f32x4 (&sc)[kTiles][2]) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          u32x4 kr[4];
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            kr[kk] = *reinterpret_cast<const u32x4*>(kt + 16 * h * kHeadDim + k_off[kk]);
#pragma unroll
          for (int ct = 0; ct < kTiles; ++ct) sc[ct][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int ct = 0; ct < kTiles; ++ct)
              sc[ct][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kr[kk]), qb[ct][kk], sc[ct][h], 0, 0, 0);
        }
        // no use of a product between the others: it would hold them up
        __builtin_amdgcn_sched_barrier(0);
      };
      // the scores in log2 units less the running maxima, -inf where a token is not seen
      auto relative = [&](int u, int gone, f32x4 (&sc)[kTiles][2]) __attribute__((always_inline)) {
        const int t0 = token(u * kBlock);
        const bool drafts = t0 + kBlock > s.hist;
        auto each = [&](auto&& change) __attribute__((always_inline)) {
          if (!kHasBias || !drafts) {
#pragma unroll
            for (int ct = 0; ct < kTiles; ++ct) {
              const float base = kHasBias ? fmaf(slope[ct], (float)(t0 + 4 * c - pos[ct]), -st[ct].m) : -st[ct].m;
#pragma unroll
              for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  sc[ct][h][i] = change(sc[ct][h][i], kHasBias ? fmaf(slope[ct], (float)(16 * h + i), base) : base);
            }
          } else {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int t = t0 + 16 * h + 4 * c + i;
                const int a = t - s.hist;
                const int p = a < 0 ? t : s.hist + (a < s.drafts ? lds_depth[a] : 0);
#pragma unroll
                for (int ct = 0; ct < kTiles; ++ct)
                  sc[ct][h][i] = change(sc[ct][h][i], fmaf(slope[ct], (float)(p - pos[ct]), -st[ct].m));
              }
          }
        };
        if constexpr (!kHasCap) {
          each([&](float x, float add) __attribute__((always_inline)) { return fmaf(x, pp.factor, add); });
        } else {
          float most = 0.f;
#pragma unroll
          for (int ct = 0; ct < kTiles; ++ct)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int i = 0; i < 4; ++i) most = fmaxf(most, fabsf(sc[ct][h][i]));
          if (!__any(most * fabsf(pp.cap_in) > kTanhSmall)) {
            each([&](float x, float add) __attribute__((always_inline)) {
              return fmaf(tanh_small(x * pp.cap_in), pp.cap_out, add);
            });
          } else {
            each([&](float x, float add) __attribute__((always_inline)) {
              return fmaf(tanh_any(x * pp.cap_in), pp.cap_out, add);
            });
          }
        }
        if (!drafts && gone == 0 && (t0 >= all_low || t0 + kBlock <= s.prefix)) return;  // all see all
#pragma unroll
        for (int ct = 0; ct < kTiles; ++ct) {
          uint32_t bits = 0;  // which of the block's tokens are drafts that the column sees
          if (drafts && draft[ct] >= 0) {
            const int o0 = t0 - s.hist;
            const int w = o0 >> 5, sh = o0 & 31;
            const uint32_t lo = w >= 0 && w < kWords ? lds_mask[draft[ct]][w] : 0u;
            const uint32_t hi = w + 1 < kWords ? lds_mask[draft[ct]][w + 1] : 0u;
            bits = __funnelshift_r(lo, hi, sh);
          }
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int t = t0 + 16 * h + 4 * c + i;
              const bool before = (t < s.hist) & ((t >= low[ct]) | (t < s.prefix)) & !padding[ct];
              const bool see = (before | ((bits >> (16 * h + 4 * c + i) & 1) != 0)) & !(gone >> h & 1);
              sc[ct][h][i] = see ? sc[ct][h][i] : -INFINITY;
            }
        }
      };
      // raises the maxima where a score passes its limit
      auto raise = [&](f32x4 (&sc)[kTiles][2]) __attribute__((always_inline)) {
        float lm[kTiles];
        bool over = false;
#pragma unroll
        for (int ct = 0; ct < kTiles; ++ct) {
          lm[ct] = max8(sc[ct][0], sc[ct][1]);
          over |= lm[ct] > kLazyRescale;
        }
        if (!__any(over | (unset != 0))) return;
#pragma unroll
        for (int ct = 0; ct < kTiles; ++ct) {
          const bool fresh = unset >> ct & 1;
          if (!__any(lm[ct] > (fresh ? -INFINITY : kLazyRescale))) continue;
          const float top = column_max(lm[ct]);
          const bool none = fresh && !(top > -INFINITY);
          // what the rounded sum really moves by, so that a large maximum loses nothing
          const float m = st[ct].m + (none ? 0.f : fresh ? top : fmaxf(top, 0.f));
          const float delta = m - st[ct].m;
          const float alpha = fresh ? 1.f : fast_exp2(-delta);
          if (!none) unset &= ~(1 << ct);
          st[ct].m = m;
          st[ct].l *= alpha;
#pragma unroll
          for (int nb = 0; nb < 8; ++nb) o[ct][nb] *= alpha;
#pragma unroll
          for (int h = 0; h < 2; ++h) sc[ct][h] -= delta;
        }
      };
      // the softmax weights as kTerms bf16 terms
      auto weights = [&](const f32x4 (&sc)[kTiles][2], u32x4 (&pt)[kTerms][kTiles]) __attribute__((always_inline)) {
#pragma unroll
        for (int ct = 0; ct < kTiles; ++ct) {
          float pr[8];
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) pr[4 * h + i] = fast_exp2(sc[ct][h][i]);
          if constexpr (kTerms == 1) {
            // the row sum adds the rounded weights that the product uses
            const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
            float l = st[ct].l;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const bf16x2 pair = {(__bf16)pr[2 * j], (__bf16)pr[2 * j + 1]};  // round to nearest even
              pt[0][ct][j] = __builtin_bit_cast(uint32_t, pair);
              l = __builtin_amdgcn_fdot2_f32_bf16(pair, ones, l, false);
            }
            st[ct].l = l;
          } else {
            st[ct].l += ((pr[0] + pr[1]) + (pr[2] + pr[3])) + ((pr[4] + pr[5]) + (pr[6] + pr[7]));
#pragma unroll
            for (int k = 0; k < kTerms; ++k)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint32_t w = pack_bf16x2(pr[2 * j], pr[2 * j + 1]);
                pt[k][ct][j] = w;
                pr[2 * j] -= __uint_as_float(w << 16);  // exact
                pr[2 * j + 1] -= __uint_as_float(w & 0xffff0000u);
              }
          }
        }
      };
      // O^T += V^T P^T: the K dimension holds tokens 4c .. 4c + 3 of both halves
      auto values = [&](const uint16_t* vt, const u32x4 (&pt)[kTerms][kTiles]) __attribute__((always_inline)) {
        __builtin_amdgcn_s_setprio(1);
        auto read_vt = [&](int nb, s16x4& v0, s16x4& v1) {
          const int off = v_row + (((2 * nb + v_ch) ^ v_swz) << 3);
          v0 = lds_read_tr16(vt + off);
          v1 = lds_read_tr16(vt + 16 * kHeadDim + off);
        };
        s16x4 nv0, nv1;
        read_vt(0, nv0, nv1);
#pragma unroll
        for (int nb = 0; nb < 8; ++nb) {
          const bf16x8 va = __builtin_bit_cast(bf16x8, __builtin_shufflevector(nv0, nv1, 0, 1, 2, 3, 4, 5, 6, 7));
          if (nb + 1 < 8) read_vt(nb + 1, nv0, nv1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int k = 0; k < kTerms; ++k)
#pragma unroll
            for (int ct = 0; ct < kTiles; ++ct)
              o[ct][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, as_bf16x8(pt[k][ct]), o[ct][nb], 0, 0, 0);
        }
        __builtin_amdgcn_s_setprio(0);
      };

      look_up(first_block);
      // The queries have arrived with the table's entries; said here, the compiler need not
      // wait for them in the loop, where that would be a wait for the blocks in flight too.
      __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
      // One step: wait for this wave's loads of it, then the barrier (every wave's have landed, and
      // every wave is done with the stage read in the previous step); the loads of the
      // step three ahead go into that stage.
      auto step = [&](int u, const uint16_t* kt, const uint16_t* vt, uint16_t* nk, uint16_t* nv)
          __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt(wait_vmcnt((kStages - 2) * kLoads));
        lds_barrier();
        const int gone = absent & 3;
        absent >>= 8;
        issue(u + (kStages - 1) * kStep, nk, nv, kStages - 2);
        const int mine = u + part_wave;
        if (mine < last_block && busy) {
          f32x4 sc[kTiles][2];
          u32x4 pt[kTerms][kTiles];
          scores(kt + part_wave * kBlockElems, sc);
          relative(mine, gone, sc);
          raise(sc);
          weights(sc, pt);
          values(vt + part_wave * kBlockElems, pt);
        }
      };
      auto start = [&]() __attribute__((always_inline)) {
        issue(first_block, lds_k0, lds_v0, 0);
        issue(first_block + kStep, lds_k1, lds_v1, 1);
        issue(first_block + 2 * kStep, lds_k2, lds_v2, 2);
      };
      // blocks without drafts need no tree, and are on their way while it is built
      const bool early = (int64_t)(first_block + 3 * kStep) * kBlock + s.skip <= s.hist;
      if (early) start();
      if (need_tree) {
        tree_of = b;
        uint32_t mask[kWords];
#pragma unroll
        for (int w = 0; w < kWords; ++w) mask[w] = tid < s.drafts && tid >> 5 == w ? 1u << (tid & 31) : 0u;
        for (int above = 1; above < s.drafts; above *= 2) {
          if (tid < kNodes) {
            lds_up[tid] = (int16_t)up;
#pragma unroll
            for (int w = 0; w < kWords; ++w) lds_mask[tid][w] = mask[w];
          }
          lds_sync();
          if (up >= 0) {
#pragma unroll
            for (int w = 0; w < kWords; ++w) mask[w] |= lds_mask[up][w];
            up = lds_up[up];
          }
          lds_sync();
        }
        int depth = -1;
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
          if (up == -2) mask[w] = 0;
          depth += __builtin_popcount(mask[w]);
        }
        if (tid < kNodes) lds_depth[tid] = (int16_t)depth;
        lds_sync();
        if (pp.window > 0 && depth >= pp.window) {  // ancestors past the window
#pragma unroll
          for (int w = 0; w < kWords; ++w)
            for (uint32_t left = mask[w]; left != 0; left &= left - 1) {
              const int a = w * 32 + __builtin_ctz(left);
              if (depth - lds_depth[a] >= pp.window) mask[w] &= ~(left & -left);
            }
        }
        if (tid < kNodes) {
#pragma unroll
          for (int w = 0; w < kWords; ++w) lds_mask[tid][w] = mask[w];
        }
        lds_sync();
      }
      if (!early) start();
#pragma unroll
      for (int ct = 0; ct < kTiles; ++ct) {
        const int qi = pp.group.of(tile * kCols + (ct * kColWaves + col_wave) * 16 + n);
        draft[ct] = row_at(ct) >= 0 ? qi : -1;
        low[ct] = 0;
        pos[ct] = s.hist;
        padding[ct] = false;
        if (draft[ct] >= 0) {
          if (pp.window > 0 || kHasBias) {
            const int depth = lds_depth[qi];
            padding[ct] = depth < 0;
            pos[ct] = s.hist + (depth < 0 ? 0 : depth);
            if (pp.window > 0 && pos[ct] >= pp.window) low[ct] = pos[ct] - pp.window + 1;
          } else if (has_drafts) {
            padding[ct] = lds_depth[qi] < 0;
          }
          all_low = low[ct] > all_low ? low[ct] : all_low;
        }
        if (kHasBias && slope[ct] < 0.f) st[ct].m = -slope[ct] * (float)pos[ct];  // near the largest bias
      }
#pragma unroll
      for (int off = 1; off < 16; off <<= 1) {
        const int other = __shfl_xor(all_low, off);
        all_low = other > all_low ? other : all_low;
      }
      all_low = __builtin_amdgcn_readfirstlane(all_low);
      for (int u = first_block; u < last_block; u += kStages * kStep) {
        step(u, lds_k0, lds_v0, lds_k3, lds_v3);
        if (u + kStep >= last_block) break;
        step(u + kStep, lds_k1, lds_v1, lds_k0, lds_v0);
        if (u + 2 * kStep >= last_block) break;
        step(u + 2 * kStep, lds_k2, lds_v2, lds_k1, lds_v1);
        if (u + 3 * kStep >= last_block) break;
        step(u + 3 * kStep, lds_k3, lds_v3, lds_k2, lds_v2);
      }
      // no load may land in a stage after the workgroup has gone on
      __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
      __syncthreads();

      if constexpr (kStep == 2) {
        // the second four waves' sums and outputs go to the first four's, lane by lane, which scale
        // both to the larger maximum
        static_assert(kStageElems * 2 == 2 * 8 * 64 * 16 && kTiles <= 2, "a column wave's outputs fit a stage's keys");
        float* const their_o = reinterpret_cast<float*>(col_wave == 0   ? lds_k0
                                                        : col_wave == 1 ? lds_k1
                                                        : col_wave == 2 ? lds_k2
                                                                        : lds_k3);
        float2* const their_ml = reinterpret_cast<float2*>(lds_v0) + col_wave * kTiles * 64;
        if (part_wave == 1) {
#pragma unroll
          for (int ct = 0; ct < kTiles; ++ct) {
            their_ml[ct * 64 + lane] = make_float2((unset >> ct & 1) ? -INFINITY : st[ct].m, st[ct].l);
#pragma unroll
            for (int nb = 0; nb < 8; ++nb)
              *reinterpret_cast<f32x4*>(their_o + ((ct * 8 + nb) * 64 + lane) * 4) = o[ct][nb];
          }
        }
        __syncthreads();
        if (part_wave == 0) {
#pragma unroll
          for (int ct = 0; ct < kTiles; ++ct) {
            const float2 ml = their_ml[ct * 64 + lane];
            const float m0 = (unset >> ct & 1) ? -INFINITY : st[ct].m;
            const float top = fmaxf(m0, ml.x);
            const float a0 = m0 > -INFINITY ? fast_exp2(m0 - top) : 0.f;
            const float a1 = ml.x > -INFINITY ? fast_exp2(ml.x - top) : 0.f;
            if (top > -INFINITY) {
              st[ct].m = top;
              unset &= ~(1 << ct);
            }
            st[ct].l = a0 * st[ct].l + a1 * ml.y;
#pragma unroll
            for (int nb = 0; nb < 8; ++nb)
              o[ct][nb] = a0 * o[ct][nb] + a1 * *reinterpret_cast<const f32x4*>(their_o + ((ct * 8 + nb) * 64 + lane) * 4);
          }
        }
        __syncthreads();
        if (part_wave != 0) continue;
      }
#pragma unroll
      for (int ct = 0; ct < kTiles; ++ct) {
        float l_tot = st[ct].l + __shfl_xor(st[ct].l, 16);
        l_tot += __shfl_xor(l_tot, 32);
        const int64_t row = row_at(ct);
        if (row < 0) continue;
        const bool none = (unset >> ct & 1) || padding[ct];  // padding is marked for the join
        if (whole_item) {
          const float inv = !none && l_tot != 0.f ? 1.0f / l_tot : 0.f;
          OutT* orow = out + row + 4 * c;
#pragma unroll
          for (int nb = 0; nb < 8; ++nb)
            store4<OutT>(orow + 16 * nb, none ? f32x4{0.f, 0.f, 0.f, 0.f} : o[ct][nb] * inv);
        } else {
          const int64_t part = slot * kCols + (ct * kColWaves + col_wave) * 16 + n;
          if (c == 0) pp.ml_ws[part] = make_float2(padding[ct] ? INFINITY : none ? -INFINITY : st[ct].m, none ? 0.f : l_tot);
          float* orow = pp.o_ws + part * kHeadDim + 4 * c;
#pragma unroll
          for (int nb = 0; nb < 8; ++nb) *reinterpret_cast<f32x4*>(orow + 16 * nb) = o[ct][nb];
        }
      }
    }
    at = behind;
  }
}

// Joins the partial outputs of the items: a workgroup per 16 columns of an item, 16 lanes of twice
// 4 dimensions per column.  Bound by the latency of its loads, so the lanes ask for the maxima
// and sums of 16 ranges at once, and for several ranges' outputs: 4 contexts of 1,024 4.7 us (8.2
// with 32 lanes that ask for range after range), the 32 MB of 64 contexts 13 (13 to 16).
constexpr int kJoinCols = 16;
constexpr int kJoinLanes = 16;
constexpr int kJoinParts = kHeadDim / (4 * kJoinLanes);
constexpr int kJoinThreads = kJoinCols * kJoinLanes;

template <typename OutT, int kCols>
__global__ __launch_bounds__(kJoinThreads) void tree_join_kernel(TreePlan pp, int join_tiles, OutT* __restrict__ out) {
  const int join_tile = (int)blockIdx.x % join_tiles;
  const int unit = (int)blockIdx.x / join_tiles;
  const int b = unit / pp.hkv, kv = unit - b * pp.hkv;
  const Seen s = seen_of(pp, b);
  const int lane = threadIdx.x % kJoinLanes;
  const int col = join_tile * kJoinCols + (int)threadIdx.x / kJoinLanes;
  if (join_tile * kJoinCols >= s.drafts * pp.group.d) return;
  const int row0 = pp.q_starts[b];
  const int64_t quota = pp.before[pp.num_seqs];
  const int tile = join_tile * kJoinCols / kCols;
  const int64_t first = pp.before[b] + ((int64_t)tile * pp.hkv + kv) * s.blocks;
  const int64_t r0 = first / quota;
  const int ranges = (int)((first + s.blocks - 1) / quota - r0) + 1;
  if (ranges == 1) return;  // its workgroup has written it
  const int qi = pp.group.of(col);
  const int64_t row = (int64_t)row0 + qi;
  if (qi >= s.drafts || row < 0 || row >= pp.total_q) return;  // for all lanes of the column
  // where a range begins with the item its partial output is the first of two
  const int second = first != r0 * quota ? 1 : 0;
  auto part_of = [&](int r) { return (2 * (r0 + r) + (r == 0 ? second : 0)) * kCols + (col - tile * kCols); };
  const float2 none = make_float2(-INFINITY, 0.f);
  float2 ml = lane < ranges ? pp.ml_ws[part_of(lane)] : none;  // of range base + lane
  float top = ml.x;
  for (int base = kJoinLanes; base < ranges; base += kJoinLanes)
    top = fmaxf(top, base + lane < ranges ? pp.ml_ws[part_of(base + lane)].x : -INFINITY);
#pragma unroll
  for (int off = kJoinLanes / 2; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
  f32x4 o[kJoinParts] = {};
  float sum = 0.f;
  if (top < INFINITY) {  // otherwise padding, which the last range has marked
    for (int base = 0; base < ranges; base += kJoinLanes) {
      if (base > 0) ml = base + lane < ranges ? pp.ml_ws[part_of(base + lane)] : none;
      const float mine = ml.x > -INFINITY ? fast_exp2(ml.x - top) : 0.f;
      sum = fmaf(mine, ml.y, sum);
      const int here = ranges - base < kJoinLanes ? ranges - base : kJoinLanes;
      auto add = [&](int i, auto at_once) __attribute__((always_inline)) {
        f32x4 x[at_once][kJoinParts];
#pragma unroll
        for (int u = 0; u < at_once; ++u)
#pragma unroll
          for (int p = 0; p < kJoinParts; ++p)
            x[u][p] = *reinterpret_cast<const f32x4*>(pp.o_ws + part_of(base + i + u) * kHeadDim +
                                                      (p * kJoinLanes + lane) * 4);
#pragma unroll
        for (int u = 0; u < at_once; ++u) {
          const float w = __shfl(mine, i + u, kJoinLanes);
          if (w > 0.f) {  // what a column without tokens has written may be NaN
#pragma unroll
            for (int p = 0; p < kJoinParts; ++p) o[p] += w * x[u][p];
          }
        }
      };
      int i = 0;
      for (; i + 4 <= here; i += 4) add(i, std::integral_constant<int, 4>());
      if (i + 2 <= here) {
        add(i, std::integral_constant<int, 2>());
        i += 2;
      }
      if (i < here) add(i, std::integral_constant<int, 1>());
    }
#pragma unroll
    for (int off = kJoinLanes / 2; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
  }
  const float inv = sum != 0.f ? 1.0f / sum : 0.f;
  OutT* const dst = out + (row * pp.hq + kv * pp.group.d + (col - qi * pp.group.d)) * kHeadDim;
#pragma unroll
  for (int p = 0; p < kJoinParts; ++p) store4<OutT>(dst + (p * kJoinLanes + lane) * 4, o[p] * inv);
}

// ------------------------------------------------------------ host

// Waves and tiles of a workgroup, and the ranges of a call.
struct Shape {
  int col_waves, tiles;
  int32_t ranges;
  int cols() const { return col_waves * tiles * 16; }
  int64_t parts() const { return 2 * (int64_t)ranges * cols(); }
  size_t o_bytes() const { return (size_t)parts() * kHeadDim * sizeof(float); }
  size_t ml_bytes() const { return (size_t)parts() * sizeof(float2); }
  size_t bytes(int32_t seqs) const { return o_bytes() + ml_bytes() + ((size_t)seqs + 1) * sizeof(int64_t); }
};

Shape shape_of(const ctx_decode_attn* h, int32_t num_seqs, int32_t max_q_len) {
  const ctx_decode_attn_desc& d = h->desc;
  const int64_t cols = (int64_t)max_q_len * (d.num_q_heads / d.num_kv_heads);
  Shape s;
  s.col_waves = cols <= 128 ? 4 : 8;
  s.tiles = cols <= 64 ? 1 : 2;
  // a workgroup per CU, but no more ranges than the longest sequences have parts of kLeastBlocks blocks
  const int64_t items = (int64_t)num_seqs * d.num_kv_heads * ((cols + s.cols() - 1) / s.cols());
  const int64_t blocks = ((int64_t)d.max_seq_len + kBlock - 1) / kBlock;
  const int64_t most = (items * blocks + kLeastBlocks - 1) / kLeastBlocks;
  const int64_t ranges = most < h->num_cus ? most : h->num_cus;
  s.ranges = ranges > 1 ? (int32_t)ranges : 1;
  return s;
}

int check_drafts(const ctx_decode_attn* h, int32_t num_seqs, int32_t max_q_len) {
  if (h->desc.page_tokens <= 0) return fail(CTX_ERR_UNSUPPORTED, "the handle was created without page_tokens");
  if (max_q_len < 0) return fail(CTX_ERR_INVALID_ARG, "max_q_len %d < 0", max_q_len);
  if (max_q_len > kMostDrafts) return fail(CTX_ERR_UNSUPPORTED, "max_q_len %d > %d", max_q_len, kMostDrafts);
  const int64_t tiles = ((int64_t)max_q_len * (h->desc.num_q_heads / h->desc.num_kv_heads) + kJoinCols - 1) / kJoinCols;
  if (!fits_launch(tiles * num_seqs * h->desc.num_kv_heads, kJoinThreads)) return fail(CTX_ERR_INVALID_ARG, "tree grid too large");
  return CTX_OK;
}

struct TreeArgs {
  const uint16_t *q, *k, *v;
  TreePlan plan;
  void* out;
  hipStream_t stream;
};

template <typename OutT, int kTerms, int kChange, int kColWaves, int kTiles>
void launch_shape(const TreeArgs& a) {
  constexpr int kCols = kColsOf<kColWaves, kTiles>;
  hipLaunchKernelGGL((tree_attn_kernel<OutT, kTerms, kChange, kColWaves, kTiles>), dim3((unsigned)a.plan.ranges),
                     dim3(64 * kWaves), 0, a.stream, a.q, a.k, a.v, a.plan, static_cast<OutT*>(a.out));
  const int join_tiles = (a.plan.max_q_len * a.plan.group.d + kJoinCols - 1) / kJoinCols;
  const int64_t grid = (int64_t)join_tiles * a.plan.num_seqs * a.plan.hkv;
  hipLaunchKernelGGL((tree_join_kernel<OutT, kCols>), dim3((unsigned)grid), dim3(kJoinThreads), 0, a.stream, a.plan,
                     join_tiles, static_cast<OutT*>(a.out));
}

template <typename OutT, int kTerms, int kChange>
void launch_change(const TreeArgs& a, const Shape& s) {
  if (s.tiles == 1)
    launch_shape<OutT, kTerms, kChange, 4, 1>(a);
  else if (s.col_waves == 4)
    launch_shape<OutT, kTerms, kChange, 4, 2>(a);
  else
    launch_shape<OutT, kTerms, kChange, 8, 2>(a);
}

template <typename OutT, int kTerms>
void launch_tree(const TreeArgs& a, int change, const Shape& s) {
  if (change == kPlain)
    launch_change<OutT, kTerms, kPlain>(a, s);
  else if (change == kBias)
    launch_change<OutT, kTerms, kBias>(a, s);
  else if (change == kCap)
    launch_change<OutT, kTerms, kCap>(a, s);
  else
    launch_change<OutT, kTerms, kCapBias>(a, s);
}

}  // namespace

extern "C" int ctx_tree_attn_workspace(ctx_decode_attn* h, int32_t num_seqs, int32_t max_q_len, size_t* bytes) {
  int rc = check_common(h, num_seqs, 1.0f);
  if (rc != CTX_OK) return rc;
  if (bytes == nullptr) return fail(CTX_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = 0;
  if ((rc = check_drafts(h, num_seqs, max_q_len)) != CTX_OK) return rc;
  if (num_seqs > 0 && max_q_len > 0) *bytes = shape_of(h, num_seqs, max_q_len).bytes(num_seqs);
  return CTX_OK;
}

extern "C" int ctx_tree_attn_run_paged(ctx_decode_attn* h, const void* q, const void* k_pages, const void* v_pages,
                                       int32_t num_pages, const int32_t* block_tables, int32_t max_pages_per_seq,
                                       const int32_t* seq_lens, const int32_t* q_starts, const int32_t* q_lens,
                                       const int32_t* parents, int32_t num_seqs, int32_t total_q, int32_t max_q_len,
                                       float scale, const ctx_attn_scores* scores, void* out, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  int rc = check_common(h, num_seqs, scale);
  if (rc != CTX_OK) return rc;
  ctx_attn_scores sc{};
  if (scores != nullptr) sc = *scores;
  rc = check_scored(h, sc, scale, num_pages, max_pages_per_seq);
  if (rc != CTX_OK) return rc;
  sc.softcap = cap_of(sc, scale);
  if (sc.doc_starts != nullptr) return fail(CTX_ERR_INVALID_ARG, "trees have no doc_starts");
  if (total_q < 0) return fail(CTX_ERR_INVALID_ARG, "total_q %d < 0", total_q);
  if ((rc = check_drafts(h, num_seqs, max_q_len)) != CTX_OK) return rc;
  if (num_seqs == 0 || max_q_len == 0 || total_q == 0) return CTX_OK;
  if (q == nullptr || k_pages == nullptr || v_pages == nullptr || block_tables == nullptr || seq_lens == nullptr ||
      q_starts == nullptr || q_lens == nullptr || parents == nullptr || out == nullptr || workspace == nullptr)
    return fail(CTX_ERR_INVALID_ARG, "NULL data pointer");
  if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out) || !aligned16(workspace))
    return fail(CTX_ERR_ALIGNMENT, "q, k_pages, v_pages, out and workspace must be 16-byte aligned");
  const ctx_decode_attn_desc& d = h->desc;
  const Shape shape = shape_of(h, num_seqs, max_q_len);
  if (workspace_bytes < shape.bytes(num_seqs))
    return fail(CTX_ERR_CAPACITY, "workspace of %zu bytes, %zu needed", workspace_bytes, shape.bytes(num_seqs));
  if ((rc = check_device(h)) != CTX_OK) return rc;
  TreePlan pp{};
  pp.block_tables = block_tables;
  pp.lens = seq_lens;
  pp.q_starts = q_starts;
  pp.q_lens = q_lens;
  pp.parents = parents;
  pp.prefix_lens = sc.prefix_lens;
  pp.slopes = sc.slopes;
  pp.window = sc.window;
  pp.max_pages = max_pages_per_seq;
  pp.num_pages = num_pages;
  pp.page_tokens = Divisor(d.page_tokens);
  pp.total_q = total_q;
  pp.max_q_len = max_q_len;
  pp.num_seqs = num_seqs;
  pp.hq = d.num_q_heads;
  pp.hkv = d.num_kv_heads;
  pp.group = Divisor(d.num_q_heads / d.num_kv_heads);
  pp.ranges = shape.ranges;
  char* const ws = static_cast<char*>(workspace);
  pp.o_ws = reinterpret_cast<float*>(ws);
  pp.ml_ws = reinterpret_cast<float2*>(ws + shape.o_bytes());
  pp.before = reinterpret_cast<int64_t*>(ws + shape.o_bytes() + shape.ml_bytes());
  pp.factor = (float)((double)scale * 1.4426950408889634);
  pp.cap_in = sc.softcap > 0.f ? scale / sc.softcap : 0.f;
  pp.cap_out = (float)((double)sc.softcap * 1.4426950408889634);
  const TreeArgs a{static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(k_pages),
                   static_cast<const uint16_t*>(v_pages), pp, out, reinterpret_cast<hipStream_t>(stream)};
  const int change = (sc.softcap > 0.f ? kCap : kPlain) + (sc.slopes != nullptr ? kBias : kPlain);
  if (d.out_dtype == CTX_DTYPE_F32)
    launch_tree<float, 3>(a, change, shape);
  else if ((sc.flags & CTX_SCORES_SPLIT_P) != 0)
    launch_tree<uint16_t, 2>(a, change, shape);
  else
    launch_tree<uint16_t, 1>(a, change, shape);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "kernel launch");
  return CTX_OK;
}
