// ctx_prefill_paged.hip -- causal prefill over paged caches with capped, biased and
// masked scores for gfx950 (MI355X), behind ctx_prefill_attn_run_paged in the C ABI
// declared in include/ctx_paged_attn.h.
//
// A query at position p sees token t of its sequence if t < prefix or
// low <= t <= p, low = max(doc, p - window + 1).  As in the contiguous prefill, the
// columns of the 16-column MFMA tiles are the consecutive (query position, head)
// pairs of one KV group, and 32-token K/V blocks go straight from memory into LDS:
//   * wide workgroups: 4 waves of kTiles 16-column tiles each share every block
//     through a three-stage tile, loaded two blocks ahead;
//   * narrow workgroups, for calls with too few columns to fill the chip: all 4 or 8
//     waves cover the same kTiles tiles, each with its share of the blocks, its own LDS
//     tiles and its own running maxima; they are merged through LDS in a fixed order.
//     With few rows over a long context several workgroups share a tile's blocks in turn,
//     and a second kernel joins their partial outputs.
// Per 32 tokens and 16 columns a wave computes S^T = K Q^T (8 MFMA 16x16x32), the
// scores' changes, the mask and an online softmax, and O^T += V^T P^T (8 MFMA per
// bf16 term of P; V^T through the LDS transpose read).
//
//   * Blocks: the tokens that some query of the workgroup sees are a prefix and a range
//     further on.  Whole blocks between the two are left out: tokens are numbered flattened,
//     as v, and token v + skip is meant from v = hole on.
//   * Pages: the cache rows of a wave's next 64 half blocks (16 tokens, always within a
//     page) are held one per lane, and looked up again when the loop has run past them.
//     (Asking for the next ones' pages a step ahead hid that wait and cost as much.)
//   * Masks: a block that every column of the wave sees whole is not masked; one that
//     none sees is passed over by the wave; tokens that no query of the workgroup sees
//     are loaded as zeros, whatever the pages hold there.
//   * Scores are kept relative to the running maximum m (log2 units): x - m in one FMA
//     of the product, two with a bias, so that neither the cap nor the bias needs a
//     pass of its own, and a bias of hundreds is taken off its maximum's without a
//     rounding between.  m moves only when a column passes it by 2^8.  A column starts
//     without a maximum and takes its first finite one.
//   * Biases are taken from the distance to the last token that the row sees of its
//     prefix or to its own position, whichever applies: the same for all tokens of a
//     row, it does not change the softmax and keeps large logits precise.
//   * bf16 outputs: weights rounded to bf16 and normalised by the sum of the rounded
//     ones, or, with CTX_SCORES_SPLIT_P, two bf16 terms (16 bits).  fp32 outputs: three
//     (24 bits).  With more than one, two tiles per wave, since three would not leave
//     registers for them.

// Bound by vector and matrix work together, at the clock that the power limit leaves: 100
// requests with 128..512 new tokens over 4,096..12,288 (32/8 heads, 16-token pages) run at
// 1,045 TFLOP/s, with slopes at 980, capped at 805, with both at 786, with fp32 outputs at
// 551; with two-term weights at 705, with slopes at 704, capped at 546; a single prompt of 10,240 tokens at 1,050..1,120 with shuffled pages and at
// 1,160..1,212 with pages in order.  A wave holds 16 columns in each of up to 3 tiles,
// since every K and V fragment read from LDS is then used three times; a fourth would
// leave no registers (256 at two waves per SIMD).

#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>
#include <cstdint>

#include "ctx_attn_common.h"
#include "ctx_paged_attn.h"
#include "ctx_paged_common.h"

namespace {

// the query tiles of one (sequence, KV head) re-read the same blocks, mostly from L2
constexpr int kLoadPolicy = 0;

constexpr int kWideWaves = 4;
constexpr int wg_waves(int split) { return split > 0 ? split : kWideWaves; }
constexpr int kBlock = 32;  // tokens
constexpr int kHalf = 16;   // tokens of half a block: on one page
constexpr int kBlockElems = kBlock * kHeadDim;
constexpr int kNowhere = 0x7ffffff0;  // a byte offset past every range
constexpr int kHeld = 64;   // half blocks whose cache rows a wave holds

// what a kernel changes of the scores
enum Change { kPlain, kBias, kCap, kCapBias };

// The cap of one-term weights is 1 - 2 / (e^2y + 1), which loses up to 3.5 * 2^-23 of the cap:
// the reciprocal, the sum below it and the maximum taken off cost 2^-23 each, exp2 half of
// that.  A weight is off by as much of itself: 2.1e-4 at this cap, a twentieth of what its
// rounding may cost (2^-8).  (Where slopes below zero make the maximum larger than the cap,
// taking it off costs 2^-24 of it: a bias of 10,000 is 6e-4.)  Calls with larger caps take the kernels of two-term weights,
// whose cap keeps a score's own precision: 16 new tokens over 20,000 29.1 us (30.5 with a
// cap of 512), 1,024 over 4,000 169 (134).  One-term kernels with that cap, in wide
// workgroups of one tile alone, took 479 and 155 us.
constexpr float kFarFrom = 512.f;

struct PagedPlan {
  const int32_t *block_tables, *lens, *q_starts, *q_lens;
  const int32_t *prefix_lens, *doc_starts;  // or null
  const float* slopes;
  int32_t window;  // or 0
  int32_t max_pages, num_pages;
  Divisor page_tokens;
  int32_t total_q, max_q_len;
  int32_t hq;
  Divisor hkv, group;
  Divisor tiles;       // workgroups per (sequence, KV head)
  int32_t num_seqs;
  int32_t units;       // sequences x KV heads
  Divisor rest;        // of them over whole XCDs, or 1
  int32_t last_first;  // the most work first
  int32_t splits;      // workgroups that share the blocks of a tile; with more than one their
  float* o_ws;         // partial outputs [splits, total_q, hq, D] and
  float2* ml_ws;       // (maximum, sum) pairs go to the workspace
  float factor;        // of the product in log2 units, without a cap
  float cap_in, cap_in2, cap_out;  // scale / cap, twice that and cap in log2 units
};

// the least or largest over a row of 16 lanes, by rotations; the rows of a wave hold the
// same columns
template <bool kMin>
__device__ __forceinline__ int columns_extreme(int x) {
  const auto with = [&](int y) { x = kMin ? (x < y ? x : y) : (x > y ? x : y); };
  with(__builtin_amdgcn_mov_dpp(x, 0x128, 0xf, 0xf, false));
  with(__builtin_amdgcn_mov_dpp(x, 0x124, 0xf, 0xf, false));
  with(__builtin_amdgcn_mov_dpp(x, 0x122, 0xf, 0xf, false));
  with(__builtin_amdgcn_mov_dpp(x, 0x121, 0xf, 0xf, false));
  return __builtin_amdgcn_readfirstlane(x);
}

// The sequence with k longer ones before it (in units of 128 tokens up to 2^10 of them;
// the first first where they are equal), for up to 64: bit by bit of the length, from the
// top, the half of the candidates that holds it.  More are taken as they come: 100 of 100 new
// tokens over 1,000..12,000 1,527 us, 1,369 if the caller has put the longest first; 65
// 1,052 and 976.
__device__ __forceinline__ int nth_longest(const int32_t* __restrict__ lens, int num_seqs, int k, int lane) {
  constexpr int kBits = 10;
  constexpr int kLenUnit = 128;
  int len = lane < num_seqs ? lens[lane] : 0;
  len = len < 0 ? 0 : len / kLenUnit < (1 << kBits) - 1 ? len / kLenUnit : (1 << kBits) - 1;
  unsigned long long left = __ballot(lane < num_seqs);
#pragma unroll
  for (int bit = kBits - 1; bit >= 0; --bit) {
    const unsigned long long ones = left & __ballot(len >> bit & 1);
    const int n = __builtin_popcountll(ones);
    if (k < n) {
      left = ones;
    } else {
      k -= n;
      left &= ~ones;
    }
  }
  const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(left >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)left, 0u));
  return __builtin_ctzll(__ballot((left >> lane & 1) && before == k));
}

// kTerms: bf16 terms of each softmax weight, 1, 2 (16 bits) or 3 (24).  kSplit: 0 for wide
// workgroups, or the waves of a narrow one.  kTiles: 16-column tiles per wave.
template <typename OutT, int kTerms, int kChange, int kSplit, int kTiles>
__global__ __launch_bounds__(64 * wg_waves(kSplit)) __attribute__((amdgpu_waves_per_eu(2))) void prefill_paged_kernel(
    const uint16_t* __restrict__ q, const uint16_t* __restrict__ kc, const uint16_t* __restrict__ vc, PagedPlan pp,
    OutT* __restrict__ out) {
  constexpr bool kSplitKv = kSplit > 0;
  constexpr int kWaves = wg_waves(kSplit);
  constexpr bool kHasBias = (kChange & 1) != 0;
  constexpr bool kHasCap = kChange >= kCap;
  constexpr int kCols = (kSplitKv ? 1 : kWaves) * kTiles * 16;
  constexpr int kStagers = kSplitKv ? 1 : kWaves;  // waves that stage a block together
  constexpr int kRounds = kHalf / (4 * kStagers);  // loads per thread and half block
  constexpr int kLoads = 2 * kRounds;              // and block, of K and of V
  constexpr float kHeadroom = kLazyRescale;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col_wave = kSplitKv ? 0 : wave;
  const int stage_wave = kSplitKv ? 0 : wave;
  const int n = lane & 15;
  const int c = lane >> 4;
  const int g = pp.group.d;
  // Workgroups are dealt to the XCDs in turn.  Eight units at a time have one XCD each,
  // whose L2 serves their tiles' re-reads; the tiles of the units left over (all of them,
  // with fewer than 8) go to the XCDs in turn.  In a grid that is not resident at once the
  // last tile, which sees the most tokens, goes first, and of up to 64 sequences the longest.
  const int whole_units = pp.units & ~(kXcds - 1);
  const int whole_blocks = whole_units * pp.tiles.d;
  int tile, unit;
  const int share = pp.splits > 1 ? (int)blockIdx.x / (pp.tiles.d * pp.units) : 0;  // of the blocks
  const int block = (int)blockIdx.x - share * (pp.tiles.d * pp.units);
  if (block < whole_blocks) {
    const int slot = block / kXcds;
    const int eight = pp.tiles.of(slot);
    tile = slot - eight * pp.tiles.d;
    unit = eight * kXcds + block % kXcds;
  } else {
    const int at = block - whole_blocks;
    tile = pp.rest.of(at);
    unit = whole_units + at - tile * pp.rest.d;
  }
  int b = pp.hkv.of(unit);
  const int kv = unit - b * pp.hkv.d;
  if (pp.last_first) {
    tile = pp.tiles.d - 1 - tile;
    if (pp.num_seqs > 1 && pp.num_seqs <= 64) b = nth_longest(pp.lens, pp.num_seqs, b, lane);
  }
  const int new_tokens = pp.q_lens[b];
  const int nq = new_tokens < pp.max_q_len ? new_tokens : pp.max_q_len;
  const int first_q = pp.group.of(tile * kCols);
  if (first_q >= nq) return;  // the whole workgroup
  const int row0 = pp.q_starts[b];
  const int seq_len = pp.lens[b] < 0 ? 0 : pp.lens[b];
  const int hist = seq_len - new_tokens;  // position of query 0
  const int64_t named = (int64_t)pp.max_pages * pp.page_tokens.d;
  int tokens = seq_len < named ? seq_len : (int)named;  // that the table can name
  tokens = tokens < kMostTokens ? tokens : kMostTokens;
  int prefix = pp.prefix_lens != nullptr ? pp.prefix_lens[b] : 0;
  prefix = prefix < 0 ? 0 : prefix < tokens ? prefix : tokens;
  const size_t row_elems = (size_t)pp.hkv.d * kHeadDim;
  const int row_bytes = (int)(row_elems * 2);
  const uint16_t* const khead = kc + (size_t)kv * kHeadDim;
  const uint16_t* const vhead = vc + (size_t)kv * kHeadDim;

  constexpr int kStageElems = (kSplitKv ? kWaves : 1) * kBlockElems;
  __shared__ __attribute__((aligned(16))) uint16_t lds_k0[kStageElems];
  __shared__ __attribute__((aligned(16))) uint16_t lds_v0[kStageElems];

  // first element of the query (and output) row of the workgroup's column col, -1 if it has none
  auto row_at = [&](int col) -> int64_t {
    const int at = tile * kCols + col;
    const int qi = pp.group.of(at);
    const int64_t row = (int64_t)row0 + qi;
    return qi < nq && row >= 0 && row < pp.total_q ? (row * pp.hq + kv * g + (at - qi * g)) * kHeadDim : -1;
  };
  // This lane's query column in each tile: the tokens low .. last that
  // it sees past the prefix (low = INT_MAX: none).  `last` is also where a bias is 0.
  int low[kTiles], last[kTiles];
  float slope[kTiles];
  bf16x8 qb[kTiles][4];
  // over the wave's rows: what some row sees past the prefix, what all see
  int some_low = INT_MAX, some_last = -1, all_low = 0, all_last = INT_MAX;
  int gap = INT_MAX;  // first position that its own row does not see
#pragma unroll
  for (int ct = 0; ct < kTiles; ++ct) {
    const int col = (col_wave * kTiles + ct) * 16 + n;
    const int64_t at = row_at(col);
    const bool valid = at >= 0;
    const int qi = pp.group.of(tile * kCols + col);
    const int head = kv * g + (tile * kCols + col - qi * g);
    const int64_t row = (int64_t)row0 + qi;
    const int p = hist + qi;
    low[ct] = 0;
    last[ct] = 0;
    slope[ct] = 0.f;
    bool sees_own = qi >= nq;  // or is no row
    if (valid) {
      const int doc = pp.doc_starts != nullptr ? pp.doc_starts[row] : 0;
      int lo = pp.window > 0 && p >= pp.window ? p - pp.window + 1 : 0;
      lo = doc > lo ? doc : lo;
      if (kHasBias) slope[ct] = pp.slopes[head] * 1.4426950408889634f;
      const int end = p < tokens ? p : tokens - 1;  // last token past the prefix
      if (lo <= end) {
        low[ct] = lo;
        last[ct] = p;
        some_low = lo < some_low ? lo : some_low;
        some_last = end > some_last ? end : some_last;
        sees_own = true;
      } else {
        low[ct] = INT_MAX;
        last[ct] = p < prefix ? p : prefix - 1;
      }
      all_low = low[ct] > all_low ? low[ct] : all_low;
      all_last = last[ct] < all_last ? last[ct] : all_last;
      const uint16_t* qrow = q + at + 8 * c;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) qb[ct][kk] = as_bf16x8(load16(qrow + 32 * kk));
    } else {
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) qb[ct][kk] = as_bf16x8(u32x4{0u, 0u, 0u, 0u});
    }
    gap = !sees_own && p < gap ? p : gap;
  }
  some_low = columns_extreme<true>(some_low);
  some_last = columns_extreme<false>(some_last);
  all_low = columns_extreme<false>(all_low);
  all_last = columns_extreme<true>(all_last);
  gap = columns_extreme<true>(gap);
  // the same over the workgroup: the tokens it reads
  int first = some_low, until = some_last + 1;
  if constexpr (!kSplitKv) {
    __shared__ int lds_seen[3][kWaves];
    if (lane == 0) {
      lds_seen[2][wave] = gap;
      lds_seen[0][wave] = some_low;
      lds_seen[1][wave] = some_last + 1;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      first = lds_seen[0][w] < first ? lds_seen[0][w] : first;
      until = lds_seen[1][w] > until ? lds_seen[1][w] : until;
      gap = lds_seen[2][w] < gap ? lds_seen[2][w] : gap;
    }
    gap = __builtin_amdgcn_readfirstlane(gap);
    first = __builtin_amdgcn_readfirstlane(first);
    until = __builtin_amdgcn_readfirstlane(until);
  }
  const int end = until > prefix ? until : prefix;  // tokens from here on are not seen
  // From gap on there may be tokens between first and until that no row sees: a padding
  // row's position, unless a later row's document takes it in.
  const bool gaps = gap < until && prefix < until;
  const int own = gaps ? hist + first_q : INT_MAX;  // position of the workgroup's first row
  __shared__ uint8_t lds_hidden[kCols + kBlock];    // whether own, own + 1, ... are such tokens
  if (gaps) {
    const int past = pp.group.of((tile + 1) * kCols + g - 1);  // the first row that the workgroup has no part of
    const int rows = (past < nq ? past : nq) - first_q;
    for (int i = tid; i < rows; i += 64 * kWaves) {
      bool seen = false;
      for (int r = i; r < rows && !seen; ++r) {
        const int64_t row = (int64_t)row0 + first_q + r;
        if (row < 0 || row >= pp.total_q) continue;
        const int doc = pp.doc_starts != nullptr ? pp.doc_starts[row] : 0;
        seen = doc <= own + i && (pp.window == 0 || r - i < pp.window);
      }
      lds_hidden[i] = !seen;
    }
    __syncthreads();
  }
  const int hole = (prefix + kBlock - 1) & -kBlock;
  const int skip = first < until && (first & -kBlock) > hole ? (first & -kBlock) - hole : 0;
  const int v_end = end - skip;
  auto token = [&](int v) { return v < hole ? v : v + skip; };
  // The wave's bounds in flattened tokens.  Tokens before the hole are the prefix's: no
  // token past it is there unless skip is 0.
  const int some_from = some_low - skip, some_to = some_last - skip;
  const int all_from = all_low - skip, all_to = all_last - skip;
  // Blocks are taken from the first on, with a bias from the last on: where scores
  // fall with the distance, the maxima hardly move once the nearest block is done (steep
  // heads raised them in every block).
  const int blocks_end = (v_end + kBlock - 1) & -kBlock;
  // this workgroup's share of them
  const int per_share = pp.splits > 1 ? (blocks_end / kBlock + pp.splits - 1) / pp.splits * kBlock : blocks_end;
  const int share_from = share * per_share;
  const int share_end = share_from + per_share < blocks_end ? share_from + per_share : blocks_end;
  auto block_at = [&](int u) { return kHasBias ? blocks_end - kBlock - u : u; };

  // The maxima start at the largest bias of the column: where biases grow with the
  // distance, the first scores are rounded near it and not near 0.
  Softmax st[kTiles];
  int unset = (1 << kTiles) - 1;  // bit ct: the column has seen no token yet
  f32x4 o[kTiles][8];
#pragma unroll
  for (int ct = 0; ct < kTiles; ++ct) {
    st[ct] = Softmax{0.f, 0.f};
    if (kHasBias && slope[ct] < 0.f) {
      const int back = prefix > 0 ? last[ct] : last[ct] - (low[ct] < last[ct] ? low[ct] : last[ct]);
      const int ahead = prefix - 1 - last[ct];
      st[ct].m = -slope[ct] * (float)(back > ahead ? back : ahead);
    }
#pragma unroll
    for (int nb = 0; nb < 8; ++nb) o[ct][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // Of the halves of the wave's next kHeld / 2 blocks, from `held` of the order on, one per
  // lane: its first cache row / 16, whether it may have tokens past the prefix that no row
  // sees (kEdge), and its tokens before the end; 0 outside the cache and past the end.
  constexpr uint32_t kEdge = 32;
  constexpr int kStep = kSplitKv ? kWaves * kBlock : kBlock;  // between a wave's blocks
  int held = 0;
  uint32_t halves = 0;
  auto look_up = [&](int u) __attribute__((always_inline)) {
    held = u;
    halves = 0;
    int half = lane;
    asm volatile("" : "+v"(half));  // nothing of this is kept in a register for the next time
    const int mine = u + (half >> 1) * kStep;
    const int at = block_at(mine) + (half & 1) * kHalf;
    const int t = token(at);
    if (mine < share_end && at < v_end) {
      const int j = pp.page_tokens.of(t);
      if (j < pp.max_pages) {
        const int page = pp.block_tables[(size_t)b * pp.max_pages + j];
        if (page >= 0 && page < pp.num_pages) {
          const int row = page * pp.page_tokens.d + (t - j * pp.page_tokens.d);
          const uint32_t edge = ((t < first) | (t + kHalf > own)) && t + kHalf > prefix ? kEdge : 0u;
          halves = (uint32_t)(row / kHalf) << 6 | edge | (uint32_t)(end - t < kHalf ? end - t : kHalf);
        }
      }
    }
  };
  // A block load writes lane L's 16 bytes at LDS base + 16 L: round r of wave w fills
  // slots 0..15 of tokens (r kStagers + w) 4 + L / 16 of a half block, so each lane fetches
  // the chunk that the swizzle puts at its slot (the swizzle repeats every 16 tokens).
  int offset[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int tok = (r * kStagers + stage_wave) * 4 + (lane >> 4);
    offset[r] = tok * row_bytes + (((lane & 15) ^ tile_swizzle(tok)) << 4);
  }
  // the words of the halves of the block at u of the order, looked up if need be
  struct Words {
    uint32_t h[2];
  };
  auto words_at = [&](int u) __attribute__((always_inline)) {
    if (u - held >= kHeld / 2 * kStep) look_up(u);
    const int i = (int)((uint32_t)(u - held) / (kStep / 2));
    return Words{{(uint32_t)__builtin_amdgcn_readlane((int)halves, i), (uint32_t)__builtin_amdgcn_readlane((int)halves, i + 1)}};
  };
  auto absent_of = [](const Words& w) { return ((w.h[0] & 31) == 0 ? 1 : 0) | ((w.h[1] & 31) == 0 ? 2 : 0); };
  // A block's loads, one instruction stream for every block (with a stream of its own for
  // ordinary blocks the compiler lost count of the loads in flight and waited for all):
  // outside the cache, past the end and, of values, where no row sees the token zeros are
  // written.  (Whatever keys give there is masked.)
  auto load_block = [&](const uint16_t* base, bool values, const Words& w, int u, uint16_t* dst)
      __attribute__((always_inline)) {
    int off[2][kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) off[0][r] = off[1][r] = offset[r];
    if (values && ((w.h[0] | w.h[1]) & kEdge)) {
      int at = lane >> 4;
      asm volatile("" : "+v"(at));  // a branch: nothing of it worked out for every block
      const int t = token(block_at(u));
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
          const int x = t + h * kHalf + (r * kStagers + stage_wave) * 4 + at;
          // x < until + kBlock, which own has kCols tokens before at most
          if (x >= prefix && (x >= own ? lds_hidden[x - own] != 0 : x < first)) off[h][r] = kNowhere;
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const char* from = reinterpret_cast<const char*>(base) + (uint64_t)(w.h[h] >> 6) * (uint32_t)(kHalf * row_bytes);
      const __amdgpu_buffer_rsrc_t rs =
          make_rsrc(reinterpret_cast<const uint16_t*>(from), (w.h[h] & 31) * (uint32_t)row_bytes);
#pragma unroll
      for (int r = 0; r < kRounds; ++r)
        load16_to_lds<kLoadPolicy>(rs, dst + h * kHalf * kHeadDim + (r * kStagers + stage_wave) * 4 * kHeadDim, off[h][r]);
    }
  };

  // per-lane LDS offsets of the operand reads within a 16-token half block
  int k_off[4];
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) k_off[kk] = n * kHeadDim + (((4 * kk + c) ^ tile_swizzle(n)) << 3);
  const int v_tok = 4 * c + (n >> 2);
  const int v_row = v_tok * kHeadDim + 4 * (n & 1);
  const int v_swz = tile_swizzle(v_tok);
  const int v_ch = (n & 3) >> 1;

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

  // The scores in log2 units less the running maxima, -inf where a token is not seen.
  // v: the block's flattened token; whole: every column sees every token; absent: bit h
  // where half h is on no page.
  auto relative = [&](int v, bool whole, int absent, f32x4 (&sc)[kTiles][2]) __attribute__((always_inline)) {
    const int t0 = token(v);
    // no token lies behind a query; otherwise the distances are absolute
    const bool before = !kHasBias || t0 + kBlock - 1 <= all_last;
    // every score becomes change(score, what is added to it)
    auto each = [&](float more, auto&& change) __attribute__((always_inline)) {
      if (before) {
#pragma unroll
        for (int ct = 0; ct < kTiles; ++ct) {
          const float less = more - st[ct].m;
          const float base = kHasBias ? fmaf(slope[ct], (float)(t0 + 4 * c - last[ct]), less) : less;
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              sc[ct][h][i] = change(sc[ct][h][i], kHasBias ? fmaf(slope[ct], (float)(16 * h + i), base) : base);
        }
      } else {
#pragma unroll
        for (int ct = 0; ct < kTiles; ++ct) {
          const int d = t0 + 4 * c - last[ct];
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              sc[ct][h][i] = change(sc[ct][h][i], fmaf(-slope[ct], fabsf((float)(d + 16 * h + i)), more - st[ct].m));
        }
      }
    };
    if constexpr (!kHasCap) {
      each(0.f, [&](float x, float add) __attribute__((always_inline)) { return fmaf(x, pp.factor, add); });
    } else if constexpr (kTerms == 1) {
      // tanh(y) = 1 - 2 / (e^2y + 1): off by what kFarFrom allows for.  (An odd polynomial
      // up to |y| = 1, 7 instructions for 5, and a test whether a block's scores all lie
      // there took as long: 100 requests over long contexts 790 TFLOP/s with either; one,
      // with large scores among them, 100 us against 95.)
      each(pp.cap_out, [&](float x, float add) __attribute__((always_inline)) {
        return fmaf(__builtin_amdgcn_rcpf(fast_exp2(x * pp.cap_in2) + 1.0f), -2.0f * pp.cap_out, add);
      });
    } else {
      float most = 0.f;
#pragma unroll
      for (int ct = 0; ct < kTiles; ++ct)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) most = fmaxf(most, fabsf(sc[ct][h][i]));
      if (!__any(most * fabsf(pp.cap_in) > kTanhSmall)) {
        each(0.f, [&](float x, float add) __attribute__((always_inline)) {
          return fmaf(tanh_small(x * pp.cap_in), pp.cap_out, add);
        });
      } else {
        each(0.f, [&](float x, float add) __attribute__((always_inline)) {
          return fmaf(tanh_any(x * pp.cap_in), pp.cap_out, add);
        });
      }
    }
    if (!whole) {
#pragma unroll
      for (int ct = 0; ct < kTiles; ++ct)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int t = t0 + 16 * h + 4 * c + i;
            // no short circuits: they became branches around every score
            const bool see = (int)((t < prefix) | ((t >= low[ct]) & (t <= last[ct]))) & ~(absent >> h);
            sc[ct][h][i] = see ? sc[ct][h][i] : -INFINITY;
          }
    }
  };
  // raises the maxima where a score passes its limit
  auto raise = [&](f32x4 (&sc)[kTiles][2]) __attribute__((always_inline)) {
    // a score above the limit moves the maximum: 2^8 above it, or any where there is none
    float lm[kTiles];
    bool over = false;
#pragma unroll
    for (int ct = 0; ct < kTiles; ++ct) {
      lm[ct] = max8(sc[ct][0], sc[ct][1]);
      over |= lm[ct] > kHeadroom;
    }
    if (!__any(over | (unset != 0))) return;
#pragma unroll
    for (int ct = 0; ct < kTiles; ++ct) {
      const bool fresh = unset >> ct & 1;
      if (!__any(lm[ct] > (fresh ? -INFINITY : kHeadroom))) continue;
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
        // the row sum adds the rounded weights that the product uses, a pair per dot product with (1, 1)
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
  // O^T += V^T P^T: the K dimension holds tokens 4c .. 4c + 3 of both halves.  Raised wave
  // priority over the product stream, and the V^T reads of one dimension group ahead of
  // their products, as in the contiguous prefill.
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
  // the block at v whole: every column of the wave sees every token of it; some: any at all
  auto is_whole = [&](int v, int absent) {
    return absent == 0 && ((v >= all_from && v + kBlock - 1 <= all_to) || v + kBlock <= prefix);
  };
  auto is_some = [&](int v) { return v < prefix || (v <= some_to && v + kBlock > some_from); };

  const int u0 = share_from + (kSplitKv ? wave * kBlock : 0);  // this wave's first block
  look_up(u0);
  // The queries have arrived with the table's entries; said here, the compiler need not
  // wait for them in the loop, where that would be a wait for the blocks in flight too.
  __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
  if constexpr (!kSplitKv) {
    __shared__ __attribute__((aligned(16))) uint16_t lds_k1[kStageElems];
    __shared__ __attribute__((aligned(16))) uint16_t lds_v1[kStageElems];
    __shared__ __attribute__((aligned(16))) uint16_t lds_k2[kStageElems];
    __shared__ __attribute__((aligned(16))) uint16_t lds_v2[kStageElems];
    int absent = 0;  // bits 2j, 2j + 1: of the block j steps on
    auto issue = [&](int u, uint16_t* dk, uint16_t* dv, int ahead) __attribute__((always_inline)) {
      const Words w = words_at(u);
      absent |= absent_of(w) << (2 * ahead);
      load_block(khead, false, w, u, dk);
      load_block(vhead, true, w, u, dv);
    };
    // One block: wait for this wave's loads of it, then the barrier (every wave's loads
    // have landed, and every wave is done with the stage read in the previous step); the
    // loads of the block two ahead go into that stage.  The three stages are distinct LDS
    // arrays named at compile time, so the compiler's wait before the reads covers only
    // this stage's loads.
    auto step = [&](int u, const uint16_t* kt, const uint16_t* vt, uint16_t* nk, uint16_t* nv) __attribute__((always_inline)) {
      __builtin_amdgcn_s_waitcnt(wait_vmcnt(2 * kLoads));
      lds_barrier();
      const int gone = absent & 3;
      absent >>= 2;
      issue(u + 2 * kBlock, nk, nv, 1);
      const int v = block_at(u);
      if (u < blocks_end && is_some(v)) {
        f32x4 sc[kTiles][2];
        u32x4 pt[kTerms][kTiles];
        scores(kt, sc);
        relative(v, is_whole(v, gone), gone, sc);
        raise(sc);
        weights(sc, pt);
        values(vt, pt);
      }
    };
    issue(0, lds_k0, lds_v0, 0);
    issue(kBlock, lds_k1, lds_v1, 1);
    // whole rounds of three steps (an exit in the middle would make the compiler wait at
    // the loop's head); the last of them may be on empty blocks
    for (int u = 0; u < blocks_end; u += 3 * kBlock) {
      step(u, lds_k0, lds_v0, lds_k2, lds_v2);
      step(u + kBlock, lds_k1, lds_v1, lds_k0, lds_v0);
      step(u + 2 * kBlock, lds_k2, lds_v2, lds_k1, lds_v1);
    }
    // no load may land in LDS after the workgroup has released it
    __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
#pragma unroll
    for (int ct = 0; ct < kTiles; ++ct) {
      float l_tot = st[ct].l + __shfl_xor(st[ct].l, 16);
      l_tot += __shfl_xor(l_tot, 32);
      // found anew: kept since the start, the rows took registers that the loop needs
      int col = (wave * kTiles + ct) * 16 + n;
      asm volatile("" : "+v"(col));
      const int64_t at = row_at(col);
      if (at >= 0) {
        const float inv = l_tot != 0.f ? 1.0f / l_tot : 0.f;
        OutT* orow = out + at + 4 * c;
#pragma unroll
        for (int nb = 0; nb < 8; ++nb) store4<OutT>(orow + 16 * nb, o[ct][nb] * inv);
      }
    }
  } else {
    // Wave w takes blocks w, w + kWaves, ... through its own K and V tiles.  A tile is
    // refilled with the wave's next block as soon as it has been read.
    uint16_t* const kt = lds_k0 + wave * kBlockElems;
    uint16_t* const vt = lds_v0 + wave * kBlockElems;
    Words w = words_at(u0);
    load_block(khead, false, w, u0, kt);
    load_block(vhead, true, w, u0, vt);
    for (int u = u0; u < share_end; u += kStep) {
      const int v = block_at(u);
      f32x4 sc[kTiles][2];
      u32x4 pt[kTerms][kTiles];
      __builtin_amdgcn_s_waitcnt(wait_vmcnt(kLoads));  // this block's K; its V is still on the way
      asm volatile("" ::: "memory");
      scores(kt, sc);
      // the tile's reads have returned before its refill is issued
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      const int gone = absent_of(w);
      w = words_at(u + kStep);
      load_block(khead, false, w, u + kStep, kt);
      relative(v, is_whole(v, gone), gone, sc);
      raise(sc);
      weights(sc, pt);
      __builtin_amdgcn_s_waitcnt(wait_vmcnt(kLoads));  // this block's V
      asm volatile("" ::: "memory");
      values(vt, pt);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      load_block(vhead, true, w, u + kStep, vt);
    }
    __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
    __syncthreads();
    // Merge, half of the dimensions at a time: wave w puts its columns' maxima, sums and
    // unnormalised outputs into its part of the tiles, 16-byte chunk ch of column j at slot
    // ch ^ (j & 15), and every thread adds up 4 dimensions of some columns in wave order.
    constexpr int kDims = kHeadDim / 2;
    constexpr int kChunks = kDims / 4;
    constexpr int kPartFloats = kCols * kDims;  // then the sums, then the maxima
    static_assert((kPartFloats + 2 * kCols) * 4 <= 2 * kBlockElems * 2,
                  "a wave's partial results must fit half of a tile array");
    auto part_of = [&](int w) {
      constexpr int kPerArray = kWaves / 2;
      return reinterpret_cast<float*>((w < kPerArray ? lds_k0 : lds_v0) + w % kPerArray * 2 * kBlockElems);
    };
    float* const mine = part_of(wave);
#pragma unroll
    for (int ct = 0; ct < kTiles; ++ct) {
      float l_tot = st[ct].l + __shfl_xor(st[ct].l, 16);
      l_tot += __shfl_xor(l_tot, 32);
      if (c == 0) {
        mine[kPartFloats + ct * 16 + n] = l_tot;
        mine[kPartFloats + kCols + ct * 16 + n] = (unset >> ct & 1) ? -INFINITY : st[ct].m;
      }
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (half > 0) __syncthreads();  // the first half has been read
#pragma unroll
      for (int ct = 0; ct < kTiles; ++ct)
#pragma unroll
        for (int nb = 0; nb < 4; ++nb)
          *reinterpret_cast<f32x4*>(mine + (ct * 16 + n) * kDims + (((4 * nb + c) ^ n) << 2)) = o[ct][4 * half + nb];
      __syncthreads();
      const int ch = tid % kChunks;
#pragma unroll
      for (int j = tid / kChunks; j < kCols; j += 64 * kWaves / kChunks) {
        const int64_t at = row_at(j);
        if (at < 0) continue;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, part_of(w)[kPartFloats + kCols + j]);
        float l = 0.f;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float m = part_of(w)[kPartFloats + kCols + j];
          const float share = m > -INFINITY ? fast_exp2(m - top) : 0.f;
          l += share * part_of(w)[kPartFloats + j];
          acc += share * *reinterpret_cast<const f32x4*>(part_of(w) + j * kDims + ((ch ^ (j & 15)) << 2));
        }
        if (pp.splits > 1) {
          const int64_t part = share * pp.total_q * (int64_t)pp.hq + at / kHeadDim;
          *reinterpret_cast<f32x4*>(pp.o_ws + part * kHeadDim + half * kDims + 4 * ch) = acc;
          if (half == 0 && ch == 0) pp.ml_ws[part] = make_float2(top, l);
        } else {
          const float inv = l != 0.f ? 1.0f / l : 0.f;
          store4<OutT>(out + at + half * kDims + 4 * ch, acc * inv);
        }
      }
    }
  }
}

// Joins the shares of a tile's blocks: one wave per (row, head), two dimensions per lane,
// the shares' weights one per lane; in share order.
constexpr int kJoinWaves = 4;

template <typename OutT>
__global__ __launch_bounds__(64 * kJoinWaves) void prefill_join_kernel(PagedPlan pp, OutT* __restrict__ out) {
  const int lane = threadIdx.x & 63;
  const int64_t part = (int64_t)blockIdx.x * kJoinWaves + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  if (part >= (int64_t)pp.total_q * pp.hq) return;
  const int row = (int)(part / pp.hq);
  bool live = false;  // rows of no sequence have no shares
  for (int base = 0; base < pp.num_seqs && !live; base += 64) {
    const int b = base + lane;
    if (b < pp.num_seqs) {
      const int64_t i = (int64_t)row - pp.q_starts[b];
      live = i >= 0 && i < pp.q_lens[b] && i < pp.max_q_len;
    }
    live = __any(live);
  }
  if (!live) return;
  const int64_t stride = (int64_t)pp.total_q * pp.hq;
  const float2 ml = lane < pp.splits ? pp.ml_ws[part + lane * stride] : make_float2(-INFINITY, 0.f);
  float top = ml.x, sum = ml.y;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
  const float weight = ml.x > -INFINITY ? fast_exp2(ml.x - top) : 0.f;
  sum *= weight;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
  float a = 0.f, b = 0.f;
#pragma unroll 8
  for (int s = 0; s < pp.splits; ++s) {
    const float2 o = *reinterpret_cast<const float2*>(pp.o_ws + (part + s * stride) * kHeadDim + 2 * lane);
    const float w = __shfl(weight, s);
    a = fmaf(w, o.x, a);
    b = fmaf(w, o.y, b);
  }
  const float inv = sum != 0.f ? 1.0f / sum : 0.f;
  if constexpr (sizeof(OutT) == 4)
    *reinterpret_cast<float2*>(out + part * kHeadDim + 2 * lane) = make_float2(a * inv, b * inv);
  else
    *reinterpret_cast<uint32_t*>(out + part * kHeadDim + 2 * lane) = pack_bf16x2(a * inv, b * inv);
}

struct PagedArgs {
  const uint16_t *q, *k, *v;
  PagedPlan plan;
  void* out;
  unsigned grid;
  hipStream_t stream;
};

// most tiles per wave: three would not leave registers for more than one term
constexpr int most_tiles_of(int terms) { return terms > 1 ? 2 : 3; }

template <typename OutT, int kTerms, int kChange, int kSplit, int kTiles>
void launch_split(const PagedArgs& a) {
  hipLaunchKernelGGL((prefill_paged_kernel<OutT, kTerms, kChange, kSplit, kTiles>), dim3(a.grid),
                     dim3(64 * wg_waves(kSplit)), 0, a.stream, a.q, a.k, a.v, a.plan, static_cast<OutT*>(a.out));
}

template <typename OutT, int kTerms, int kChange>
void launch_change(const PagedArgs& a, int split, int tiles) {
  constexpr int kMostTiles = most_tiles_of(kTerms);
  if (split == 8) return launch_split<OutT, kTerms, kChange, 8, kMostTiles>(a);
  if (split == 4) return launch_split<OutT, kTerms, kChange, 4, kMostTiles>(a);
  if (tiles == 1) return launch_split<OutT, kTerms, kChange, 0, 1>(a);
  if (tiles == 2) return launch_split<OutT, kTerms, kChange, 0, 2>(a);
  launch_split<OutT, kTerms, kChange, 0, kMostTiles>(a);
}

template <typename OutT, int kTerms>
void launch_paged(const PagedArgs& a, int change, int split, int tiles) {
  if (change == kPlain)
    launch_change<OutT, kTerms, kPlain>(a, split, tiles);
  else if (change == kBias)
    launch_change<OutT, kTerms, kBias>(a, split, tiles);
  else if (change == kCap)
    launch_change<OutT, kTerms, kCap>(a, split, tiles);
  else
    launch_change<OutT, kTerms, kCapBias>(a, split, tiles);
  if (a.plan.splits > 1) {
    const int64_t parts = (int64_t)a.plan.total_q * a.plan.hq;
    hipLaunchKernelGGL((prefill_join_kernel<OutT>), dim3((unsigned)((parts + kJoinWaves - 1) / kJoinWaves)),
                       dim3(64 * kJoinWaves), 0, a.stream, a.plan, static_cast<OutT*>(a.out));
  }
}

}  // namespace

extern "C" int ctx_prefill_attn_run_paged(ctx_decode_attn* h, const void* q, const void* k_pages, const void* v_pages,
                                          int32_t num_pages, const int32_t* block_tables, int32_t max_pages_per_seq,
                                          const int32_t* seq_lens, const int32_t* q_starts, const int32_t* q_lens,
                                          int32_t num_seqs, int32_t total_q, int32_t max_q_len, float scale,
                                          const ctx_attn_scores* scores, void* out, void* stream) {
  int rc = check_common(h, num_seqs, scale);
  if (rc != CTX_OK) return rc;
  ctx_attn_scores sc{};
  if (scores != nullptr) sc = *scores;
  rc = check_scored(h, sc, scale, num_pages, max_pages_per_seq);
  if (rc != CTX_OK) return rc;
  sc.softcap = cap_of(sc, scale);
  if (total_q < 0 || max_q_len < 0)
    return fail(CTX_ERR_INVALID_ARG, "total_q and max_q_len must not be negative (%d, %d)", total_q, max_q_len);
  if (num_seqs == 0 || max_q_len == 0 || total_q == 0) return CTX_OK;
  if (q == nullptr || k_pages == nullptr || v_pages == nullptr || block_tables == nullptr || seq_lens == nullptr ||
      q_starts == nullptr || q_lens == nullptr || out == nullptr)
    return fail(CTX_ERR_INVALID_ARG, "NULL data pointer");
  if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out))
    return fail(CTX_ERR_ALIGNMENT, "q, k_pages, v_pages and out must be 16-byte aligned");
  rc = check_device(h);
  if (rc != CTX_OK) return rc;
  const ctx_decode_attn_desc& d = h->desc;
  const int g = d.num_q_heads / d.num_kv_heads;
  PagedPlan pp{};
  pp.block_tables = block_tables;
  pp.lens = seq_lens;
  pp.q_starts = q_starts;
  pp.q_lens = q_lens;
  pp.prefix_lens = sc.prefix_lens;
  pp.doc_starts = sc.doc_starts;
  pp.slopes = sc.slopes;
  pp.window = sc.window;
  pp.max_pages = max_pages_per_seq;
  pp.num_pages = num_pages;
  pp.page_tokens = Divisor(d.page_tokens);
  pp.total_q = total_q;
  pp.max_q_len = max_q_len < total_q ? max_q_len : total_q;
  pp.hq = d.num_q_heads;
  pp.hkv = Divisor(d.num_kv_heads);
  pp.group = Divisor(g);
  pp.num_seqs = num_seqs;
  pp.factor = (float)((double)scale * 1.4426950408889634);
  pp.cap_in = sc.softcap > 0.f ? scale / sc.softcap : 0.f;
  pp.cap_in2 = (float)((double)pp.cap_in * 2.8853900817779268);
  pp.cap_out = (float)((double)sc.softcap * 1.4426950408889634);
  const int64_t cols = (int64_t)pp.max_q_len * g;
  const int64_t units = (int64_t)num_seqs * d.num_kv_heads;
  const auto grid_of = [&](int64_t wg_cols) { return units * ((cols + wg_cols - 1) / wg_cols); };
  const int64_t cus = h->num_cus;
  // most tokens that a row can see, as far as the host knows.  A handle for contexts far
  // longer than a call's gets that call a kernel made for long ones: with max_seq_len 32,768
  // instead of the longest context 16 fresh tokens 17.1 us for 9.7, 4 requests with 5 over
  // 100 25.4 for 8.8, 400 fresh ones 15.0 for 13.1; from 1,000 tokens of context on the same.
  const int terms = d.out_dtype == CTX_DTYPE_F32                                        ? 3
                    : (sc.flags & CTX_SCORES_SPLIT_P) != 0 || sc.softcap > kFarFrom ? 2
                                                                                      : 1;
  const int most_tiles = most_tiles_of(terms);
  int64_t context = d.max_seq_len;
  if (sc.window > 0 && sc.prefix_lens == nullptr && (int64_t)sc.window + most_tiles * 16 < context)
    context = (int64_t)sc.window + most_tiles * 16;
  // Narrow workgroups as long as all of them are resident at once (two of 4 waves per
  // CU), as in the contiguous prefill: in a second round each pays its start and its merge
  // again.  With one per CU or fewer they have 8 waves: 256 new tokens over 4,000 34 us (4
  // waves 42, wide 82).  Not for short contexts, which leave a wave few blocks: 400 fresh
  // tokens 13.5 us wide, 15.8 narrow.
  const int64_t narrow = grid_of(most_tiles * 16);
  const int split = context <= 16 * kBlock || narrow > 2 * cus ? 0 : narrow > cus ? 4 : 8;
  // Wide ones have fewer tiles per wave where there would be too few to fill the chip: one
  // tile as long as all workgroups are resident (three per CU), two (of three) as long as
  // about all are (two per CU).  Of 1, 2 and 3 tiles: 1,024 new tokens over 4,000 117, 124
  // and 149 us, 2,048 248, 186 and 209, 4,096 484, 395 and 397; 8 requests with up to 120 over
  // 600 24, 26 and 32, with up to 300 54, 59 and 46.
  const auto wide = [&](int t) { return grid_of(kWideWaves * t * 16); };
  const int tiles = split > 0             ? most_tiles
                    : wide(1) <= 3 * cus ? 1
                    : most_tiles > 2 && 4 * wide(2) <= 9 * cus ? 2
                                                               : most_tiles;
  // Where 8-wave workgroups are fewer than the CUs several share a tile's blocks, through
  // the workspace and a second launch: as many as fit there, leave each a context of 512
  // tokens and the join a wave's lanes.  16 new tokens over 20,000 29 us (142 alone).  With
  // 256, 512 and 1,024 tokens: 16 over 2,000 15.8, 17.7 and 19.9 us, over 4,000 20.6, 18.9 and
  // 20.8, over 8,000 22.7, 22.5 and 21.7; 5 over 3,000 14.9, 15.1 and 19.1.
  pp.splits = 1;
  if (split == 8) {
    const int64_t slots = h->max_ranges + d.max_batch;
    int64_t most = cus / narrow;
    most = slots / total_q < most ? slots / total_q : most;
    most = context / 512 < most ? context / 512 : most;
    most = most < 64 ? most : 64;
    if (most > 1) pp.splits = (int32_t)most;
  }
  pp.o_ws = h->o_ws;
  pp.ml_ws = h->ml_ws;
  const int64_t blocks = split > 0 ? narrow * pp.splits : wide(tiles);
  // kMostTokens: indexes past the last stay in 32 bits
  if (units > kMostTokens || blocks > kMostTokens || cols > kMostTokens)
    return fail(CTX_ERR_INVALID_ARG, "prefill grid too large");
  pp.units = (int32_t)units;
  pp.tiles = Divisor((int32_t)(blocks / pp.splits / units));
  pp.rest = Divisor(units % kXcds > 0 ? (int32_t)(units % kXcds) : 1);
  pp.last_first = split == 0 && blocks > 2 * cus;
  const PagedArgs a{static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(k_pages),
                    static_cast<const uint16_t*>(v_pages), pp, out, (unsigned)blocks,
                    reinterpret_cast<hipStream_t>(stream)};
  const int change = (sc.softcap > 0.f ? kCap : kPlain) + (sc.slopes != nullptr ? kBias : kPlain);
  if (terms == 3)
    launch_paged<float, 3>(a, change, split, tiles);
  else if (terms == 2)
    launch_paged<uint16_t, 2>(a, change, split, tiles);
  else
    launch_paged<uint16_t, 1>(a, change, split, tiles);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "kernel launch");
  return CTX_OK;
}
