// ctx_kv_pages.hip -- the pages of paged caches for gfx950 (MI355X): forked, grown, trimmed
// and freed rows of a block table with counts of the pages' use, and the copies and
// compaction of the data, behind the C ABI declared in include/ctx_kv_pages.h.
//
//   * Counts change by integer atomics, whose order does not matter; pages are handed out
//     the lowest first, by a prefix sum over the rows' needs and one over the free
//     pages, so that what a call does depends on its inputs alone.  (A stack of free
//     pages would need no pass over the counts, but its order would follow that of the
//     atomics.)
//   * A resize of more than a few short rows takes three launches: the pages given back (a
//     workgroup per row), the needs and the free pages (one workgroup: 4 bytes a page, read if
//     anything grows, and again past 65,536 pages), and the tables (a workgroup per row).  Bound
//     by the latency of loads that follow from each other: a workgroup plans 256 rows of 512 pages in 14 us.
//   * Compaction is in place.  A token moves to a place no later than its own, so the
//     places that the first i tokens go to hold, of what is still needed, only these
//     tokens themselves: a workgroup takes one head of one sequence's keys or values
//     through blocks of tokens in order, and writes a block once all of it has been read.

#include <hip/hip_runtime.h>

#include <cstdint>

#include "ctx_attn_common.h"
#include "ctx_kv_pages.h"

namespace {

struct Rows {
  int32_t* tables;
  int32_t max_pages, page_tokens, num_seqs;
  int32_t* refs;
  int32_t num_pages;
};

__device__ __forceinline__ int64_t clipped(const Rows& r, int32_t len) {
  const int64_t most = (int64_t)r.max_pages * r.page_tokens;
  return len < 0 ? 0 : len < most ? len : most;
}
__device__ __forceinline__ int pages_of(const Rows& r, int64_t len) {
  return (int)((len + r.page_tokens - 1) / r.page_tokens);
}
__device__ __forceinline__ bool is_page(const Rows& r, int32_t page) { return page >= 0 && page < r.num_pages; }
__device__ __forceinline__ void count(const Rows& r, int32_t page, int by) {
  if (is_page(r, page)) atomicAdd(r.refs + page, by);
}

// ------------------------------------------------------------ fork

constexpr int kRowThreads = 256;

__device__ __forceinline__ bool forks(const int32_t* parents, int num_seqs, int b) {
  const int p = parents[b];
  return p >= 0 && p < num_seqs && p != b;
}

// One workgroup per row.  A row is written only by its own workgroup, and no row that is
// written is another's parent.
__global__ __launch_bounds__(kRowThreads) void fork_kernel(Rows r, int32_t* lens, const int32_t* __restrict__ parents) {
  const int b = blockIdx.x;
  if (!forks(parents, r.num_seqs, b)) return;
  const int p = parents[b];
  if (forks(parents, r.num_seqs, p)) return;
  const int32_t len = lens[p];
  const int had = pages_of(r, clipped(r, lens[b])), get = pages_of(r, clipped(r, len));
  int32_t* const row = r.tables + (size_t)b * r.max_pages;
  const int32_t* const from = r.tables + (size_t)p * r.max_pages;
  for (int j = threadIdx.x; j < r.max_pages; j += kRowThreads) {
    if (j < had) count(r, row[j], -1);
    const int32_t page = j < get ? from[j] : -1;
    row[j] = page;
    count(r, page, 1);
  }
  __syncthreads();  // all have read the row's own length
  if (threadIdx.x == 0) lens[b] = len;
}

// ------------------------------------------------------------ resize

struct Resize {
  Rows rows;
  const int32_t *lens, *new_lens;
  int32_t *granted, *copies;
  int32_t* offsets;  // [num_seqs] into fresh, -1: not granted
  int32_t* copied;   // [num_seqs] whether the first of them replaces the last page
  int32_t* fresh;    // [num_pages] the free pages that are handed out
};

// The pages past row b's new length, by `threads` threads.
__device__ __forceinline__ void give_back(const Resize& a, int b, int tid, int threads) {
  const Rows& r = a.rows;
  const int had = pages_of(r, clipped(r, a.lens[b])), get = pages_of(r, clipped(r, a.new_lens[b]));
  int32_t* const row = r.tables + (size_t)b * r.max_pages;
  for (int j = get + tid; j < had; j += threads) {
    count(r, row[j], -1);
    row[j] = -1;
  }
}

__global__ __launch_bounds__(kRowThreads) void give_back_kernel(Resize a) {
  give_back(a, blockIdx.x, threadIdx.x, kRowThreads);
}

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;
constexpr int kPlanLoads = 8;  // of counts, per thread at once
constexpr int32_t kSmallRows = kPlanWaves, kSmallWidth = 256;  // rows and entries of a row that one launch resizes

// Sum of x over the threads before this one; *total over all.
__device__ __forceinline__ int64_t scan(int64_t x, int64_t* lds, int64_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t sum = x;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int64_t y = __shfl_up(sum, off);
    if (lane >= off) sum += y;
  }
  __syncthreads();  // lds is free
  if (lane == 63) lds[wave] = sum;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    before += w < wave ? lds[w] : 0;
    all += lds[w];
  }
  *total = all;
  return before + sum - x;
}

// Who gets which free pages, by one workgroup.
__device__ __forceinline__ void plan(const Resize& a, int64_t* lds_scan) {
  const Rows& r = a.rows;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // pages that row b needs, whether the first replaces its last one, and whether it can have them at all
  struct Need {
    int pages;
    bool again, fits;
  };
  auto need_of = [&](int b) {
    Need x{0, false, false};
    if (b >= r.num_seqs) return x;
    const int64_t len = clipped(r, a.lens[b]);
    const int64_t want = a.new_lens[b] < 0 ? 0 : a.new_lens[b];
    x.fits = want <= (int64_t)r.max_pages * r.page_tokens;
    if (!x.fits || want <= len) return x;
    const int had = pages_of(r, len);
    if (len % r.page_tokens > 0) {
      const int32_t last = r.tables[(size_t)b * r.max_pages + had - 1];
      x.again = is_page(r, last) && r.refs[last] > 1;
    }
    x.pages = pages_of(r, want) - had + (x.again ? 1 : 0);
    return x;
  };
  const Need own = need_of(tid);  // of the first rows, often all of them
  int64_t needed = 0;
  for (int base = 0; base < r.num_seqs; base += kPlanThreads) {
    int64_t all = 0;
    (void)scan((base == 0 ? own : need_of(base + tid)).pages, lds_scan, &all);
    needed += all;
  }
  // free pages before each wave's share of them, and in all
  const int per = (int)(((int64_t)r.num_pages + kPlanThreads - 1) / kPlanThreads) * 64;  // pages of a wave
  const int64_t first = (int64_t)wave * per;
  int64_t mine = 0, free_pages = 0, before = 0;
  const bool kept = per <= 64 * 64;  // lane j keeps which of the wave's pages 64 j .. 64 j + 63 are free
  unsigned long long bits = 0;
  auto is_free = [&](int i) {  // a load without a branch, so that several are on their way at once
    const int64_t page = first + i + lane;
    const int32_t refs = r.refs[page < r.num_pages ? page : r.num_pages - 1];
    return i < per && page < r.num_pages && refs <= 0;
  };
  if (needed > 0 && r.num_pages > 0) {
    for (int i = 0; i < per; i += 64 * kPlanLoads) {
      bool there[kPlanLoads];
#pragma unroll
      for (int u = 0; u < kPlanLoads; ++u) there[u] = is_free(i + 64 * u);
#pragma unroll
      for (int u = 0; u < kPlanLoads; ++u) {
        const unsigned long long who = __ballot(there[u]);
        if (lane == i / 64 + u) bits = who;
        mine += __builtin_popcountll(who);
      }
    }
    before = scan(lane == 0 ? mine : 0, lds_scan, &free_pages);
    before = __shfl(before, 0);
  }
  int64_t upto = 0;  // needed by the rows before these
  for (int base = 0; base < r.num_seqs; base += kPlanThreads) {
    const int b = base + tid;
    const Need x = base == 0 ? own : need_of(b);
    int64_t all = 0;
    const int64_t at = upto + scan(x.pages, lds_scan, &all);
    if (b < r.num_seqs) {
      const bool ok = x.fits && (x.pages == 0 || at + x.pages <= free_pages);
      a.offsets[b] = ok ? (int32_t)(x.pages == 0 ? 0 : at) : -1;
      a.copied[b] = ok && x.again ? 1 : 0;
    }
    upto += all;
  }
  // the lowest free pages, as many as may be handed out
  const int64_t most = needed < free_pages ? needed : free_pages;
  auto hand_out = [&](int i, unsigned long long who) {
    const int64_t at =
        before + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u));
    if ((who >> lane & 1) && at < most) a.fresh[at] = (int32_t)(first + i + lane);
    before += __builtin_popcountll(who);
  };
  if (kept) {
    for (int i = 0; i < per && before < most; i += 64) hand_out(i, __shfl(bits, i / 64));
  } else {
    for (int i = 0; i < per && before < most; i += 64 * kPlanLoads) {
      bool there[kPlanLoads];
#pragma unroll
      for (int u = 0; u < kPlanLoads; ++u) there[u] = is_free(i + 64 * u);
#pragma unroll
      for (int u = 0; u < kPlanLoads; ++u) hand_out(i + 64 * u, __ballot(there[u]));
    }
  }
}

__global__ __launch_bounds__(kPlanThreads) void plan_kernel(Resize a) {
  __shared__ int64_t lds_scan[kPlanWaves];
  plan(a, lds_scan);
}

// Row b's new pages, and what is said of it, by `threads` threads, which meet in `meet` once all
// have read its lengths.
template <typename Meet>
__device__ __forceinline__ void grow(const Resize& a, int b, int tid, int threads, Meet meet) {
  const Rows& r = a.rows;
  const int64_t len = clipped(r, a.lens[b]);
  const int64_t want = a.new_lens[b] < 0 ? 0 : a.new_lens[b];
  const int at = a.offsets[b];
  const int again = a.copied[b];
  if (at >= 0 && want > len) {
    const int had = pages_of(r, len), get = pages_of(r, want);
    int32_t* const row = r.tables + (size_t)b * r.max_pages;
    for (int j = had - again + tid; j < get; j += threads) {
      const int32_t page = a.fresh[at + j - had + again];
      if (j < had) {
        const int32_t last = row[j];
        count(r, last, -1);
        reinterpret_cast<int2*>(a.copies)[b] = make_int2(last, page);
      }
      row[j] = page;
      atomicExch(r.refs + page, 1);
    }
  }
  meet();
  if (tid == 0) {
    a.granted[b] = at >= 0 ? (int32_t)want : (int32_t)len;
    if (!again) reinterpret_cast<int2*>(a.copies)[b] = make_int2(-1, -1);
  }
}

__global__ __launch_bounds__(kRowThreads) void grow_kernel(Resize a) {
  grow(a, blockIdx.x, threadIdx.x, kRowThreads, [] { __syncthreads(); });
}

// All three for few short rows, a wave per row.
__global__ __launch_bounds__(kPlanThreads) void resize_kernel(Resize a) {
  __shared__ int64_t lds_scan[kPlanWaves];
  const int lane = threadIdx.x & 63;
  const int b = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  if (b < a.rows.num_seqs) give_back(a, b, lane, 64);
  // The counts change in L2, past this CU's cache, which may hold lines with some of them, read for
  // lengths or tables beside them: once a wave's atomics are done it drops these lines.
  __builtin_amdgcn_s_waitcnt(0);
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  __syncthreads();
  plan(a, lds_scan);
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  if (b < a.rows.num_seqs) grow(a, b, lane, 64, [] { __builtin_amdgcn_wave_barrier(); });
}

// ------------------------------------------------------------ copy

constexpr int kCopyThreads = 256;
constexpr int kCopyLoads = 8;  // 16 bytes each
constexpr int kCopyChunk = kCopyThreads * kCopyLoads * 16;

__global__ __launch_bounds__(kCopyThreads) void copy_kernel(uint16_t* k, uint16_t* v, const int32_t* __restrict__ copies,
                                                            int32_t num_pages, int64_t page_bytes, int32_t parts) {
  const int part = (int)blockIdx.x % parts;
  const int pair = (int)blockIdx.x / parts;
  const int2 c = reinterpret_cast<const int2*>(copies)[pair];
  if (c.x < 0 || c.x >= num_pages || c.y < 0 || c.y >= num_pages || c.x == c.y) return;
  char* const base = reinterpret_cast<char*>(blockIdx.y == 0 ? k : v) + (int64_t)part * kCopyChunk;
  const int64_t left = page_bytes - (int64_t)part * kCopyChunk;
  const int64_t bytes = left < kCopyChunk ? left : kCopyChunk;
  const char* const src = base + (int64_t)c.x * page_bytes;
  char* const dst = base + (int64_t)c.y * page_bytes;
  const __amdgpu_buffer_rsrc_t from = make_rsrc(reinterpret_cast<const uint16_t*>(src), (uint32_t)bytes);
  const __amdgpu_buffer_rsrc_t to = make_rsrc(reinterpret_cast<const uint16_t*>(dst), (uint32_t)bytes);
  u32x4 x[kCopyLoads];
#pragma unroll
  for (int i = 0; i < kCopyLoads; ++i)
    x[i] = __builtin_bit_cast(
        u32x4, __builtin_amdgcn_raw_buffer_load_b128(from, (i * kCopyThreads + (int)threadIdx.x) * 16, 0, kLoadAux));
#pragma unroll
  for (int i = 0; i < kCopyLoads; ++i)
    __builtin_amdgcn_raw_buffer_store_b128(x[i], to, (i * kCopyThreads + (int)threadIdx.x) * 16, 0, 0);
}

// ------------------------------------------------------------ compact

constexpr int kMoveThreads = 256;
constexpr int kMoveLoads = 8;  // of 16 bytes per thread and block
constexpr int kMoveLanes = 16;                              // of a token's row of one head
constexpr int kMoveRows = kMoveThreads / kMoveLanes;        // tokens per load of the workgroup
constexpr int kMoveTokens = kMoveRows * kMoveLoads;         // of a block
static_assert(kMoveTokens <= kMoveThreads && kMoveLanes * 8 == kHeadDim, "a thread lists one token of a block");

struct Compact {
  uint16_t *k, *v;
  const int32_t *tables, *lens, *q_starts, *q_lens, *keep, *keep_lens;
  int32_t num_pages, max_pages, page_tokens, hkv, total_q;
  int32_t* new_lens;
};

// One workgroup per (sequence, cache, head).  What it takes is what the longest sequence's workgroups
// take, at 30 GB/s each: 12 contexts of 8,192..16,384 tokens 208 us, 3.8 TB/s, the copy rate as
// long as all are at work.  (Several could share a sequence's head, if each wrote its block once the
// blocks before it had been read; that needs counters, which the call has no workspace for.)  (Half a head per workgroup, in parts of 128 bytes: 227; a quarter: 268;
// twice the loads in flight: 209, but 0.8 us more for the accepted paths of 64 requests.)
__global__ __launch_bounds__(kMoveThreads) void compact_kernel(Compact a) {
  __shared__ int32_t lds_from[3][kMoveTokens], lds_to[3][kMoveTokens];  // cache rows, -1: nothing to move
  const int tid = threadIdx.x;
  const int slices = 2 * a.hkv;
  const int b = (int)blockIdx.x / slices;
  const int slice = (int)blockIdx.x - b * slices;
  const int len = a.lens[b] < 0 ? 0 : a.lens[b];
  const int n = a.q_lens[b] < 0 ? 0 : a.q_lens[b] < len ? a.q_lens[b] : len;
  const int kept = a.keep_lens[b] < 0 ? 0 : a.keep_lens[b] < n ? a.keep_lens[b] : n;
  const int hist = len - n;
  if (slice == 0 && tid == 0 && a.new_lens != nullptr) a.new_lens[b] = hist + kept;
  const int64_t row0 = a.q_starts[b];
  const int32_t* const table = a.tables + (size_t)b * a.max_pages;
  uint16_t* const base = (slice < a.hkv ? a.k : a.v) + (size_t)(slice < a.hkv ? slice : slice - a.hkv) * kHeadDim;
  // A list of where the tokens of a block come from and go to is made in three steps, each of which
  // uses what the one before has loaded a block earlier, so that nothing waits for a chain of loads.
  struct Place {
    int page, slot;
  };
  auto which = [&](int i0) {  // the kept token that this thread lists, -1: none
    const int64_t row = row0 + i0 + tid;
    const bool there = tid < kMoveTokens && i0 + tid < kept && row >= 0 && row < a.total_q;
    return there ? a.keep[row] : -1;
  };
  auto place = [&](int t, bool there) {
    const int j = there ? t / a.page_tokens : 0;
    const bool named = there && j < a.max_pages;
    return Place{named ? table[j] : -1, t - j * a.page_tokens};
  };
  auto row_of = [&](const Place& p) {
    return p.page >= 0 && p.page < a.num_pages ? p.page * a.page_tokens + p.slot : -1;
  };
  Place from, to;
  auto find = [&](int i0, int t) {
    const int i = i0 + tid;
    const bool moves = t >= 0 && t < n && t != i;
    from = place(hist + t, moves);
    to = place(hist + i, moves);
  };
  auto list = [&](int buf) {
    if (tid < kMoveTokens) {
      const int to_row = row_of(to);
      lds_from[buf][tid] = to_row < 0 ? -1 : row_of(from);
      lds_to[buf][tid] = to_row;
    }
  };
  const int group = tid / kMoveLanes;
  const int at = (tid % kMoveLanes) * 8;
  const size_t row_elems = (size_t)a.hkv * kHeadDim;
  // Blocks in order: the next one's tokens are read before this one's are written, which no
  // token behind it needs any more.
  u32x4 x[kMoveLoads], next[kMoveLoads];
  auto read = [&](int buf, u32x4 (&to)[kMoveLoads]) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kMoveLoads; ++u) {
      const int row = lds_from[buf][u * kMoveRows + group];
      to[u] = u32x4{0u, 0u, 0u, 0u};
      if (row >= 0) to[u] = load16(base + row * row_elems + at);
    }
  };
  int kept_token = which(0);
  find(0, kept_token);
  kept_token = which(kMoveTokens);
  list(0);
  find(kMoveTokens, kept_token);
  kept_token = which(2 * kMoveTokens);
  __syncthreads();
  read(0, next);
  list(1);
  find(2 * kMoveTokens, kept_token);
  kept_token = which(3 * kMoveTokens);
  for (int i0 = 0, buf = 0; i0 < kept; i0 += kMoveTokens, buf = buf == 2 ? 0 : buf + 1) {
    // every thread's loads of this block have arrived before any store
#pragma unroll
    for (int u = 0; u < kMoveLoads; ++u) {
      x[u] = next[u];
      asm volatile("" : "+v"(x[u]));
    }
    __syncthreads();  // and the next block's list is there
    list(buf == 0 ? 2 : buf - 1);
    find(i0 + 3 * kMoveTokens, kept_token);
    kept_token = which(i0 + 4 * kMoveTokens);
    read(buf == 2 ? 0 : buf + 1, next);
#pragma unroll
    for (int u = 0; u < kMoveLoads; ++u) {
      const int i = u * kMoveRows + group;
      if (lds_from[buf][i] >= 0) __builtin_nontemporal_store(x[u], reinterpret_cast<u32x4*>(base + lds_to[buf][i] * row_elems + at));
    }
  }
}

int check_rows(ctx_decode_attn* h, int32_t num_seqs, int32_t max_pages, int32_t num_pages) {
  int rc = check_common(h, num_seqs, 1.0f);
  if (rc != CTX_OK) return rc;
  if (h->desc.page_tokens <= 0) return fail(CTX_ERR_UNSUPPORTED, "the handle was created without page_tokens");
  if (num_pages < 0 || max_pages <= 0)
    return fail(CTX_ERR_INVALID_ARG, "num_pages must not be negative and max_pages_per_seq must be positive");
  if ((int64_t)num_pages * h->desc.page_tokens > kMostTokens)
    return fail(CTX_ERR_UNSUPPORTED, "caches of more than %d tokens", kMostTokens);
  if (!fits_launch(num_seqs, kRowThreads)) return fail(CTX_ERR_INVALID_ARG, "grid of rows too large");
  return CTX_OK;
}

Rows rows_of(const ctx_decode_attn* h, int32_t* tables, int32_t max_pages, int32_t num_seqs, int32_t* refs,
             int32_t num_pages) {
  return Rows{tables, max_pages, h->desc.page_tokens, num_seqs, refs, num_pages};
}

// Whether two arrays of 32-bit values share any.
bool overlap(const void* a, int64_t a_values, const void* b, int64_t b_values) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
  return a_values > 0 && b_values > 0 && p < q + (uintptr_t)b_values * 4 && q < p + (uintptr_t)a_values * 4;
}

struct Array {
  const void* data;
  int64_t values;
};

// Whether one of the arrays that a call writes, the first `written` ones, shares values with another of them all.
template <int kArrays>
bool any_overlap(const Array (&x)[kArrays], int written) {
  for (int i = 0; i < written; ++i)
    for (int j = i + 1; j < kArrays; ++j)
      if (overlap(x[i].data, x[i].values, x[j].data, x[j].values)) return true;
  return false;
}

int launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CTX_OK : hip_fail(e, "kernel launch");
}

}  // namespace

extern "C" int ctx_kv_fork_run_paged(ctx_decode_attn* h, int32_t* block_tables, int32_t max_pages_per_seq,
                                     int32_t* seq_lens, int32_t num_seqs, const int32_t* parents, int32_t* page_refs,
                                     int32_t num_pages, void* stream) {
  int rc = check_rows(h, num_seqs, max_pages_per_seq, num_pages);
  if (rc != CTX_OK) return rc;
  if (num_seqs == 0) return CTX_OK;
  if (block_tables == nullptr || seq_lens == nullptr || parents == nullptr ||
      (page_refs == nullptr && num_pages > 0))
    return fail(CTX_ERR_INVALID_ARG, "NULL data pointer");
  const int64_t seqs = num_seqs;
  if (any_overlap({{block_tables, seqs * max_pages_per_seq}, {seq_lens, seqs}, {page_refs, num_pages}, {parents, seqs}}, 3))
    return fail(CTX_ERR_INVALID_ARG, "block_tables, seq_lens, page_refs and parents may not overlap");
  if ((rc = check_device(h)) != CTX_OK) return rc;
  hipLaunchKernelGGL(fork_kernel, dim3((unsigned)num_seqs), dim3(kRowThreads), 0, reinterpret_cast<hipStream_t>(stream),
                     rows_of(h, block_tables, max_pages_per_seq, num_seqs, page_refs, num_pages), seq_lens, parents);
  return launched();
}

extern "C" size_t ctx_kv_resize_workspace(int32_t num_seqs, int32_t num_pages) {
  const size_t seqs = num_seqs > 0 ? (size_t)num_seqs : 0, pages = num_pages > 0 ? (size_t)num_pages : 0;
  return (2 * seqs + pages) * sizeof(int32_t);
}

extern "C" int ctx_kv_resize_run_paged(ctx_decode_attn* h, int32_t* block_tables, int32_t max_pages_per_seq,
                                       const int32_t* seq_lens, const int32_t* new_lens, int32_t num_seqs,
                                       int32_t* page_refs, int32_t num_pages, int32_t* granted, int32_t* copies,
                                       void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_rows(h, num_seqs, max_pages_per_seq, num_pages);
  if (rc != CTX_OK) return rc;
  if (num_seqs == 0) return CTX_OK;
  if (block_tables == nullptr || seq_lens == nullptr || new_lens == nullptr || (page_refs == nullptr && num_pages > 0) ||
      granted == nullptr || copies == nullptr || workspace == nullptr)
    return fail(CTX_ERR_INVALID_ARG, "NULL data pointer");
  if (!aligned16(workspace) || (reinterpret_cast<uintptr_t>(copies) & 7u) != 0)
    return fail(CTX_ERR_ALIGNMENT, "workspace must be 16-byte and copies 8-byte aligned");
  const size_t need = ctx_kv_resize_workspace(num_seqs, num_pages);
  if (workspace_bytes < need) return fail(CTX_ERR_CAPACITY, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
  const int64_t seqs = num_seqs;
  // granted may be one of the lengths themselves
  const bool over_lens = granted == seq_lens, over_new = granted == new_lens;
  if (any_overlap({{block_tables, seqs * max_pages_per_seq}, {page_refs, num_pages}, {copies, 2 * seqs},
                   {workspace, (int64_t)(need / sizeof(int32_t))}, {granted, seqs}, {seq_lens, over_lens ? 0 : seqs},
                   {new_lens, over_new ? 0 : seqs}}, 5) ||
      (over_lens && !over_new && overlap(seq_lens, seqs, new_lens, seqs)))
    return fail(CTX_ERR_INVALID_ARG,
                "block_tables, page_refs, granted, copies and workspace may not overlap each other or an input, but for "
                "granted seq_lens or new_lens themselves");
  if ((rc = check_device(h)) != CTX_OK) return rc;
  Resize a{};
  a.rows = rows_of(h, block_tables, max_pages_per_seq, num_seqs, page_refs, num_pages);
  a.lens = seq_lens;
  a.new_lens = new_lens;
  a.granted = granted;
  a.copies = copies;
  a.offsets = static_cast<int32_t*>(workspace);
  a.copied = a.offsets + num_seqs;
  a.fresh = a.copied + num_seqs;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  // One launch for few short rows, a wave each.  Growth by 40 tokens and the trim of it, with one and with three
  // launches (us, in a graph): 8 rows of 64 entries 16.1 / 17.8, 16 17.2 / 18.3, 24 24.6 / 23.9, 64 28.7 / 19.0; of
  // 131,072 pages 31.5 / 33.6.  Whole rows emptied and filled: 16 of 128 entries 18.0 / 18.2, of 256 20.3 / 19.1, of
  // 512 24.8 / 21.6, one of 8,192 89 / 38.
  if (num_seqs <= kSmallRows && max_pages_per_seq <= kSmallWidth) {
    hipLaunchKernelGGL(resize_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
    return launched();
  }
  hipLaunchKernelGGL(give_back_kernel, dim3((unsigned)num_seqs), dim3(kRowThreads), 0, s, a);
  hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
  hipLaunchKernelGGL(grow_kernel, dim3((unsigned)num_seqs), dim3(kRowThreads), 0, s, a);
  return launched();
}

extern "C" int ctx_kv_copy_run_paged(ctx_decode_attn* h, void* k_pages, void* v_pages, int32_t num_pages,
                                     const int32_t* copies, int32_t num_copies, void* stream) {
  int rc = check_rows(h, 0, 1, num_pages);
  if (rc != CTX_OK) return rc;
  if (num_copies < 0) return fail(CTX_ERR_INVALID_ARG, "num_copies %d < 0", num_copies);
  if (num_copies == 0 || num_pages == 0) return CTX_OK;
  if (k_pages == nullptr || v_pages == nullptr || copies == nullptr) return fail(CTX_ERR_INVALID_ARG, "NULL data pointer");
  if (!aligned16(k_pages) || !aligned16(v_pages) || (reinterpret_cast<uintptr_t>(copies) & 7u) != 0)
    return fail(CTX_ERR_ALIGNMENT, "k_pages and v_pages must be 16-byte and copies 8-byte aligned");
  const int64_t page_bytes = (int64_t)h->desc.page_tokens * h->desc.num_kv_heads * kHeadDim * 2;
  const int64_t parts = (page_bytes + kCopyChunk - 1) / kCopyChunk;
  if (!fits_launch(parts * num_copies, kCopyThreads)) return fail(CTX_ERR_INVALID_ARG, "copy grid too large");
  if ((rc = check_device(h)) != CTX_OK) return rc;
  hipLaunchKernelGGL(copy_kernel, dim3((unsigned)(parts * num_copies), 2), dim3(kCopyThreads), 0,
                     reinterpret_cast<hipStream_t>(stream), static_cast<uint16_t*>(k_pages),
                     static_cast<uint16_t*>(v_pages), copies, num_pages, page_bytes, (int32_t)parts);
  return launched();
}

extern "C" int ctx_kv_compact_run_paged(ctx_decode_attn* h, void* k_pages, void* v_pages, int32_t num_pages,
                                        const int32_t* block_tables, int32_t max_pages_per_seq,
                                        const int32_t* seq_lens, const int32_t* q_starts, const int32_t* q_lens,
                                        const int32_t* keep, const int32_t* keep_lens, int32_t num_seqs,
                                        int32_t total_q, int32_t* new_lens, void* stream) {
  int rc = check_rows(h, num_seqs, max_pages_per_seq, num_pages);
  if (rc != CTX_OK) return rc;
  if (total_q < 0) return fail(CTX_ERR_INVALID_ARG, "total_q %d < 0", total_q);
  if (num_seqs == 0) return CTX_OK;
  if (k_pages == nullptr || v_pages == nullptr || block_tables == nullptr || seq_lens == nullptr || q_starts == nullptr ||
      q_lens == nullptr || keep_lens == nullptr || (keep == nullptr && total_q > 0))
    return fail(CTX_ERR_INVALID_ARG, "NULL data pointer");
  if (!aligned16(k_pages) || !aligned16(v_pages))
    return fail(CTX_ERR_ALIGNMENT, "k_pages and v_pages must be 16-byte aligned");
  const int64_t grid = (int64_t)num_seqs * 2 * h->desc.num_kv_heads;
  if (!fits_launch(grid, kMoveThreads)) return fail(CTX_ERR_INVALID_ARG, "compaction grid too large");
  const int64_t seqs = num_seqs;
  if (new_lens != nullptr && any_overlap({{new_lens, seqs}, {seq_lens, seqs}, {q_starts, seqs}, {q_lens, seqs},
                                          {keep_lens, seqs}, {keep, total_q}, {block_tables, seqs * max_pages_per_seq}}, 1))
    return fail(CTX_ERR_INVALID_ARG, "new_lens may not overlap an input");
  const int64_t cache = (int64_t)num_pages * h->desc.page_tokens * h->desc.num_kv_heads * kHeadDim / 2;
  if (overlap(k_pages, cache, v_pages, cache)) return fail(CTX_ERR_INVALID_ARG, "k_pages and v_pages may not overlap");
  if ((rc = check_device(h)) != CTX_OK) return rc;
  Compact a{};
  a.k = static_cast<uint16_t*>(k_pages);
  a.v = static_cast<uint16_t*>(v_pages);
  a.tables = block_tables;
  a.lens = seq_lens;
  a.q_starts = q_starts;
  a.q_lens = q_lens;
  a.keep = keep;
  a.keep_lens = keep_lens;
  a.num_pages = num_pages;
  a.max_pages = max_pages_per_seq;
  a.page_tokens = h->desc.page_tokens;
  a.hkv = h->desc.num_kv_heads;
  a.total_q = total_q;
  a.new_lens = new_lens;
  hipLaunchKernelGGL(compact_kernel, dim3((unsigned)grid), dim3(kMoveThreads), 0, reinterpret_cast<hipStream_t>(stream), a);
  return launched();
}
