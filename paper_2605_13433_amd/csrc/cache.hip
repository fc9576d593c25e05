// Pages of the key-value cache: room for new tokens (with copy on write), their rows,
// forks, ends of sequences, and moving the used pages together.
//
// The bookkeeping is whole numbers, small and a chain of steps: extend and compact
// plan in one work-group (the free pages are found in order, 16384 counts a round, by
// wave ballots and one scan of 256 sums), fork and free take a work-group a row.  The
// rest is copies, bound by HBM: 16 bytes a lane, several loads of a thread in flight.
#include <algorithm>

#include "cache.h"
#include "device.h"

namespace hstu {

namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_WAVES = PLAN_THREADS / 64;
constexpr int ROUND = 16;                    // counts a thread looks at in one round
constexpr int ROW_THREADS = 256;

// ------------------------------------------------------------- block helpers
// Sum of x over the lower threads of the work-group; `total` receives the sum of all.
// Ends with a barrier, so that `sums` can be used again.
__device__ __forceinline__ int32_t block_prefix(int32_t x, int32_t *sums, int tid, int32_t &total) {
  const int32_t incl = wave_prefix(x);
  if ((tid & 63) == 63) sums[tid >> 6] = incl;
  __syncthreads();
  int32_t before = 0, all = 0;
  for (int w = 0; w < PLAN_WAVES; ++w) {
    const int32_t s = sums[w];
    before += w < (tid >> 6) ? s : 0;
    all += s;
  }
  __syncthreads();
  total = all;
  return before + incl - x;
}

struct CollectSmem {
  int32_t at[ROUND * PLAN_WAVES + 1];
};

// The counts of pages p0 + k PLAN_THREADS + tid (past the pool none is read).
__device__ __forceinline__ void load_counts(const int32_t *refs, int64_t p0, int32_t pages,
                                            int tid, int32_t (&c)[ROUND]) {
#pragma unroll
  for (int k = 0; k < ROUND; ++k) {
    const int64_t p = p0 + k * PLAN_THREADS + tid;
    c[k] = p < pages ? refs[p] : 0;
  }
}

// Writes the pages p that `want(p, count)` names to out[0 ..], in order, until `most` of
// them are found; returns their number.  `c` holds the first round's counts.  All
// threads.
template <typename Want>
__device__ __forceinline__ int32_t collect(const int32_t *refs, int32_t pages, int32_t *out,
                                           int32_t most, CollectSmem &sm, int tid,
                                           int32_t (&c)[ROUND], Want want) {
  const int lane = tid & 63, wv = tid >> 6;
  int32_t got = 0;
  for (int64_t p0 = 0; p0 < pages && got < most; p0 += ROUND * PLAN_THREADS) {
    if (p0 > 0) load_counts(refs, p0, pages, tid, c);
    uint64_t hit[ROUND];
#pragma unroll
    for (int k = 0; k < ROUND; ++k) {
      const int64_t p = p0 + k * PLAN_THREADS + tid;
      hit[k] = __ballot(p < pages && want((int32_t)p, c[k]));
      if (lane == 0) sm.at[k * PLAN_WAVES + wv] = __popcll(hit[k]);
    }
    __syncthreads();
    if (wv == 0) {                      // ROUND * PLAN_WAVES = 256 sums, four a lane
      constexpr int PER = ROUND * PLAN_WAVES / 64;
      int32_t v[PER], sum = 0;
#pragma unroll
      for (int x = 0; x < PER; ++x) {
        v[x] = sum;
        sum += sm.at[lane * PER + x];
      }
      const int32_t incl = wave_prefix(sum);
#pragma unroll
      for (int x = 0; x < PER; ++x) sm.at[lane * PER + x] = incl - sum + v[x];
      if (lane == 63) sm.at[ROUND * PLAN_WAVES] = incl;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ROUND; ++k) {
      const int32_t at = got + sm.at[k * PLAN_WAVES + wv] +
                         __popcll(hit[k] & ((1ull << lane) - 1));
      if (((hit[k] >> lane) & 1) && at < most)
        out[at] = (int32_t)(p0 + k * PLAN_THREADS + tid);
    }
    got += sm.at[ROUND * PLAN_WAVES];
    __syncthreads();
  }
  return got < most ? got : most;
}

// Keeps the loads above it from being sunk to their use (emits nothing).
__device__ __forceinline__ void issue_fence() { asm volatile("" ::: "memory"); }

// Copies `bytes` (a multiple of 16) from src to dst, threads tid of nt.
__device__ __forceinline__ void copy16(const char *src, char *dst, int64_t bytes, int tid, int nt) {
  const int64_t n = bytes >> 4;
  int64_t x = tid;
  for (; x + 3 * nt < n; x += 4 * nt) {
    const uint4 a = ((const uint4 *)src)[x], b = ((const uint4 *)src)[x + nt],
                c = ((const uint4 *)src)[x + 2 * nt], d = ((const uint4 *)src)[x + 3 * nt];
    issue_fence();
    ((uint4 *)dst)[x] = a;
    ((uint4 *)dst)[x + nt] = b;
    ((uint4 *)dst)[x + 2 * nt] = c;
    ((uint4 *)dst)[x + 3 * nt] = d;
  }
  for (; x < n; x += nt) ((uint4 *)dst)[x] = ((const uint4 *)src)[x];
}

// --------------------------------------------------------------------- clear
__global__ void cache_clear_kernel(CacheDev c) {
  const int64_t entries = (int64_t)c.slots * c.max_pages;
  const int64_t step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t x = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; x < entries; x += step)
    c.tables[x] = -1;
  for (int64_t x = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; x < c.num_pages; x += step)
    c.refs[x] = 0;
  for (int64_t x = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; x < c.slots; x += step)
    c.lens[x] = 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) *c.status = 0;
}

// -------------------------------------------------------------------- extend
// A row's plan: pages it needs, the first of them in the list of free pages, the shared
// page that is copied (-1: none); `need` < 0: refused.
struct RowPlan {
  int32_t need, base, shared, len;
};
// A copy that the second launch makes: `rows` tokens of page src into page dst.
struct PageCopy {
  int32_t src, dst, rows;
};

// LDS room of the plan: owners of the slots, free pages (both in the workspace where
// there are more), and rows that need more pages than a thread writes by itself.
constexpr int OWNERS_LDS = 8192, FRESH_LDS = 4096, PAGES_ALONE = 4;

// One row: what it needs.  `owner` holds the first row that names each slot.
__device__ __forceinline__ RowPlan plan_row(const CacheDev &c, int32_t r, int32_t s, int32_t cnt,
                                            const int32_t *owner, int &bad) {
  RowPlan p{-1, 0, -1, 0};
  if (s < 0 || s >= c.slots) {
    bad |= HSTU_CACHE_BAD_SLOT;
    return p;
  }
  if (__hip_atomic_load(&owner[s], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != r) {
    bad |= HSTU_CACHE_TWICE;
    return p;
  }
  if (cnt < 0) {
    bad |= HSTU_CACHE_BAD_COUNT;
    return p;
  }
  p.len = slot_len(c.lens, c.slots, c.capacity, s);
  if (cnt > c.capacity - p.len) {
    bad |= HSTU_CACHE_FULL;
    return p;
  }
  const int32_t had = pages_of(p.len, c.log_page);
  p.need = pages_of((int64_t)p.len + cnt, c.log_page) - had;
  if (cnt > 0 && (p.len & ((1 << c.log_page) - 1)) != 0) {
    const int32_t last = c.tables[(int64_t)s * c.max_pages + had - 1];
    if (last >= 0 && last < c.num_pages && c.refs[last] > 1) {
      p.shared = last;
      ++p.need;
    }
  }
  return p;
}

// The chain of steps bounds it: the counts of the first 16384 pages are loaded before
// anything else, owners and free pages lie in LDS, a thread keeps its row in registers
// and writes up to PAGES_ALONE pages of it, the rest a wave a row.  (With all of this in
// device memory and a wave a row: 32 rows of one token 15.7 us, 64 prompts 16.5.)
__global__ void __launch_bounds__(PLAN_THREADS)
cache_extend_kernel(CacheDev c, const int32_t *slot_ids, const int32_t *counts, int32_t n,
                    int32_t *start, int32_t *owner_ws, RowPlan *plan, int32_t *fresh_ws,
                    PageCopy *copies) {
  __shared__ int32_t sums[PLAN_WAVES];
  __shared__ CollectSmem cs;
  __shared__ int32_t owner_lds[OWNERS_LDS], fresh_lds[FRESH_LDS];
  __shared__ int32_t wide[PLAN_THREADS], n_wide;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  int32_t refs0[ROUND];
  load_counts(c.refs, 0, c.num_pages, tid, refs0);
  const int32_t s0 = tid < n ? slot_ids[tid] : -1, cnt0 = tid < n ? counts[tid] : 0;
  int32_t *owner = c.slots <= OWNERS_LDS ? owner_lds : owner_ws;
  if (tid == 0) n_wide = 0;
  for (int r = tid; r < n; r += PLAN_THREADS) {
    const int32_t s = r < PLAN_THREADS ? s0 : slot_ids[r];
    if (s >= 0 && s < c.slots) atomicExch(&owner[s], n);
  }
  if (owner == owner_ws) __threadfence();
  __syncthreads();
  for (int r = tid; r < n; r += PLAN_THREADS) {
    const int32_t s = r < PLAN_THREADS ? s0 : slot_ids[r];
    if (s >= 0 && s < c.slots) atomicMin(&owner[s], r);
  }
  if (owner == owner_ws) __threadfence();
  __syncthreads();

  int64_t run = 0;
  int bad = 0;
  RowPlan mine{-1, 0, -1, 0};                 // this thread's first row
  for (int r0 = 0; r0 < n; r0 += PLAN_THREADS) {
    const int r = r0 + tid;
    RowPlan p{-1, 0, -1, 0};
    if (r < n)
      p = plan_row(c, r, r0 == 0 ? s0 : slot_ids[r], r0 == 0 ? cnt0 : counts[r], owner, bad);
    // two scans, so that 1024 rows of up to 2^31 pages each do not overflow
    int32_t all_hi = 0, all_lo = 0;
    const int32_t want = p.need > 0 ? p.need : 0;
    int64_t hi = 0;
    if (__syncthreads_or(want >> 15)) hi = block_prefix(want >> 15, sums, tid, all_hi);
    const int64_t lo = block_prefix(want & 32767, sums, tid, all_lo);
    const int64_t base = run + (hi << 15) + lo;
    p.base = (int32_t)(base < INT32_MAX ? base : INT32_MAX);   // (past every pool)
    if (r0 == 0) mine = p;
    else if (r < n) plan[r] = p;
    run += ((int64_t)all_hi << 15) + all_lo;
  }
  const int32_t total = (int32_t)(run < c.num_pages ? run : c.num_pages);
  int32_t *fresh = total <= FRESH_LDS ? fresh_lds : fresh_ws;
  const int32_t got = collect(c.refs, c.num_pages, fresh, total, cs, tid, refs0,
                              [](int32_t, int32_t count) { return count == 0; });
  __syncthreads();

  for (int r0 = 0; r0 < n; r0 += PLAN_THREADS) {
    const int r = r0 + tid;
    const RowPlan p = r0 == 0 ? mine : r < n ? plan[r] : RowPlan{-1, 0, -1, 0};
    if (r < n) {
      const int32_t s = r0 == 0 ? s0 : slot_ids[r];
      const bool ok = p.need == 0 || (p.need > 0 && (int64_t)p.base + p.need <= got);
      if (p.need > 0 && !ok) bad |= HSTU_CACHE_FULL;
      PageCopy pc{-1, -1, 0};
      if (ok) {
        const int32_t first = pages_of(p.len, c.log_page) - (p.shared >= 0 ? 1 : 0);
        int32_t *row = c.tables + (int64_t)s * c.max_pages + first;
        for (int x = 0; x < p.need && x < PAGES_ALONE; ++x) {
          const int32_t page = fresh[p.base + x];
          row[x] = page;
          c.refs[page] = 1;
        }
        if (p.need > PAGES_ALONE) wide[atomicAdd(&n_wide, 1)] = r;
        if (p.shared >= 0) {
          pc = PageCopy{p.shared, fresh[p.base], p.len & ((1 << c.log_page) - 1)};
          atomicSub(&c.refs[p.shared], 1);
        }
        c.lens[s] = p.len + (r0 == 0 ? cnt0 : counts[r]);
        if (r0 == 0) plan[r] = p;             // for the waves below
      }
      copies[r] = pc;
      start[r] = ok ? p.len : -1;
    }
    __syncthreads();
    const int many = n_wide;
    for (int x = wv; x < many; x += PLAN_WAVES) {
      const RowPlan q = plan[wide[x]];
      const int32_t s = slot_ids[wide[x]];
      int32_t *row = c.tables + (int64_t)s * c.max_pages + pages_of(q.len, c.log_page) -
                     (q.shared >= 0 ? 1 : 0);
      for (int y = PAGES_ALONE + lane; y < q.need; y += 64) {
        const int32_t page = fresh[q.base + y];
        row[y] = page;
        c.refs[page] = 1;
      }
    }
    __syncthreads();
    if (tid == 0) n_wide = 0;
    __syncthreads();
  }
  if (bad) atomicOr(c.status, bad);
}

// One work-group a (row, layer and k or v): the shared last pages' tokens.
__global__ void __launch_bounds__(ROW_THREADS)
cache_copy_kernel(CacheDev c, const PageCopy *copies) {
  const PageCopy pc = copies[blockIdx.x];
  if (pc.src < 0) return;
  const int layer = blockIdx.y >> 1;
  char *pool = ((blockIdx.y & 1) ? c.v : c.k) + layer * c.layer_bytes;
  const int64_t page = (int64_t)c.row_bytes << c.log_page;
  copy16(pool + pc.src * page, pool + pc.dst * page, (int64_t)pc.rows * c.row_bytes, threadIdx.x,
         ROW_THREADS);
  if (c.ts && blockIdx.y == 0)
    for (int x = threadIdx.x; x < pc.rows; x += ROW_THREADS)
      c.ts[((int64_t)pc.dst << c.log_page) + x] = c.ts[((int64_t)pc.src << c.log_page) + x];
}

// --------------------------------------------------------------------- write
constexpr int WRITE_TOKENS = 16;             // of a work-group

// Work-group b of a write: row r's work-groups are write_base(off[r], r) .. -- apart for
// every batch of rows, whatever their lengths, since floor(a / 16) + ceil(L / 16) <=
// floor((a + L) / 16) + 1.
__device__ __forceinline__ int64_t write_base(int64_t off, int64_t r) {
  return (off < 0 ? 0 : off) / WRITE_TOKENS + r;
}

// The last of n rows whose base is at most b (-1: none), by every wave for itself: 64
// rows are looked at in a round, so 4096 rows take two.
__device__ __forceinline__ int32_t write_row(const int64_t *off, int32_t n, int64_t b, int lane) {
  int32_t lo = -1, len = n;                    // the answer is lo or one of the len rows behind
  while (len > 0) {
    const int32_t step = (len + 63) / 64;
    const int64_t r = (int64_t)lo + 1 + (int64_t)lane * step;
    const bool before = r <= (int64_t)lo + len && write_base(off[r <= (int64_t)lo + len ? r : lo + 1],
                                                             r) <= b;
    const int hits = __popcll(__ballot(before));
    if (hits == 0) break;
    const int32_t at = lo + 1 + (hits - 1) * step;
    const int32_t left = lo + len - at;        // rows behind `at`
    lo = at;
    len = left < step - 1 ? left : step - 1;
  }
  return lo;
}

// A work-group writes up to WRITE_TOKENS of a row's tokens, a wave every fourth: the
// pages of its tokens are looked up, and lane x moves 16-byte unit x of the k and v rows
// of all of them.  Every load runs, on a clamped index where its token is none, so that
// the table's and the rows' latencies overlap and nothing waits in a branch; the stores
// alone ask.  64 prompts of 16..4096 tokens, 166 MB read and written: 61 us with the
// loads in branches and as many work-groups for every row, 43 without the branches, 33
// (5.0 TB/s, a copy's rate) with the work-groups dealt by length.
__global__ void __launch_bounds__(ROW_THREADS)
cache_write_kernel(CacheDev c, int32_t layer, const char *__restrict__ k,
                   const char *__restrict__ v, const int64_t *__restrict__ ts,
                   const int32_t *__restrict__ slot_ids, const int32_t *__restrict__ start,
                   const int64_t *__restrict__ off, int32_t n, int64_t total, int32_t max_new) {
  constexpr int W = ROW_THREADS / 64, U = WRITE_TOKENS / W;    // tokens of a wave
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t r = __builtin_amdgcn_readfirstlane(write_row(off, n, blockIdx.x, lane));
  if (r < 0) return;
  const int32_t s = slot_ids[r], at0 = start[r];
  int64_t first = off[r], end = off[r + 1];
  const int64_t t0 = ((int64_t)blockIdx.x - write_base(first, r)) * WRITE_TOKENS;
  first = first < 0 ? 0 : (first > total ? total : first);
  end = end < first ? first : (end > total ? total : end);
  end = end - first > max_new ? first + max_new : end;
  if ((s < 0) | (s >= c.slots) | (at0 < 0) | (t0 >= end - first)) return;
  const int32_t *table = c.tables + (int64_t)s * c.max_pages;
  const int32_t units = c.row_bytes >> 4;                      // of a row, k and v each
  const int64_t pool = layer * c.layer_bytes;
  // pool rows and source rows of the wave's tokens w, w + W, ..; row -1: no such token,
  // or no place for it
  int32_t row[U];
  int64_t src[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int64_t t = t0 + w + W * i, pos = at0 + t;
    src[i] = t < end - first ? first + t : end - 1;
    row[i] = table[(pos < c.capacity ? pos : c.capacity - 1) >> c.log_page];
  }
  issue_fence();
  bool looked_up = false;
  for (int32_t x = lane; x < 2 * units; x += 64) {
    const bool is_v = x >= units;
    const int64_t col = 16 * (int64_t)(is_v ? x - units : x);
    const char *from = (is_v ? v : k) + col;
    char *to = (is_v ? c.v : c.k) + pool + col;
    uint4 val[U];
#pragma unroll
    for (int i = 0; i < U; ++i) val[i] = *(const uint4 *)(from + src[i] * c.row_bytes);
    issue_fence();
    if (!looked_up) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int64_t t = t0 + w + W * i, pos = at0 + t;
        const bool there = (t < end - first) & (pos < c.capacity);
        row[i] = there ? page_row(row[i], c.num_pages, c.log_page, (int32_t)pos) : -1;
      }
      looked_up = true;
    }
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (row[i] >= 0) *(uint4 *)(to + (int64_t)row[i] * c.row_bytes) = val[i];
  }
  if (ts && lane < U) {
    int32_t mine = -1;
    int64_t from = 0;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      mine = lane == i ? row[i] : mine;
      from = lane == i ? src[i] : from;
    }
    if (mine >= 0) c.ts[mine] = ts[from];
  }
}

// ------------------------------------------------------------- fork and free
// Whether an earlier row names the target of row r too.  All threads of the block.
__device__ __forceinline__ bool named_before(const int32_t *dst, int r) {
  const int32_t mine = dst[r];
  int twice = 0;
  for (int x = threadIdx.x; x < r; x += ROW_THREADS) twice |= dst[x] == mine ? 1 : 0;
  return __syncthreads_or(twice) != 0;
}

// First launch: what every source holds is noted and counted before any target
// changes.  len_of[r] = -1: the row is skipped.
__global__ void __launch_bounds__(ROW_THREADS)
cache_fork_note_kernel(CacheDev c, const int32_t *src, const int32_t *dst, int32_t *len_of,
                       int32_t *noted) {
  const int r = blockIdx.x, tid = threadIdx.x;
  const int32_t s = src[r], d = dst[r];
  const bool twice = named_before(dst, r);
  const bool none = s < 0 || s >= c.slots || d < 0 || d >= c.slots;
  if (none || twice) {
    if (tid == 0) {
      len_of[r] = -1;
      atomicOr(c.status, none ? HSTU_CACHE_BAD_SLOT : HSTU_CACHE_TWICE);
    }
    return;
  }
  const int32_t len = slot_len(c.lens, c.slots, c.capacity, s);
  const int32_t pages = pages_of(len, c.log_page);
  if (tid == 0) len_of[r] = len;
  for (int x = tid; x < pages; x += ROW_THREADS) {
    const int32_t p = c.tables[(int64_t)s * c.max_pages + x];
    noted[(int64_t)r * c.max_pages + x] = p;
    if (p >= 0 && p < c.num_pages) atomicAdd(&c.refs[p], 1);
  }
}

// Second launch: the targets' old pages are given back, their tables replaced.
__global__ void __launch_bounds__(ROW_THREADS)
cache_fork_set_kernel(CacheDev c, const int32_t *dst, const int32_t *len_of,
                      const int32_t *noted) {
  const int r = blockIdx.x, tid = threadIdx.x;
  const int32_t len = len_of[r];
  if (len < 0) return;
  const int32_t d = dst[r];
  const int32_t had = pages_of(slot_len(c.lens, c.slots, c.capacity, d), c.log_page);
  const int32_t has = pages_of(len, c.log_page);
  int32_t *row = c.tables + (int64_t)d * c.max_pages;
  for (int x = tid; x < (had > has ? had : has); x += ROW_THREADS) {
    if (x < had) {
      const int32_t p = row[x];
      if (p >= 0 && p < c.num_pages) atomicSub(&c.refs[p], 1);
    }
    row[x] = x < has ? noted[(int64_t)r * c.max_pages + x] : -1;
  }
  __syncthreads();                       // (every thread has read the old length)
  if (tid == 0) c.lens[d] = len;
}

__global__ void __launch_bounds__(ROW_THREADS)
cache_free_kernel(CacheDev c, const int32_t *slot_ids) {
  __shared__ int32_t held;
  const int tid = threadIdx.x;
  const int32_t s = slot_ids[blockIdx.x];
  if (s < 0 || s >= c.slots) {
    if (tid == 0) atomicOr(c.status, HSTU_CACHE_BAD_SLOT);
    return;
  }
  // whoever takes the length frees the pages: a slot named twice is freed once
  if (tid == 0) held = atomicExch(&c.lens[s], 0);
  __syncthreads();
  const int32_t len = held < 0 ? 0 : (held > c.capacity ? c.capacity : held);
  int32_t *row = c.tables + (int64_t)s * c.max_pages;
  for (int x = tid; x < pages_of(len, c.log_page); x += ROW_THREADS) {
    const int32_t p = row[x];
    if (p >= 0 && p < c.num_pages) atomicSub(&c.refs[p], 1);
    row[x] = -1;
  }
}

// ------------------------------------------------------------------- compact
struct Moves {
  int32_t live, count;
};

// One search finds both ends of the moves: with `live` pages in use, the free pages
// before page `live` and then the used ones from it on, equally many.  `list` receives
// the former (targets), then the latter (sources).
__global__ void __launch_bounds__(PLAN_THREADS)
cache_compact_plan_kernel(CacheDev c, Moves *mv, int32_t *list, int32_t *to, int32_t *live_out) {
  __shared__ int32_t sums[PLAN_WAVES];
  __shared__ CollectSmem cs;
  const int tid = threadIdx.x;
  int32_t counts[ROUND], mine = 0;
  for (int64_t p0 = ROUND * PLAN_THREADS; p0 < c.num_pages; p0 += ROUND * PLAN_THREADS) {
    load_counts(c.refs, p0, c.num_pages, tid, counts);
#pragma unroll
    for (int k = 0; k < ROUND; ++k) mine += counts[k] != 0 ? 1 : 0;
  }
  load_counts(c.refs, 0, c.num_pages, tid, counts);           // (kept for the search)
#pragma unroll
  for (int k = 0; k < ROUND; ++k) mine += counts[k] != 0 ? 1 : 0;
  int32_t live = 0;
  block_prefix(mine, sums, tid, live);
  const int32_t found = collect(c.refs, c.num_pages, list, c.num_pages, cs, tid, counts,
                                [live](int32_t p, int32_t count) {
                                  return p < live ? count == 0 : count != 0;
                                });
  const int32_t m = found / 2;
  __syncthreads();
  for (int x = tid; x < m; x += PLAN_THREADS) {
    const int32_t d = list[x], s = list[m + x];
    to[s] = d;
    c.refs[d] = c.refs[s];
    c.refs[s] = 0;
  }
  if (tid == 0) {
    *mv = Moves{live, m};
    *live_out = live;
  }
}

// The pages' rows (a work-group a page of one pool at a time) and the tables.
__global__ void __launch_bounds__(ROW_THREADS)
cache_compact_move_kernel(CacheDev c, const Moves *mv, const int32_t *list, const int32_t *to) {
  const Moves m = *mv;
  if (m.count == 0) return;
  const int tid = threadIdx.x;
  const int pools = 2 * c.layers;
  const int64_t page = (int64_t)c.row_bytes << c.log_page;
  for (int64_t x = blockIdx.x; x < (int64_t)m.count * pools; x += gridDim.x) {
    const int32_t which = (int32_t)(x / pools), y = (int32_t)(x - (int64_t)which * pools);
    char *pool = ((y & 1) ? c.v : c.k) + (y >> 1) * c.layer_bytes;
    const int64_t d = list[which], s = list[m.count + which];
    copy16(pool + s * page, pool + d * page, page, tid, ROW_THREADS);
    if (c.ts && y == 0)
      for (int t = tid; t < (1 << c.log_page); t += ROW_THREADS)
        c.ts[(d << c.log_page) + t] = c.ts[(s << c.log_page) + t];
  }
  const int64_t entries = (int64_t)c.slots * c.max_pages;
  for (int64_t x = (int64_t)blockIdx.x * ROW_THREADS + tid; x < entries;
       x += (int64_t)gridDim.x * ROW_THREADS) {
    const int32_t p = c.tables[x];
    if (p >= m.live && p < c.num_pages) c.tables[x] = to[p];
  }
}

// ------------------------------------------------------------------ workspace
// extend: owner [slots], plan [slots], copies [slots], fresh [num_pages]; fork: len_of
// [slots], noted [slots][max_pages]; compact: moves, list and to [num_pages].
struct CacheWs {
  size_t owner, plan, copies, fresh, len_of, noted, moves, list, to, total;
};
CacheWs cache_ws(int32_t slots, int32_t num_pages, int32_t max_pages) {
  CacheWs w{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += align_up(bytes);
    return o;
  };
  w.owner = take(sizeof(int32_t) * (size_t)slots);
  w.plan = take(sizeof(RowPlan) * (size_t)slots);
  w.copies = take(sizeof(PageCopy) * (size_t)slots);
  w.fresh = take(sizeof(int32_t) * (size_t)num_pages);
  w.total = at;
  at = 0;
  w.len_of = take(sizeof(int32_t) * (size_t)slots);
  w.noted = take(sizeof(int32_t) * (size_t)slots * (size_t)max_pages);
  w.total = std::max(w.total, at);
  at = 0;
  w.moves = take(sizeof(Moves));
  w.list = take(sizeof(int32_t) * (size_t)num_pages);
  w.to = take(sizeof(int32_t) * (size_t)num_pages);
  w.total = std::max(w.total, at);
  return w;
}

// n rows of one of the row calls.
int check_rows(int32_t n, const CacheDev &d) {
  if (n < 0) return fail(HSTU_EINVAL, "n = %d < 0", n);
  if (n > d.slots) return fail(HSTU_EINVAL, "n = %d rows for %d slots", n, d.slots);
  return HSTU_OK;
}

int launched(const char *what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? HSTU_OK : hip_fail(e, what);
}

}  // namespace

int check_cache(const hstu_cache *c, CacheDev *d) {
  if (!c) return fail(HSTU_EINVAL, "the cache is NULL");
  if (c->dtype != HSTU_BF16 && c->dtype != HSTU_F32)
    return fail(HSTU_EINVAL, "dtype %d is not HSTU_BF16 or HSTU_F32", (int)c->dtype);
  if (c->layers < 1) return fail(HSTU_EINVAL, "layers = %d < 1", c->layers);
  if (c->num_pages < 1) return fail(HSTU_EINVAL, "num_pages = %d < 1", c->num_pages);
  if (c->page_size < 1 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)))
    return fail(HSTU_EINVAL, "page_size = %d is not a power of two up to 1024", c->page_size);
  if (c->H < 1) return fail(HSTU_EINVAL, "H = %d < 1", c->H);
  if (c->H > 64) return fail(HSTU_ENOTSUP, "H = %d > 64", c->H);
  if (c->d != 32 && c->d != 64 && c->d != 128)
    return fail(HSTU_EINVAL, "d = %d is not 32, 64 or 128", c->d);
  if (c->dtype == HSTU_BF16 && c->d == 32)
    return fail(HSTU_ENOTSUP, "bf16 path supports d = 64 or 128, got 32");
  if (c->slots < 1) return fail(HSTU_EINVAL, "slots = %d < 1", c->slots);
  if (c->slots > 1 << 24) return fail(HSTU_ENOTSUP, "slots = %d > 2^24", c->slots);
  if (c->max_pages < 1) return fail(HSTU_EINVAL, "max_pages = %d < 1", c->max_pages);
  if ((int64_t)c->num_pages * c->page_size > INT32_MAX)
    return fail(HSTU_ENOTSUP, "num_pages * page_size = %lld >= 2^31",
                (long long)c->num_pages * c->page_size);
  if ((int64_t)c->max_pages * c->page_size > INT32_MAX)
    return fail(HSTU_ENOTSUP, "max_pages * page_size = %lld >= 2^31",
                (long long)c->max_pages * c->page_size);
  if (c->layers > 16384) return fail(HSTU_ENOTSUP, "layers = %d > 16384", c->layers);
  if (!c->k || !c->v || !c->tables || !c->lens || !c->refs || !c->status)
    return fail(HSTU_EINVAL, "the cache's k, v, tables, lens, refs and status must be non-null");
  if (((uintptr_t)c->k | (uintptr_t)c->v) % 16)
    return fail(HSTU_EINVAL, "the cache's k and v must be 16-byte aligned");
  d->k = (char *)c->k;
  d->v = (char *)c->v;
  d->ts = c->ts;
  d->tables = c->tables;
  d->lens = c->lens;
  d->refs = c->refs;
  d->status = c->status;
  d->layers = c->layers;
  d->num_pages = c->num_pages;
  d->log_page = __builtin_ctz((unsigned)c->page_size);
  d->slots = c->slots;
  d->max_pages = c->max_pages;
  d->capacity = c->max_pages * c->page_size;
  d->row_bytes = c->H * c->d * (c->dtype == HSTU_BF16 ? 2 : 4);
  d->layer_bytes = (int64_t)c->num_pages * c->page_size * d->row_bytes;
  return HSTU_OK;
}

}  // namespace hstu

using namespace hstu;

extern "C" {

size_t hstu_cache_workspace_bytes(const hstu_cache *c) {
  clear_last_error();
  CacheDev d;
  if (check_cache(c, &d) != HSTU_OK) return 0;
  return cache_ws(d.slots, d.num_pages, d.max_pages).total;
}

int hstu_cache_clear(const hstu_cache *c, void *stream) {
  clear_last_error();
  CacheDev d;
  const int rc = check_cache(c, &d);
  if (rc != HSTU_OK) return rc;
  hipStream_t s = (hipStream_t)stream;
  prof::Scope ps("cache_clear", s);
  hipLaunchKernelGGL(cache_clear_kernel, dim3(256), dim3(256), 0, s, d);
  return launched("cache clear launch");
}

int hstu_cache_extend(const hstu_cache *c, const int32_t *slot_ids, const int32_t *counts,
                      int32_t n, int32_t *start, void *workspace, size_t workspace_bytes,
                      void *stream) {
  clear_last_error();
  CacheDev d;
  int rc = check_cache(c, &d);
  if (rc == HSTU_OK) rc = check_rows(n, d);
  if (rc != HSTU_OK || n == 0) return rc;
  if (!slot_ids || !counts || !start)
    return fail(HSTU_EINVAL, "slot_ids, counts and start must be non-null");
  const CacheWs w = cache_ws(d.slots, d.num_pages, d.max_pages);
  if ((rc = check_workspace_bytes(w.total, workspace, workspace_bytes)) != HSTU_OK) return rc;
  char *ws = (char *)workspace;
  hipStream_t s = (hipStream_t)stream;
  PageCopy *copies = (PageCopy *)(ws + w.copies);
  {
    prof::Scope ps("cache_extend", s);
    hipLaunchKernelGGL(cache_extend_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, d, slot_ids, counts,
                       n, start, (int32_t *)(ws + w.owner), (RowPlan *)(ws + w.plan),
                       (int32_t *)(ws + w.fresh), copies);
  }
  if ((rc = launched("cache extend launch")) != HSTU_OK) return rc;
  prof::Scope ps("cache_copy", s);
  hipLaunchKernelGGL(cache_copy_kernel, dim3((unsigned)n, 2 * (unsigned)d.layers),
                     dim3(ROW_THREADS), 0, s, d, (const PageCopy *)copies);
  return launched("cache copy launch");
}

int hstu_cache_write(const hstu_cache *c, int32_t layer, const void *k, const void *v,
                     const int64_t *timestamps, const int32_t *slot_ids, const int32_t *start,
                     const int64_t *row_offsets, int32_t n, int64_t total_rows, int32_t max_new,
                     void *stream) {
  clear_last_error();
  CacheDev d;
  int rc = check_cache(c, &d);
  if (rc == HSTU_OK) rc = check_rows(n, d);
  if (rc != HSTU_OK) return rc;
  if (layer < 0 || layer >= d.layers)
    return fail(HSTU_EINVAL, "layer = %d of %d", layer, d.layers);
  if (total_rows < 0) return fail(HSTU_EINVAL, "total_rows = %lld < 0", (long long)total_rows);
  if (max_new < 0) return fail(HSTU_EINVAL, "max_new = %d < 0", max_new);
  if (timestamps && !d.ts)
    return fail(HSTU_EINVAL, "timestamps given for a cache without ts");
  if (n == 0 || total_rows == 0 || max_new == 0) return HSTU_OK;
  if (!k || !v || !slot_ids || !start || !row_offsets)
    return fail(HSTU_EINVAL, "k, v, slot_ids, start and row_offsets must be non-null");
  if (((uintptr_t)k | (uintptr_t)v) % 16)
    return fail(HSTU_EINVAL, "k and v must be 16-byte aligned");
  const int64_t groups = total_rows / WRITE_TOKENS + n;        // (see write_base)
  if (groups > 1 << 24)
    return fail(HSTU_ENOTSUP, "total_rows = %lld > 2^28 - 16 n", (long long)total_rows);
  hipStream_t s = (hipStream_t)stream;
  prof::Scope ps("cache_write", s);
  hipLaunchKernelGGL(cache_write_kernel, dim3((unsigned)groups), dim3(ROW_THREADS), 0, s, d, layer,
                     (const char *)k, (const char *)v, timestamps, slot_ids, start, row_offsets, n,
                     total_rows, max_new);
  return launched("cache write launch");
}

int hstu_cache_fork(const hstu_cache *c, const int32_t *src, const int32_t *dst, int32_t n,
                    void *workspace, size_t workspace_bytes, void *stream) {
  clear_last_error();
  CacheDev d;
  int rc = check_cache(c, &d);
  if (rc == HSTU_OK) rc = check_rows(n, d);
  if (rc != HSTU_OK || n == 0) return rc;
  if (!src || !dst) return fail(HSTU_EINVAL, "src and dst must be non-null");
  const CacheWs w = cache_ws(d.slots, d.num_pages, d.max_pages);
  if ((rc = check_workspace_bytes(w.total, workspace, workspace_bytes)) != HSTU_OK) return rc;
  char *ws = (char *)workspace;
  hipStream_t s = (hipStream_t)stream;
  prof::Scope ps("cache_fork", s);
  hipLaunchKernelGGL(cache_fork_note_kernel, dim3((unsigned)n), dim3(ROW_THREADS), 0, s, d, src,
                     dst, (int32_t *)(ws + w.len_of), (int32_t *)(ws + w.noted));
  if ((rc = launched("cache fork launch")) != HSTU_OK) return rc;
  hipLaunchKernelGGL(cache_fork_set_kernel, dim3((unsigned)n), dim3(ROW_THREADS), 0, s, d, dst,
                     (const int32_t *)(ws + w.len_of), (const int32_t *)(ws + w.noted));
  return launched("cache fork launch");
}

int hstu_cache_free(const hstu_cache *c, const int32_t *slot_ids, int32_t n, void *stream) {
  clear_last_error();
  CacheDev d;
  int rc = check_cache(c, &d);
  if (rc == HSTU_OK) rc = check_rows(n, d);
  if (rc != HSTU_OK || n == 0) return rc;
  if (!slot_ids) return fail(HSTU_EINVAL, "slot_ids must be non-null");
  hipStream_t s = (hipStream_t)stream;
  prof::Scope ps("cache_free", s);
  hipLaunchKernelGGL(cache_free_kernel, dim3((unsigned)n), dim3(ROW_THREADS), 0, s, d, slot_ids);
  return launched("cache free launch");
}

int hstu_cache_compact(const hstu_cache *c, int32_t *live, void *workspace, size_t workspace_bytes,
                       void *stream) {
  clear_last_error();
  CacheDev d;
  int rc = check_cache(c, &d);
  if (rc != HSTU_OK) return rc;
  if (!live) return fail(HSTU_EINVAL, "live must be non-null");
  const CacheWs w = cache_ws(d.slots, d.num_pages, d.max_pages);
  if ((rc = check_workspace_bytes(w.total, workspace, workspace_bytes)) != HSTU_OK) return rc;
  int dev = 0;
  if ((rc = current_device(&dev)) != HSTU_OK) return rc;
  char *ws = (char *)workspace;
  hipStream_t s = (hipStream_t)stream;
  int32_t *list = (int32_t *)(ws + w.list), *to = (int32_t *)(ws + w.to);
  {
    prof::Scope ps("cache_compact_plan", s);
    hipLaunchKernelGGL(cache_compact_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, d,
                       (Moves *)(ws + w.moves), list, to, live);
  }
  if ((rc = launched("cache compact launch")) != HSTU_OK) return rc;
  prof::Scope ps("cache_compact_move", s);
  hipLaunchKernelGGL(cache_compact_move_kernel, dim3(8u * (unsigned)device_info(dev).num_cu),
                     dim3(ROW_THREADS), 0, s, d, (const Moves *)(ws + w.moves),
                     (const int32_t *)list, (const int32_t *)to);
  return launched("cache compact launch");
}

}  // extern "C"
