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

// Writes the pages p of [from, to) whose count is zero (ZERO) or not to out[0 ..], in
// order, until `most` of them are found; returns their number.  All threads.
template <bool ZERO>
__device__ int32_t collect(const int32_t *refs, int32_t from, int32_t to, int32_t *out,
                           int32_t most, CollectSmem &sm, int tid) {
  const int lane = tid & 63, wv = tid >> 6;
  int32_t got = 0;
  for (int64_t p0 = from; p0 < to && got < most; p0 += ROUND * PLAN_THREADS) {
    int32_t c[ROUND];
#pragma unroll
    for (int k = 0; k < ROUND; ++k) {
      const int64_t p = p0 + k * PLAN_THREADS + tid;
      c[k] = p < to ? refs[p] : (ZERO ? 1 : 0);
    }
    uint64_t hit[ROUND];
#pragma unroll
    for (int k = 0; k < ROUND; ++k) {
      hit[k] = __ballot(ZERO ? c[k] == 0 : c[k] != 0);
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

// Copies `bytes` (a multiple of 16) from src to dst, threads tid of nt.
__device__ __forceinline__ void copy16(const char *src, char *dst, int64_t bytes, int tid, int nt) {
  const int64_t n = bytes >> 4;
  int64_t x = tid;
  for (; x + 3 * nt < n; x += 4 * nt) {
    const uint4 a = ((const uint4 *)src)[x], b = ((const uint4 *)src)[x + nt],
                c = ((const uint4 *)src)[x + 2 * nt], d = ((const uint4 *)src)[x + 3 * nt];
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
// A row's plan: pages it needs, the first of them in `fresh`, the shared page that is
// copied (-1: none); `need` < 0: refused.
struct RowPlan {
  int32_t need, base, shared, reserved;
};
// A copy that the second launch makes: `rows` tokens of page src into page dst.
struct PageCopy {
  int32_t src, dst, rows;
};

__global__ void __launch_bounds__(PLAN_THREADS)
cache_extend_kernel(CacheDev c, const int32_t *slot_ids, const int32_t *counts, int32_t n,
                    int32_t *start, int32_t *owner, RowPlan *plan, int32_t *fresh,
                    PageCopy *copies) {
  __shared__ int32_t sums[PLAN_WAVES];
  __shared__ CollectSmem cs;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  // the first row that names a slot owns it
  for (int r = tid; r < n; r += PLAN_THREADS) {
    const int32_t s = slot_ids[r];
    if (s >= 0 && s < c.slots) atomicExch(&owner[s], n);
  }
  __threadfence();
  __syncthreads();
  for (int r = tid; r < n; r += PLAN_THREADS) {
    const int32_t s = slot_ids[r];
    if (s >= 0 && s < c.slots) atomicMin(&owner[s], r);
  }
  __threadfence();
  __syncthreads();

  int64_t run = 0;
  int bad = 0;
  for (int r0 = 0; r0 < n; r0 += PLAN_THREADS) {
    const int r = r0 + tid;
    RowPlan p{-1, 0, -1, 0};
    if (r < n) {
      const int32_t s = slot_ids[r], cnt = counts[r];
      if (s < 0 || s >= c.slots) {
        bad |= HSTU_CACHE_BAD_SLOT;
      } else if (__hip_atomic_load(&owner[s], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != r) {
        bad |= HSTU_CACHE_TWICE;
      } else if (cnt < 0) {
        bad |= HSTU_CACHE_BAD_COUNT;
      } else {
        const int32_t len = slot_len(c.lens, c.slots, c.capacity, s);
        if (cnt > c.capacity - len) {
          bad |= HSTU_CACHE_FULL;
        } else {
          const int32_t had = pages_of(len, c.log_page);
          p.need = pages_of((int64_t)len + cnt, c.log_page) - had;
          if (cnt > 0 && (len & ((1 << c.log_page) - 1)) != 0) {
            const int32_t last = c.tables[(int64_t)s * c.max_pages + had - 1];
            if (last >= 0 && last < c.num_pages && c.refs[last] > 1) {
              p.shared = last;
              ++p.need;
            }
          }
        }
      }
    }
    // two scans, so that 1024 rows of up to 2^31 pages each do not overflow
    int32_t all_hi = 0, all_lo = 0;
    const int32_t want = p.need > 0 ? p.need : 0;
    const int64_t hi = block_prefix(want >> 15, sums, tid, all_hi);
    const int64_t lo = block_prefix(want & 32767, sums, tid, all_lo);
    const int64_t base = run + (hi << 15) + lo;
    p.base = (int32_t)(base < INT32_MAX ? base : INT32_MAX);   // (past every pool)
    if (r < n) plan[r] = p;
    run += ((int64_t)all_hi << 15) + all_lo;
  }
  const int32_t total = (int32_t)(run < c.num_pages ? run : c.num_pages);
  const int32_t got = collect<true>(c.refs, 0, c.num_pages, fresh, total, cs, tid);
  __syncthreads();

  for (int r = wv; r < n; r += PLAN_WAVES) {
    const RowPlan p = plan[r];
    const int32_t s = slot_ids[r];
    const bool ok = p.need == 0 || (p.need > 0 && (int64_t)p.base + p.need <= got);
    if (p.need > 0 && !ok) bad |= HSTU_CACHE_FULL;
    PageCopy pc{-1, -1, 0};
    int32_t at = -1;
    if (ok) {
      const int32_t len = slot_len(c.lens, c.slots, c.capacity, s);
      const int32_t first = pages_of(len, c.log_page) - (p.shared >= 0 ? 1 : 0);
      int32_t *row = c.tables + (int64_t)s * c.max_pages + first;
      for (int x = lane; x < p.need; x += 64) {
        const int32_t page = fresh[p.base + x];
        row[x] = page;
        c.refs[page] = 1;
      }
      if (p.shared >= 0) pc = PageCopy{p.shared, fresh[p.base], len & ((1 << c.log_page) - 1)};
      at = len;
    }
    if (lane == 0) {
      if (ok) {
        c.lens[s] = at + counts[r];
        if (p.shared >= 0) atomicSub(&c.refs[p.shared], 1);
      }
      copies[r] = pc;
      start[r] = at;
    }
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

// One work-group per row and WRITE_TOKENS of its tokens; a thread moves 16 bytes at a
// time, four of them in flight.
__global__ void __launch_bounds__(ROW_THREADS)
cache_write_kernel(CacheDev c, int32_t layer, const char *k, const char *v, const int64_t *ts,
                   const int32_t *slot_ids, const int32_t *start, const int64_t *off,
                   int64_t total) {
  const int r = blockIdx.x, tid = threadIdx.x;
  const int32_t s = slot_ids[r], at0 = start[r];
  int64_t first = off[r], end = off[r + 1];
  if (s < 0 || s >= c.slots || at0 < 0) return;
  first = first < 0 ? 0 : (first > total ? total : first);
  end = end < first ? first : (end > total ? total : end);
  const int64_t t0 = (int64_t)blockIdx.y * WRITE_TOKENS;
  const int64_t left = end - first - t0;
  if (left <= 0) return;
  const int32_t tokens = left < WRITE_TOKENS ? (int32_t)left : WRITE_TOKENS;
  const int32_t *table = c.tables + (int64_t)s * c.max_pages;
  // pool row of token t0 + t, -1 where it has no place
  auto row_of = [&](int32_t t) -> int32_t {
    const int64_t pos = (int64_t)at0 + t0 + t;
    if (pos >= c.capacity) return -1;
    return page_row(table[pos >> c.log_page], c.num_pages, c.log_page, (int32_t)pos);
  };
  const uint32_t units = (uint32_t)c.row_bytes >> 4;           // of a row, k and v each
  const uint32_t all = (uint32_t)tokens * 2 * units;
  char *kp = c.k + layer * c.layer_bytes, *vp = c.v + layer * c.layer_bytes;
  constexpr int U = 4;
  for (uint32_t x0 = tid; x0 < all; x0 += U * ROW_THREADS) {
    uint4 val[U];
    char *to[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const uint32_t x = x0 + i * ROW_THREADS;
      const uint32_t xc = x < all ? x : x0;
      const uint32_t t = xc / (2 * units), rem = xc - t * (2 * units);
      const bool is_v = rem >= units;
      const int64_t col = 16 * (int64_t)(is_v ? rem - units : rem);
      const int32_t row = row_of((int32_t)t);
      val[i] = *(const uint4 *)((is_v ? v : k) + (first + t0 + t) * c.row_bytes + col);
      to[i] = x < all && row >= 0 ? (is_v ? vp : kp) + (int64_t)row * c.row_bytes + col : nullptr;
    }
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (to[i]) *(uint4 *)to[i] = val[i];
  }
  if (ts && tid < tokens) {
    const int32_t row = row_of(tid);
    if (row >= 0) c.ts[row] = ts[first + t0 + tid];
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

__global__ void __launch_bounds__(PLAN_THREADS)
cache_compact_plan_kernel(CacheDev c, Moves *mv, int32_t *src, int32_t *dst, int32_t *to,
                          int32_t *live_out) {
  __shared__ int32_t sums[PLAN_WAVES];
  __shared__ CollectSmem cs;
  const int tid = threadIdx.x;
  int32_t mine = 0;
  for (int64_t p0 = 0; p0 < c.num_pages; p0 += ROUND * PLAN_THREADS) {
#pragma unroll
    for (int k = 0; k < ROUND; ++k) {
      const int64_t p = p0 + k * PLAN_THREADS + tid;
      mine += p < c.num_pages && c.refs[p] != 0 ? 1 : 0;
    }
  }
  int32_t live = 0;
  block_prefix(mine, sums, tid, live);
  const int32_t m = collect<true>(c.refs, 0, live, dst, live, cs, tid);
  collect<false>(c.refs, live, c.num_pages, src, m, cs, tid);
  __syncthreads();
  for (int x = tid; x < m; x += PLAN_THREADS) {
    const int32_t s = src[x], d = dst[x];
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
cache_compact_move_kernel(CacheDev c, const Moves *mv, const int32_t *src, const int32_t *dst,
                          const int32_t *to) {
  const Moves m = *mv;
  if (m.count == 0) return;
  const int tid = threadIdx.x;
  const int pools = 2 * c.layers;
  const int64_t page = (int64_t)c.row_bytes << c.log_page;
  for (int64_t x = blockIdx.x; x < (int64_t)m.count * pools; x += gridDim.x) {
    const int32_t which = (int32_t)(x / pools), y = (int32_t)(x - (int64_t)which * pools);
    char *pool = ((y & 1) ? c.v : c.k) + (y >> 1) * c.layer_bytes;
    const int64_t s = src[which], d = dst[which];
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
// [slots], noted [slots][max_pages]; compact: moves, src, dst, to [num_pages].
struct CacheWs {
  size_t owner, plan, copies, fresh, len_of, noted, moves, src, dst, to, total;
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
  w.src = take(sizeof(int32_t) * (size_t)num_pages);
  w.dst = take(sizeof(int32_t) * (size_t)num_pages);
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
  const int64_t parts = ((int64_t)std::min(max_new, d.capacity) + WRITE_TOKENS - 1) / WRITE_TOKENS;
  if (parts > 65535)
    return fail(HSTU_ENOTSUP, "max_new = %d > %d", max_new, 65535 * WRITE_TOKENS);
  hipStream_t s = (hipStream_t)stream;
  prof::Scope ps("cache_write", s);
  hipLaunchKernelGGL(cache_write_kernel, dim3((unsigned)n, (unsigned)parts), dim3(ROW_THREADS), 0,
                     s, d, layer, (const char *)k, (const char *)v, timestamps, slot_ids, start,
                     row_offsets, total_rows);
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
  int32_t *src = (int32_t *)(ws + w.src), *dst = (int32_t *)(ws + w.dst),
          *to = (int32_t *)(ws + w.to);
  {
    prof::Scope ps("cache_compact_plan", s);
    hipLaunchKernelGGL(cache_compact_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, d,
                       (Moves *)(ws + w.moves), src, dst, to, live);
  }
  if ((rc = launched("cache compact launch")) != HSTU_OK) return rc;
  prof::Scope ps("cache_compact_move", s);
  hipLaunchKernelGGL(cache_compact_move_kernel, dim3(8u * (unsigned)device_info(dev).num_cu),
                     dim3(ROW_THREADS), 0, s, d, (const Moves *)(ws + w.moves),
                     (const int32_t *)src, (const int32_t *)dst, (const int32_t *)to);
  return launched("cache compact launch");
}

}  // extern "C"
