// Attention of one new token of every sequence over the paged cache, split over the
// sequences' length and joined.
//
//   o = sum over seen j of silu(alpha <q, k_j> + bias_j) / N v_j
//
// There is no softmax, so a chunk's result is a plain sum and the join adds the
// chunks' sums in order.  A token costs 4 d H operations and 2 rows of d H elements
// read once: two operations a byte in bf16, far below what the vector ALUs give, so
// HBM bounds it, and the products stay on the vector ALUs (a matrix instruction would
// work on 16 rows where there is one).
//
// Layout: a lane holds 16 bytes of one head's row, so a head takes LPH = row bytes / 16
// lanes and a wave holds HS = 64 / LPH head slots: `hpw` heads (the largest power of
// two that divides H, at most HS, so that no lane idles) of 64 / (LPH hpw) tokens.  A
// lane keeps its head and columns for the whole chunk: q in 8 (or 4) registers, the
// sum in as many, and nothing crosses lanes but the score (a DPP sum over the LPH
// lanes) and, at the end, the sums of the waves and token slots through LDS.
// The biases of a group's (token, head) pairs are found by one lane each, for U steps
// at once, and handed out by shuffles, so the bucket rule does not run in every lane.
//
// Work: with `total` seen tokens in the batch a chunk is about total / target tokens,
// the same for all sequences, so that the last work-group ends with the others; every
// work-group finds its own chunk from the lengths (two scans over the batch), which
// costs about a microsecond and saves a launch that would plan.
#include <algorithm>
#include <cmath>

#include "cache.h"
#include "device.h"

namespace hstu {

namespace {

constexpr int THREADS = 256;
constexpr int WAVES = THREADS / 64;
// Steps (16 bytes of k and of v a lane) in flight.  Four steps, four waves a SIMD and
// as many work-groups as fit at once (CHUNKS_PER_CU) measured best; 128 sequences of up
// to 4096 tokens, 4 heads of 128 / 32 of up to 65536, 8 heads (us, whole call): 45 /
// 906; two steps 48 / 942, eight steps on three waves a SIMD 57 / 956 (eight chunks a
// compute unit 52 / 848: the long batch would gain, the usual one lose), work-groups of
// 512 threads 52 / 984.
constexpr int U = 4;

struct PParams {
  CacheDev c;
  const char *kl, *vl;                       // the layer's pools
  const void *q, *u;
  const float *pos_w, *time_w;
  const int32_t *slot_ids;
  void *o, *y;
  float *part;                               // [chunks][H * d]
  int2 *chunks;                              // [rows] first chunk, number of chunks
  int32_t rows, N, nb, H, d;
  int32_t window, sinks;
  int32_t log_hpw;                           // log2 of the heads of a wave
  int32_t target;                            // chunks to aim at
  float alpha;
};

struct Chunk {
  int32_t row, slot, len, x0, x1;            // seen tokens x0 .. x1 - 1 of the row
  Seen seen;
};

// k and v are read once: non-temporal loads keep them from displacing what is used
// again (U = 8: 62 / 1040 us without, 57 / 956 with).
__device__ __forceinline__ uint4 load_once(const char *p) {
  typedef unsigned u32x4n __attribute__((ext_vector_type(4)));
  const u32x4n v = __builtin_nontemporal_load((const u32x4n *)p);
  return make_uint4(v[0], v[1], v[2], v[3]);
}

struct ScanSmem {
  int64_t sums[WAVES];
  Chunk mine;
};

__device__ __forceinline__ Seen row_seen(const PParams &P, int r, int32_t &slot, int32_t &len) {
  slot = P.slot_ids[r];
  len = slot_len(P.c.lens, P.c.slots, P.c.capacity, slot);
  return seen_by_last(len, P.window, P.sinks);
}

// Sum over the work-group; every thread gets it.
__device__ __forceinline__ int64_t block_sum(int64_t x, int64_t *sums, int tid) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(x, m, 64);
  if ((tid & 63) == 0) sums[tid >> 6] = x;
  __syncthreads();
  int64_t all = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) all += sums[w];
  __syncthreads();
  return all;
}

// The work-group's chunk `item` of the batch, in row order; false past the last one.
// Rows are looked at THREADS at a time, all of them in both scans (the first THREADS
// are kept from one to the other).  The first work-group notes every row's chunks for
// the join.
__device__ __forceinline__ bool find_chunk(const PParams &P, int item, int step, ScanSmem &sm,
                                           int tid) {
  int32_t slot0 = -1, len0 = 0;
  Seen s0{0, 0, 0};
  if (tid < P.rows) s0 = row_seen(P, tid, slot0, len0);
  int64_t total = s0.count;
  for (int r = tid + THREADS; r < P.rows; r += THREADS) {
    int32_t slot, len;
    total += row_seen(P, r, slot, len).count;
  }
  total = block_sum(total, sm.sums, tid);
  const int32_t C = chunk_len(total, P.target, step);
  if (tid == 0) sm.mine.row = -1;
  __syncthreads();
  int32_t before = 0;
  const bool notes = blockIdx.x == 0 && blockIdx.y == 0;
  for (int r0 = 0; r0 < P.rows && (before <= item || notes); r0 += THREADS) {
    const int r = r0 + tid;
    Seen s = s0;
    int32_t slot = slot0, len = len0;
    if (r0 > 0) {
      s = Seen{0, 0, 0};
      if (r < P.rows) s = row_seen(P, r, slot, len);
    }
    const int32_t n = chunks_of(s.count, C);
    const int32_t incl = wave_prefix(n);
    if ((tid & 63) == 63) sm.sums[tid >> 6] = incl;
    __syncthreads();
    int32_t first = before + incl - n, all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const int32_t x = (int32_t)sm.sums[w];
      first += w < (tid >> 6) ? x : 0;
      all += x;
    }
    if (item >= first && item < first + n) {
      const int32_t x0 = (item - first) * C;
      sm.mine = Chunk{r, slot, len, x0, chunk_end(x0, s.count, C), s};
    }
    if (notes && r < P.rows) P.chunks[r] = make_int2(first, n);
    before += all;
    __syncthreads();
  }
  return sm.mine.row >= 0;
}

// ------------------------------------------------------------- element types
template <typename T> struct Elem;
template <> struct Elem<u16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(uint4 x, float (&f)[8]) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[2 * e] = __uint_as_float(w[e] << 16);
      f[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ float to_float(u16 x) { return bf2f(x); }
  static __device__ __forceinline__ u16 from_float(float x) {
    return (u16)(pack2(x, x) & 0xffffu);
  }
};
template <> struct Elem<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(uint4 x, float (&f)[4]) {
    f[0] = __uint_as_float(x.x); f[1] = __uint_as_float(x.y);
    f[2] = __uint_as_float(x.z); f[3] = __uint_as_float(x.w);
  }
  static __device__ __forceinline__ float to_float(float x) { return x; }
  static __device__ __forceinline__ float from_float(float x) { return x; }
};

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(
                                           0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}

// Sum over aligned groups of LPH lanes, in every lane: within quads, then (all lanes of
// a quad alike) by mirroring halves and rows of 16.
template <int LPH>
__device__ __forceinline__ float head_sum(float x) {
  static_assert(LPH == 8 || LPH == 16 || LPH == 32, "lanes of a head");
  x = dpp_add<0xB1>(x);                                  // quad_perm 1,0,3,2
  x = dpp_add<0x4E>(x);                                  // quad_perm 2,3,0,1
  x = dpp_add<0x141>(x);                                 // row_half_mirror
  if constexpr (LPH >= 16) x = dpp_add<0x140>(x);        // row_mirror
  if constexpr (LPH >= 32) x += __shfl_xor(x, 16, 64);
  return x;
}

template <typename T, int D>
__global__ void __launch_bounds__(THREADS, 4)
paged_attn_kernel(PParams P) {
  constexpr int E = Elem<T>::N;              // elements of a lane
  constexpr int LPH = D / E, HS = 64 / LPH;
  constexpr int LOG_HS = HS == 8 ? 3 : HS == 4 ? 2 : 1;
  __shared__ ScanSmem sm;
  __shared__ float red[WAVES][64][E + 1];
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int log_tpw = LOG_HS - P.log_hpw, tpw = 1 << log_tpw, hpw = 1 << P.log_hpw;
  const int gt = U << log_tpw;               // tokens of a group of steps
  if (!find_chunk(P, blockIdx.x, WAVES * gt, sm, tid)) return;
  const Chunk ch = sm.mine;
  const int32_t *table = P.c.tables + (int64_t)ch.slot * P.c.max_pages;
  const int32_t last = ch.len - 1;

  // this lane's head, columns and token slot
  const int hslot = lane / LPH, sub = lane % LPH;
  const int head = (int)blockIdx.y * hpw + (hslot & (hpw - 1)), tslot = hslot >> P.log_hpw;
  const uint32_t col = (uint32_t)(head * D + sub * E) * sizeof(T);
  // ... and the (step, head slot) pair whose bias it finds
  const int bstep = lane / HS, bhs = lane % HS;
  const int bhead = (int)blockIdx.y * hpw + (bhs & (hpw - 1));
  const int btok = (bstep << log_tpw) + (bhs >> P.log_hpw);
  const bool pair = lane < U * HS;

  float q[E];
  Elem<T>::unpack(*(const uint4 *)((const char *)P.q +
                                   (int64_t)ch.row * P.H * D * sizeof(T) + col), q);
  int64_t ts_last = 0;
  if (P.time_w) {
    const int32_t r = page_row(table[last >> P.c.log_page], P.c.num_pages, P.c.log_page, last);
    ts_last = r >= 0 ? P.c.ts[r] : 0;
  }
  const float inv_n = 1.0f / (float)P.N;
  float acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.0f;

  // pool row of token t of a group from x0 on, -1 past the chunk or without a page
  auto row_at = [&](int x) -> int32_t {
    if (x >= ch.x1) return -1;
    const int32_t pos = ch.seen.at(x);
    return page_row(table[pos >> P.c.log_page], P.c.num_pages, P.c.log_page, pos);
  };
  int x0 = ch.x0 + w * gt;
  int32_t row = lane < gt ? row_at(x0 + lane) : -1;
  for (; x0 < ch.x1; x0 += WAVES * gt) {
    uint4 kx[U], vx[U];
    uint32_t have = 0;
#pragma unroll
    for (int s = 0; s < U; ++s) {
      const int32_t r = __shfl(row, (s << log_tpw) + tslot, 64);
      have |= r >= 0 ? 1u << s : 0u;
      const int64_t at = (int64_t)(r >= 0 ? r : 0) * P.c.row_bytes + col;
      kx[s] = load_once(P.kl + at);
      vx[s] = load_once(P.vl + at);
    }
    // the biases of the group's pairs, a lane each
    float bias = 0.0f;
    if (P.pos_w || P.time_w) {
      const int32_t brow = __shfl(row, btok, 64);
      const int x = x0 + btok;
      if (pair && brow >= 0) {
        if (P.pos_w) {
          const int64_t i = (int64_t)ch.seen.at(x) - last + P.N - 1;
          if (i >= 0 && i < 2 * (int64_t)P.N - 1)
            bias = P.pos_w[(int64_t)bhead * (2 * (int64_t)P.N - 1) + i];
        }
        if (P.time_w)
          bias += P.time_w[bhead * P.nb + time_bucket32(ts_last - P.c.ts[brow], P.nb)];
      }
    }
    // the next group's rows, whose loads end under this group's products
    const int xn = x0 + WAVES * gt;
    row = lane < gt && xn < ch.x1 ? row_at(xn + lane) : -1;
#pragma unroll
    for (int s = 0; s < U; ++s) {
      float f[E], dot = 0.0f;
      Elem<T>::unpack(kx[s], f);
#pragma unroll
      for (int e = 0; e < E; ++e) dot = __builtin_fmaf(q[e], f[e], dot);
      dot = head_sum<LPH>(dot);
      const float x = __builtin_fmaf(P.alpha, dot, __shfl(bias, s * HS + hslot, 64));
      const float a = x * sigmoid_f(x) * inv_n;
      Elem<T>::unpack(vx[s], f);
      // a token that is not there adds nothing, whatever lies in the pool's first row
      if ((have >> s) & 1) {
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = __builtin_fmaf(a, f[e], acc[e]);
      }
    }
  }

  // the waves and token slots of each head and column, added in order
#pragma unroll
  for (int e = 0; e < E; ++e) red[w][lane][e] = acc[e];
  __syncthreads();
  float *out = P.part + (int64_t)blockIdx.x * P.H * D + (int64_t)blockIdx.y * hpw * D;
  for (int x = tid; x < hpw * D; x += THREADS) {
    const int l = x / E, e = x % E;          // lane of token slot 0
    float sum = 0.0f;
    for (int ww = 0; ww < WAVES; ++ww)
      for (int t = 0; t < tpw; ++t) sum += red[ww][l + t * (hpw * LPH)][e];
    out[x] = sum;
  }
}

// --------------------------------------------------------------------- join
constexpr int JOIN_THREADS = 512;
constexpr int JOIN_WAVES = JOIN_THREADS / 64;

__device__ __forceinline__ float join_sum(float x, float *sums, int tid) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(x, m, 64);
  if ((tid & 63) == 0) sums[tid >> 6] = x;
  __syncthreads();
  float all = 0.0f;
#pragma unroll
  for (int w = 0; w < JOIN_WAVES; ++w) all += sums[w];
  __syncthreads();
  return all;
}

// One work-group a row: the chunks' sums added (groups of threads take every
// `slices`-th chunk, whose sums are added in order), rounded to the output's type as
// the plain forward rounds o before LayerNorm reads it, then LayerNorm x u.
template <typename T>
__global__ void __launch_bounds__(JOIN_THREADS)
paged_join_kernel(PParams P) {
  extern __shared__ float sh[];               // [slices][F]; o at last in the first F
  __shared__ float sums[JOIN_WAVES];
  const int r = blockIdx.x, tid = threadIdx.x;
  const int F = P.H * P.d, F4 = F / 4;
  const int2 mine = P.chunks[r];              // (x is in the buffer also where y is 0)
  const int slices = F4 < JOIN_THREADS ? JOIN_THREADS / F4 : 1;
  float4 *part = (float4 *)sh;
  float *o = sh;                              // (a thread writes what it alone reads)
  const float4 *src = (const float4 *)P.part + (int64_t)mine.x * F4;
  for (int x = tid; x < slices * F4; x += JOIN_THREADS) {
    const int c0 = x / F4, col = x - c0 * F4;
    float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int c = c0; c < mine.y; c += slices) {
      const float4 b = src[(int64_t)c * F4 + col];
      a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
    }
    part[x] = a;
  }
  __syncthreads();
  float sum = 0.0f;
  for (int f = tid; f < F; f += JOIN_THREADS) {
    float a = 0.0f;
    for (int c = 0; c < slices; ++c) a += sh[(size_t)c * F + f];
    const T v = Elem<T>::from_float(a);
    ((T *)P.o)[(int64_t)r * F + f] = v;
    o[f] = Elem<T>::to_float(v);
    sum += o[f];
  }
  const float mean = join_sum(sum, sums, tid) / (float)F;
  float sq = 0.0f;
  for (int f = tid; f < F; f += JOIN_THREADS) sq += (o[f] - mean) * (o[f] - mean);
  const float rstd = rsqrtf(join_sum(sq, sums, tid) / (float)F + HSTU_LN_EPS);
  for (int f = tid; f < F; f += JOIN_THREADS) {
    const int64_t at = (int64_t)r * F + f;
    ((T *)P.y)[at] =
        Elem<T>::from_float((o[f] - mean) * rstd * Elem<T>::to_float(((const T *)P.u)[at]));
  }
}

// ------------------------------------------------------------------ launches
// Heads of a wave: the largest power of two that divides H, at most what fits.
int log_heads_per_wave(const hstu_cache *c) {
  const int lph = c->d * (c->dtype == HSTU_BF16 ? 2 : 4) / 16;
  int l = 0;
  while (!((c->H >> l) & 1) && (2 << l) * lph <= 64) ++l;
  return l;
}

// Chunks to aim at: CHUNKS_PER_CU work-groups for a compute unit over all head groups.
constexpr int CHUNKS_PER_CU = 4;
int target_chunks(const hstu_cache *c, int dev) {
  const int groups = c->H >> log_heads_per_wave(c);
  return std::max(1, CHUNKS_PER_CU * device_info(dev).num_cu / groups);
}

struct PagedWs {
  size_t chunks, part, total;
};
PagedWs paged_ws(const hstu_cache *c, int32_t rows, int dev) {
  PagedWs w;
  w.chunks = 0;
  w.part = align_up(sizeof(int2) * (size_t)rows);
  w.total = w.part + align_up(sizeof(float) * (size_t)c->H * c->d *
                              (size_t)(target_chunks(c, dev) + rows));
  return w;
}

int check_paged_rows(int32_t rows) {
  if (rows < 0) return fail(HSTU_EINVAL, "rows = %d < 0", rows);
  if (rows > 65536) return fail(HSTU_ENOTSUP, "rows = %d > 65536", rows);
  return HSTU_OK;
}

}  // namespace

}  // namespace hstu

using namespace hstu;

extern "C" {

size_t hstu_paged_attn_workspace_bytes(const hstu_cache *c, int32_t rows) {
  clear_last_error();
  CacheDev d;
  int dev = 0;
  if (check_cache(c, &d) != HSTU_OK || check_paged_rows(rows) != HSTU_OK ||
      current_device(&dev) != HSTU_OK)
    return 0;
  return std::max(paged_ws(c, rows, dev).total, kAlign);
}

int hstu_paged_attn_fwd(const void *q, const void *u, const hstu_cache *c, int32_t layer,
                        const int32_t *slot_ids, int32_t rows, int32_t max_len,
                        const hstu_rab *rab, const hstu_window *win, hstu_paged_out *out,
                        void *stream) {
  clear_last_error();
  PParams P{};
  int rc = check_cache(c, &P.c);
  if (rc == HSTU_OK) rc = check_paged_rows(rows);
  if (rc != HSTU_OK) return rc;
  if (layer < 0 || layer >= c->layers)
    return fail(HSTU_EINVAL, "layer = %d of %d", layer, c->layers);
  if (!out) return fail(HSTU_EINVAL, "out is NULL");
  // sizes, tables and the window as for the jagged calls (the type is checked already;
  // the bf16 kernels' limit on H * num_buckets, which their LDS tables set, is not ours)
  static const char dummy = 0;
  Problem p;
  hstu_rab r = rab ? *rab : hstu_rab{};
  r.timestamps = (const int64_t *)&dummy;      // the cache's ts stand in for them
  rc = validate(&dummy, &dummy, &dummy, &dummy, (const int64_t *)&dummy, 1, max_len, c->H, c->d,
                &r, HSTU_F32, 1, &p);
  if (rc == HSTU_OK) rc = set_window(win, &p);
  if (rc != HSTU_OK) return rc;
  if (p.has_time && !c->ts)
    return fail(HSTU_EINVAL, "rab->time_w given for a cache without ts");
  if (rows == 0) return HSTU_OK;
  if (!q || !u || !slot_ids || !out->y || !out->o)
    return fail(HSTU_EINVAL, "q, u, slot_ids, out->y and out->o must be non-null");
  if (((uintptr_t)q) % 16) return fail(HSTU_EINVAL, "q must be 16-byte aligned");
  int dev = 0;
  if ((rc = current_device(&dev)) != HSTU_OK) return rc;
  const PagedWs ws = paged_ws(c, rows, dev);
  if ((rc = check_workspace_bytes(ws.total, out->workspace, out->workspace_bytes)) != HSTU_OK)
    return rc;
  P.kl = P.c.k + layer * P.c.layer_bytes;
  P.vl = P.c.v + layer * P.c.layer_bytes;
  P.q = q;
  P.u = u;
  P.pos_w = p.has_pos ? r.pos_w : nullptr;
  P.time_w = p.has_time ? r.time_w : nullptr;
  P.slot_ids = slot_ids;
  P.o = out->o;
  P.y = out->y;
  P.chunks = (int2 *)((char *)out->workspace + ws.chunks);
  P.part = (float *)((char *)out->workspace + ws.part);
  P.rows = rows;
  P.N = max_len;
  P.nb = p.nb;
  P.H = c->H;
  P.d = c->d;
  P.window = win ? p.window : max_len;
  P.sinks = p.sinks;
  P.log_hpw = log_heads_per_wave(c);
  P.target = target_chunks(c, dev);
  P.alpha = p.alpha;
  hipStream_t s = (hipStream_t)stream;
  const dim3 grid((unsigned)(P.target + rows), (unsigned)(P.H >> P.log_hpw));
  {
    prof::Scope ps("paged_attn", s);
    if (c->dtype == HSTU_BF16) {
      auto kfn = c->d == 64 ? paged_attn_kernel<u16, 64> : paged_attn_kernel<u16, 128>;
      hipLaunchKernelGGL(kfn, grid, dim3(THREADS), 0, s, P);
    } else {
      auto kfn = c->d == 32   ? paged_attn_kernel<float, 32>
                 : c->d == 64 ? paged_attn_kernel<float, 64>
                              : paged_attn_kernel<float, 128>;
      hipLaunchKernelGGL(kfn, grid, dim3(THREADS), 0, s, P);
    }
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "paged attention launch");
  const int F = P.H * P.d;
  const size_t sh =
      sizeof(float) * F * (size_t)(F / 4 < JOIN_THREADS ? JOIN_THREADS / (F / 4) : 1);
  {
    prof::Scope ps("paged_join", s);
    auto kfn = c->dtype == HSTU_BF16 ? paged_join_kernel<u16> : paged_join_kernel<float>;
    hipLaunchKernelGGL(kfn, dim3((unsigned)rows), dim3(JOIN_THREADS), sh, s, P);
  }
  e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "paged join launch");
  return HSTU_OK;
}

}  // extern "C"
