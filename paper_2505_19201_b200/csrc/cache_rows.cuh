// A paged cache that a program holds itself: appending rows, and choosing the pages a query attends to.
#pragma once
#include "common.cuh"

#define CACHE_THREADS 256

// The cache as the kernels see it (dream_cache of the C ABI).
struct CacheView {
  void *k, *v, *bounds;
  const int *page_table;
  long long page_stride, head_stride, token_stride, table_stride;
  int n_pages, page_tokens, page_shift, hkv, n_seqs, pages_per_seq;
  __device__ __forceinline__ bool token_ok(int seq, int slot) const { return seq < n_seqs && slot >= 0 && (slot >> page_shift) < pages_per_seq; }
  // Page that holds entry j of a sequence's table; -1 for a number that is no page.
  __device__ __forceinline__ int page(int seq, int j) const {
    const int p = page_table[(long long)seq * table_stride + j];
    return (unsigned)p < (unsigned)n_pages ? p : -1;
  }
  __device__ __forceinline__ long long at(int p, int kvh, int t) const { return p * page_stride + kvh * head_stride + t * token_stride; }
};
__device__ __forceinline__ void cache_bad_index(int *status) { if (status) atomicMax(status, DREAM_DEV_BAD_INDEX); }

// Eight elements, as one 16-byte vector.
template <typename T> __device__ __forceinline__ void unpack8(const uint4 &q, float (&f)[8]) {
  const T *h = reinterpret_cast<const T *>(&q);
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = to_f(h[i]);
}
template <typename T> __device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  uint4 q;
  T *h = reinterpret_cast<T *>(&q);
#pragma unroll
  for (int i = 0; i < 8; ++i) h[i] = from_f<T>(f[i]);
  return q;
}

struct CacheAppendArgs {
  CacheView c;
  const void *q, *k_new, *v_new;
  long long q_ld, k_ld, v_ld, q_out_ld;
  void *q_out;
  const int *row_seq, *slots, *positions;
  const float2 *rope;                      // [n_pos][rot / 2], or null (rot = 0 then)
  int rows, heads, hd, n_pos, rot, interleaved;
  int main_blocks;                         // blocks per row that move it; behind them one per KV head for the bounds
  int *status;
};

// A head's elements are worked on in units of 16: two vectors whose elements are rotated with one another, a[i] with b[i], or sixteen
// consecutive elements, whose neighbours are (interleaved) or which stay as they are (past rot).  First elements of unit u's two vectors:
__device__ __forceinline__ void append_unit(const CacheAppendArgs &a, int u, int &ia, int &ib) {
  const bool split = u * 16 < a.rot && !a.interleaved;
  ia = split ? u * 8 : u * 16;
  ib = split ? u * 8 + a.rot / 2 : u * 16 + 8;
}
// The rotation of unit u, in 32 bits; rounded once, by whoever stores.
__device__ __forceinline__ void append_rotate(const CacheAppendArgs &a, int u, int pos, float (&x)[8], float (&y)[8]) {
  if (u * 16 >= a.rot) return;
  const float4 *t = reinterpret_cast<const float4 *>(a.rope + (long long)pos * (a.rot / 2) + u * 8);
  float cs[16];
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<float4 *>(cs + 4 * i) = t[i];
  if (!a.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float c = cs[2 * i], s = cs[2 * i + 1], p = x[i], q = y[i];
      x[i] = p * c - q * s;
      y[i] = q * c + p * s;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {            // pair i: elements 2 i and 2 i + 1 of the sixteen
      float &p = i < 4 ? x[2 * i] : y[2 * i - 8], &q = i < 4 ? x[2 * i + 1] : y[2 * i - 7];
      const float c = cs[2 * i], s = cs[2 * i + 1], p0 = p, q0 = q;
      p = p0 * c - q0 * s;
      q = q0 * c + p0 * s;
    }
  }
}

// grid (rows, main_blocks + KV heads with bounds).  Blocks below main_blocks: a thread takes one unit of one head of the row, queries first, then
// keys, then values.  The others: where the row fills its page, the bounds of one KV head of the page, from the rows of this call
// (rotated once more: the same values) and, for tokens that came earlier, from the cache.
template <typename T>
__global__ void __launch_bounds__(CACHE_THREADS)
k_cache_append(const __grid_constant__ CacheAppendArgs a) {
  kernel_entry(TR_k_cache_append);
  const int r = blockIdx.x, seq = a.row_seq[r], slot = a.slots[r], units = a.hd / 16;
  if (seq < 0) return;
  const int pos = a.positions ? a.positions[r] : slot;
  const bool ok = a.c.token_ok(seq, slot) && (!a.rot || (unsigned)pos < (unsigned)a.n_pos);
  if ((int)blockIdx.y < a.main_blocks) {
    const int i = blockIdx.y * CACHE_THREADS + threadIdx.x, hh = i / units, u = i - hh * units;
    if (!ok) {
      if (i == 0) cache_bad_index(a.status);
      return;
    }
    if (hh >= a.heads + 2 * a.c.hkv) return;
    int ia, ib;
    append_unit(a, u, ia, ib);
    const T *src;
    T *dst = nullptr;
    const bool is_v = hh >= a.heads + a.c.hkv;
    if (hh < a.heads) {
      src = (const T *)a.q + r * a.q_ld + (long long)hh * a.hd;
      dst = (T *)a.q_out + r * a.q_out_ld + (long long)hh * a.hd;
    } else {
      const int kvh = hh - a.heads - (is_v ? a.c.hkv : 0), page = a.c.page(seq, slot >> a.c.page_shift);
      src = is_v ? (const T *)a.v_new + r * a.v_ld + (long long)kvh * a.hd : (const T *)a.k_new + r * a.k_ld + (long long)kvh * a.hd;
      if (page < 0) {
        if (u == 0) cache_bad_index(a.status);
        return;
      }
      dst = (T *)(is_v ? a.c.v : a.c.k) + a.c.at(page, kvh, slot & (a.c.page_tokens - 1));
    }
    uint4 va = *reinterpret_cast<const uint4 *>(src + ia), vb = *reinterpret_cast<const uint4 *>(src + ib);
    if (!is_v && u * 16 < a.rot) {
      float x[8], y[8];
      unpack8<T>(va, x);
      unpack8<T>(vb, y);
      append_rotate(a, u, pos, x, y);
      va = pack8<T>(x);
      vb = pack8<T>(y);
    }
    *reinterpret_cast<uint4 *>(dst + ia) = va;
    *reinterpret_cast<uint4 *>(dst + ib) = vb;
    return;
  }
  // ---- bounds
  const int pt = a.c.page_tokens;
  if (!ok || (slot & (pt - 1)) != pt - 1) return;
  __shared__ int from[256];                  // row of this call that holds the page's token, -1: it is in the cache already
  __shared__ float red[2][CACHE_THREADS / 32][256];
  __shared__ int missing;
  const int kvh = blockIdx.y - a.main_blocks, first = slot - (pt - 1), tid = threadIdx.x, page = a.c.page(seq, slot >> a.c.page_shift);
  if (page < 0) return;
  if (tid == 0) missing = 0;
  __syncthreads();
  for (int t = tid; t < pt; t += CACHE_THREADS) {       // as a rule the rows of a sequence stand in order
    const int rr = r - (pt - 1) + t;
    const bool here = rr >= 0 && a.row_seq[rr] == seq && a.slots[rr] == first + t;
    from[t] = here ? rr : -1;
    if (!here) missing = 1;
  }
  __syncthreads();
  if (missing) {
    for (int rr = tid; rr < a.rows; rr += CACHE_THREADS)
      if (a.row_seq[rr] == seq && a.slots[rr] >= first && a.slots[rr] <= slot) from[a.slots[rr] - first] = rr;
    __syncthreads();
  }
  const int u = tid % units, groups = CACHE_THREADS / units;
  int ia, ib;
  append_unit(a, u, ia, ib);
  float lo[16], hi[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) { lo[i] = INFINITY; hi[i] = -INFINITY; }
  for (int t = tid / units; t < pt; t += groups) {
    const int rr = from[t];
    float x[8], y[8];
    if (rr >= 0) {
      const int p = a.positions ? a.positions[rr] : first + t;
      if (a.rot && (unsigned)p >= (unsigned)a.n_pos) continue;         // a row that is not written
      const T *src = (const T *)a.k_new + rr * a.k_ld + (long long)kvh * a.hd;
      unpack8<T>(*reinterpret_cast<const uint4 *>(src + ia), x);
      unpack8<T>(*reinterpret_cast<const uint4 *>(src + ib), y);
      append_rotate(a, u, p, x, y);
#pragma unroll
      for (int i = 0; i < 8; ++i) { x[i] = to_f(from_f<T>(x[i])); y[i] = to_f(from_f<T>(y[i])); }
    } else {
      const T *src = (const T *)a.c.k + a.c.at(page, kvh, t);
      unpack8<T>(*reinterpret_cast<const uint4 *>(src + ia), x);
      unpack8<T>(*reinterpret_cast<const uint4 *>(src + ib), y);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo[i] = fminf(lo[i], x[i]); hi[i] = fmaxf(hi[i], x[i]);
      lo[8 + i] = fminf(lo[8 + i], y[i]); hi[8 + i] = fmaxf(hi[8 + i], y[i]);
    }
  }
  for (int o = units; o < 32; o <<= 1)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      lo[i] = fminf(lo[i], __shfl_xor_sync(0xffffffffu, lo[i], o));
      hi[i] = fmaxf(hi[i], __shfl_xor_sync(0xffffffffu, hi[i], o));
    }
  if ((tid & 31) < units)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int d = i < 8 ? ia + i : ib + i - 8;
      red[0][tid >> 5][d] = lo[i];
      red[1][tid >> 5][d] = hi[i];
    }
  __syncthreads();
  T *out = (T *)a.c.bounds + ((long long)page * a.c.hkv + kvh) * 2 * a.hd;
  for (int i = tid; i < 2 * a.hd; i += CACHE_THREADS) {
    const int which = i >= a.hd, d = i - which * a.hd;
    float m = red[which][0][d];
    for (int w = 1; w < CACHE_THREADS / 32; ++w) m = which ? fmaxf(m, red[1][w][d]) : fminf(m, red[0][w][d]);
    out[i] = from_f<T>(m);
  }
}

// ---------------------------------------------------------------------------------------
// The pages a query attends to.  Scores of pages [keep_first, own - keep_last] as 32-bit keys of the same order (0 is below every number), then the
// place of the cut among them.

struct CacheSelectArgs {
  CacheView c;
  const void *q;
  long long q_ld;
  const int *row_seq, *row_pos;
  int group, hd, budget, keep_first, keep_last;
  uint32_t *keys;                          // [row][KV head][pages_per_seq]
  int *ids;
  int *status;
};

__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return v == v ? u ^ (u & 0x80000000u ? 0xffffffffu : 0x80000000u) : 0u;
}
// Pages up to the row's own; 0 for a row without any.
__device__ __forceinline__ int select_pages(const CacheSelectArgs &a, int seq, int pos) {
  return seq >= 0 && pos >= 0 && a.c.token_ok(seq, pos) ? (pos >> a.c.page_shift) + 1 : 0;
}

#define SCORE_PAGES 64                       // pages of a block
#define SELECT_THREADS 256

// grid (rows * KV heads, ceil(pages_per_seq / SCORE_PAGES)).  A warp takes page after page, its lanes the channels.
template <typename T>
__global__ void __launch_bounds__(CACHE_THREADS)
k_cache_scores(const __grid_constant__ CacheSelectArgs a) {
  kernel_entry(TR_k_cache_scores);
  const int r = blockIdx.x / a.c.hkv, kvh = blockIdx.x % a.c.hkv, seq = a.row_seq[r], pos = a.row_pos[r], n = select_pages(a, seq, pos);
  if (n <= a.budget) return;                 // all of them are kept
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, end = min(n - a.keep_last, (int)(blockIdx.y + 1) * SCORE_PAGES);
  uint32_t *keys = a.keys + (long long)blockIdx.x * a.c.pages_per_seq;
  for (int p = max(a.keep_first, (int)blockIdx.y * SCORE_PAGES) + warp; p < end; p += CACHE_THREADS / 32) {
    const int page = a.c.page(seq, p);
    if (page < 0) {
      if (lane == 0) { cache_bad_index(a.status); keys[p] = 0u; }
      continue;
    }
    const T *lo = (const T *)a.c.bounds + ((long long)page * a.c.hkv + kvh) * 2 * a.hd, *hi = lo + a.hd;
    float best = -INFINITY;
    for (int g = 0; g < a.group; ++g) {
      const T *q = (const T *)a.q + r * a.q_ld + (long long)(kvh * a.group + g) * a.hd;
      double s = 0.0;
      for (int d = lane; d < a.hd; d += 32) {
        const float x = to_f(q[d]);
        s += (double)x * (double)to_f(x >= 0.f ? hi[d] : lo[d]);
      }
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      best = fmaxf(best, (float)s);
    }
    if (lane == 0) keys[p] = order_key(best);
  }
}

// grid (rows * KV heads).  Radix selection of the cut, eight bits a turn, then the kept pages in order.
__global__ void __launch_bounds__(SELECT_THREADS)
k_cache_select(const __grid_constant__ CacheSelectArgs a) {
  kernel_entry(TR_k_cache_select);
  const int r = blockIdx.x / a.c.hkv, seq = a.row_seq[r], pos = a.row_pos[r], n = select_pages(a, seq, pos), tid = threadIdx.x;
  int *ids = a.ids + (long long)blockIdx.x * a.budget;
  if (seq >= 0 && pos >= 0 && !n && tid == 0) cache_bad_index(a.status);
  if (n <= a.budget) {
    for (int i = tid; i < a.budget; i += SELECT_THREADS) ids[i] = i < n ? i : -1;
    return;
  }
  __shared__ int hist[256], scan[SELECT_THREADS / 32], cut_bin, cut_left;
  const uint32_t *keys = a.keys + (long long)blockIdx.x * a.c.pages_per_seq;
  const int p0 = a.keep_first, p1 = n - a.keep_last, lane = tid & 31, warp = tid >> 5;
  int left = a.budget - a.keep_first - a.keep_last;             // to be taken by score: fewer than the p1 - p0 there are
  uint32_t prefix = 0u, mask = 0u;
  for (int shift = 24; shift >= 0 && left > 0; shift -= 8) {
    hist[tid] = 0;
    __syncthreads();
    for (int p = p0 + tid; p < p1; p += SELECT_THREADS)
      if ((keys[p] & mask) == prefix) atomicAdd(hist + (keys[p] >> shift & 255), 1);
    __syncthreads();
    // how many lie in this bin or above: the bin in which the cut falls
    int own = hist[255 - tid], sum = own;
    for (int o = 1; o < 32; o <<= 1) { const int t = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += t; }
    if (lane == 31) scan[warp] = sum;
    __syncthreads();
    for (int w = 0; w < warp; ++w) sum += scan[w];
    if (sum >= left && sum - own < left) { cut_bin = 255 - tid; cut_left = left - (sum - own); }
    __syncthreads();
    prefix |= (uint32_t)cut_bin << shift;
    mask |= 255u << shift;
    left = cut_left;
    __syncthreads();
  }
  // keys above the cut stay, and of those on it the first `left`; without a cut (nothing is taken by score) none
  const bool none = a.budget == a.keep_first + a.keep_last;
  int done = 0, ties = 0;                                       // pages written, pages on the cut passed
  for (int base = 0; base < n; base += SELECT_THREADS) {
    const int p = base + tid;
    const uint32_t key = p >= p0 && p < p1 ? keys[p] : 0u;
    const bool forced = p < n && (p < p0 || p >= p1), cand = p >= p0 && p < p1 && !none, tie = cand && key == prefix;
    // two counts in one scan: ties in the upper half
    int own = tie ? 1 << 16 : 0, sum = own;
    for (int o = 1; o < 32; o <<= 1) { const int t = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += t; }
    __syncthreads();
    if (lane == 31) scan[warp] = sum;
    __syncthreads();
    int tie_at = ties + (sum - own >> 16), all = 0;
    for (int w = 0; w < SELECT_THREADS / 32; ++w) { if (w < warp) tie_at += scan[w] >> 16; all += scan[w] >> 16; }
    ties += all;
    const bool keep = forced || (cand && key > prefix) || (tie && tie_at < left);
    const unsigned b = __ballot_sync(0xffffffffu, keep);
    __syncthreads();
    if (lane == 0) scan[warp] = __popc(b);
    __syncthreads();
    int at = done + __popc(b & ((1u << lane) - 1u));
    for (int w = 0; w < SELECT_THREADS / 32; ++w) { if (w < warp) at += scan[w]; done += scan[w]; }
    if (keep) ids[at] = p;
  }
}
