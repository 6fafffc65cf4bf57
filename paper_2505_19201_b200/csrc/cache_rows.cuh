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

template <typename T> struct CaInf;
template <> struct CaInf<bf16> { static constexpr uint32_t BITS = 0x7f80u; };
template <> struct CaInf<f16> { static constexpr uint32_t BITS = 0x7c00u; };

struct CacheAppendArgs {
  CacheView c;
  const void *q, *k_new, *v_new;
  long long q_ld, k_ld, v_ld, q_out_ld;
  void *q_out;
  const int *row_seq, *slots, *positions;
  const float2 *rope;                      // [n_pos][rot / 2], or null (rot = 0 then)
  int rows, heads, hd, n_pos, rot, interleaved;
  int chunk_rows, chunk_blocks;            // the grid: chunks of rows, the blocks of one
  int bound_blocks, bound_rows;            // the first blocks of a chunk, which look for full pages, and rows of one of them
  int head_lanes, block_rows, head_blocks; // of the others: threads of a row's unit, which take a head each at a time; rows of a block; blocks that share the heads
  int *status;
};

// A head's elements are worked on in units of 16: two vectors whose elements are rotated with one another, a[i] with b[i], or sixteen
// consecutive elements, whose neighbours are (interleaved) or which stay as they are (past rot).  First elements of unit u's two vectors:
__device__ __forceinline__ void append_unit(const CacheAppendArgs &a, int u, int &ia, int &ib) {
  const bool split = u * 16 < a.rot && !a.interleaved;
  ia = split ? u * 8 : u * 16;
  ib = split ? u * 8 + a.rot / 2 : u * 16 + 8;
}
// The rotary factors of unit u at a position.
__device__ __forceinline__ void append_factors(const CacheAppendArgs &a, int u, int pos, float (&cs)[16]) {
  const float4 *t = reinterpret_cast<const float4 *>(a.rope + (long long)pos * (a.rot / 2) + u * 8);
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<float4 *>(cs + 4 * i) = t[i];
}
// The rotation of a unit, in 32 bits, rounded once.
template <typename T>
__device__ __forceinline__ void append_rotate(bool interleaved, const float (&cs)[16], uint4 &va, uint4 &vb) {
  float x[8], y[8];
  unpack8<T>(va, x);
  unpack8<T>(vb, y);
  if (!interleaved) {
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
  va = pack8<T>(x);
  vb = pack8<T>(y);
}

__device__ __forceinline__ uint32_t min_pair(uint32_t a, uint32_t b, bf16) { __nv_bfloat162 r = __hmin2(*reinterpret_cast<__nv_bfloat162 *>(&a), *reinterpret_cast<__nv_bfloat162 *>(&b)); return *reinterpret_cast<uint32_t *>(&r); }
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b, bf16) { __nv_bfloat162 r = __hmax2(*reinterpret_cast<__nv_bfloat162 *>(&a), *reinterpret_cast<__nv_bfloat162 *>(&b)); return *reinterpret_cast<uint32_t *>(&r); }
__device__ __forceinline__ uint32_t min_pair(uint32_t a, uint32_t b, f16) { __half2 r = __hmin2(*reinterpret_cast<__half2 *>(&a), *reinterpret_cast<__half2 *>(&b)); return *reinterpret_cast<uint32_t *>(&r); }
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b, f16) { __half2 r = __hmax2(*reinterpret_cast<__half2 *>(&a), *reinterpret_cast<__half2 *>(&b)); return *reinterpret_cast<uint32_t *>(&r); }

// The bounds of one KV head of the page that row r fills, by a whole block: from the rows of this call (rotated once more: the same
// values) and, for tokens that came earlier, from the cache.
template <typename T>
__device__ __forceinline__ void append_bounds(const CacheAppendArgs &a, int r, int kvh, int *from, uint32_t (*red)[CACHE_THREADS / 32][128]) {
  const int pt = a.c.page_tokens, seq = a.row_seq[r], slot = a.slots[r], first = slot - (pt - 1), tid = threadIdx.x, units = a.hd / 16;
  const int page = a.c.page(seq, slot >> a.c.page_shift);
  __syncthreads();                           // (the row before may still be read from)
  int missing = 0;
  for (int t = tid; t < pt; t += CACHE_THREADS) {       // as a rule the rows of a sequence stand in order
    const int rr = r - (pt - 1) + t;
    const bool here = rr >= 0 && a.row_seq[rr] == seq && a.slots[rr] == first + t;
    from[t] = here ? rr : -1;                // -1: it is in the cache already
    missing |= !here;
  }
  if (__syncthreads_or(missing)) {
    for (int rr = tid; rr < a.rows; rr += CACHE_THREADS)
      if (a.row_seq[rr] == seq && a.slots[rr] >= first && a.slots[rr] <= slot) from[a.slots[rr] - first] = rr;
    __syncthreads();
  }
  const int u = tid % units, groups = CACHE_THREADS / units;
  int ia, ib;
  append_unit(a, u, ia, ib);
  uint32_t lo[8], hi[8];
  const uint32_t plus = CaInf<T>::BITS * 0x10001u;         // two infinities
#pragma unroll
  for (int i = 0; i < 8; ++i) { lo[i] = plus; hi[i] = plus | 0x80008000u; }
  const auto load = [&](int t, uint4 &va, uint4 &vb) {
    const int rr = from[t];
    const T *src = rr >= 0 ? (const T *)a.k_new + rr * a.k_ld + (long long)kvh * a.hd : (const T *)a.c.k + a.c.at(page, kvh, t);
    va = *reinterpret_cast<const uint4 *>(src + ia);
    vb = *reinterpret_cast<const uint4 *>(src + ib);
  };
  for (int t0 = tid / units; t0 < pt; t0 += 2 * groups) {
    uint4 va[2], vb[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) if (t0 + j * groups < pt) load(t0 + j * groups, va[j], vb[j]);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int t = t0 + j * groups;
      if (t >= pt) continue;
      const int rr = from[t];
      if (rr >= 0 && a.rot) {
        const int p = a.positions ? a.positions[rr] : first + t;
        if ((unsigned)p >= (unsigned)a.n_pos) continue;                // a row that is not written
        if (u * 16 < a.rot) {
          float cs[16];
          append_factors(a, u, p, cs);
          append_rotate<T>(a.interleaved, cs, va[j], vb[j]);
        }
      }
      const uint32_t w[8] = {va[j].x, va[j].y, va[j].z, va[j].w, vb[j].x, vb[j].y, vb[j].z, vb[j].w};
#pragma unroll
      for (int i = 0; i < 8; ++i) { lo[i] = min_pair(lo[i], w[i], T()); hi[i] = max_pair(hi[i], w[i], T()); }
    }
  }
  for (int o = units; o < 32; o <<= 1)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo[i] = min_pair(lo[i], __shfl_xor_sync(0xffffffffu, lo[i], o), T());
      hi[i] = max_pair(hi[i], __shfl_xor_sync(0xffffffffu, hi[i], o), T());
    }
  if ((tid & 31) < units)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int d = (i < 4 ? ia + 2 * i : ib + 2 * i - 8) / 2;
      red[0][tid >> 5][d] = lo[i];
      red[1][tid >> 5][d] = hi[i];
    }
  __syncthreads();
  uint32_t *out = reinterpret_cast<uint32_t *>((T *)a.c.bounds + ((long long)page * a.c.hkv + kvh) * 2 * a.hd);
  for (int i = tid; i < a.hd; i += CACHE_THREADS) {
    const int which = i >= a.hd / 2, d = i - which * (a.hd / 2);
    uint32_t m = red[which][0][d];
    for (int w = 1; w < CACHE_THREADS / 32; ++w) m = which ? max_pair(m, red[1][w][d], T()) : min_pair(m, red[0][w][d], T());
    out[i] = m;
  }
}

// Bound by HBM, or by latency where there are few rows.  The grid is in chunks of rows.  The first blocks of a chunk look for rows that fill a page, a few rows and one
// KV head each; the others move rows: a thread has one unit of a row and takes it from HEADS heads (queries, then keys, then values), two at a time; the row's place and
// the unit's rotary factors it looks up once.  Measured with 5871 rows of 16 + 2 x 8 heads of 256, 193 MB: 42.9 us (4.5 TB/s), 37.5 of them without bounds; with 16 heads
// a thread 46.2 (one and a quarter waves of blocks), with 4 heads 44.3 (more look-ups); with four units of any heads a thread, each with factors and divisions of its own,
// 54; with all the blocks that look for pages at the grid's start, four times the rows take 155 us in place of 145 (their rows are read from HBM twice).
#define APPEND_HEADS 8
template <typename T, int HEADS>
__global__ void __launch_bounds__(CACHE_THREADS, 4)
k_cache_append(const __grid_constant__ CacheAppendArgs a) {
  kernel_entry(TR_k_cache_append);
  const int chunk = blockIdx.x / a.chunk_blocks, at = blockIdx.x - chunk * a.chunk_blocks;
  if (at < a.bound_blocks) {
    __shared__ int from[256];
    __shared__ uint32_t red[2][CACHE_THREADS / 32][128];
    const int kvh = at % a.c.hkv, r0 = chunk * a.chunk_rows + at / a.c.hkv * a.bound_rows, lane = threadIdx.x & 31, pt = a.c.page_tokens;
    // which of the rows fill a page: the same in every warp
    const int r = r0 + lane;
    bool fills = false;
    if (lane < a.bound_rows && r < a.rows) {
      const int seq = a.row_seq[r], slot = a.slots[r], pos = a.positions ? a.positions[r] : slot;
      fills = seq >= 0 && a.c.token_ok(seq, slot) && (slot & (pt - 1)) == pt - 1 && (!a.rot || (unsigned)pos < (unsigned)a.n_pos) && a.c.page(seq, slot >> a.c.page_shift) >= 0;
    }
    for (unsigned left = __ballot_sync(0xffffffffu, fills); left; left &= left - 1) append_bounds<T>(a, r0 + __ffs(left) - 1, kvh, from, red);
    return;
  }
  const int units = a.hd / 16, block = at - a.bound_blocks, rows_at = block / a.head_blocks, part = block - rows_at * a.head_blocks;
  const int u = threadIdx.x % units, rest = threadIdx.x / units, hl = rest % a.head_lanes;
  const long long r = (long long)chunk * a.chunk_rows + rows_at * a.block_rows + rest / a.head_lanes;
  if (r >= a.rows) return;
  const int n_heads = a.heads + 2 * a.c.hkv, h0 = part * (a.head_lanes * HEADS) + hl;      // heads h0, h0 + head_lanes, ...
  int ia, ib;
  append_unit(a, u, ia, ib);
  // where a head's unit comes from
  const auto load = [&](int hh, uint4 &va, uint4 &vb) {
    const bool is_v = hh >= a.heads + a.c.hkv;
    const T *src = hh < a.heads ? (const T *)a.q + r * a.q_ld + (long long)hh * a.hd
                   : !is_v ? (const T *)a.k_new + r * a.k_ld + (long long)(hh - a.heads) * a.hd
                           : (const T *)a.v_new + r * a.v_ld + (long long)(hh - a.heads - a.c.hkv) * a.hd;
    va = *reinterpret_cast<const uint4 *>(src + (is_v ? u * 16 : ia));                    // (values are not rotated: sixteen elements as they stand)
    vb = *reinterpret_cast<const uint4 *>(src + (is_v ? u * 16 + 8 : ib));
  };
  constexpr int AT_ONCE = HEADS > 1 ? 2 : 1;
  uint4 va[AT_ONCE], vb[AT_ONCE];
#pragma unroll
  for (int j = 0; j < AT_ONCE; ++j) if (h0 + j * a.head_lanes < n_heads) load(h0 + j * a.head_lanes, va[j], vb[j]);
  const int seq = a.row_seq[r], slot = a.slots[r], pos = a.positions ? a.positions[r] : slot;
  if (seq < 0) return;
  if (!a.c.token_ok(seq, slot) || (a.rot && (unsigned)pos >= (unsigned)a.n_pos)) {
    if (u == 0) cache_bad_index(a.status);
    return;
  }
  const int page = a.c.page(seq, slot >> a.c.page_shift);
  const bool turn = u * 16 < a.rot;
  float cs[16];
  if (turn) append_factors(a, u, pos, cs);
  if (page < 0 && u == 0 && hl == 0) cache_bad_index(a.status);
#pragma unroll 1
  for (int j0 = 0; j0 < HEADS; j0 += AT_ONCE) {
    if (j0 > 0)
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) if (h0 + (j0 + j) * a.head_lanes < n_heads) load(h0 + (j0 + j) * a.head_lanes, va[j], vb[j]);
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int hh = h0 + (j0 + j) * a.head_lanes;
      if (hh >= n_heads || (hh >= a.heads && page < 0)) continue;
      const bool is_v = hh >= a.heads + a.c.hkv;
      T *dst = hh < a.heads ? (T *)a.q_out + r * a.q_out_ld + (long long)hh * a.hd
                            : (T *)(is_v ? a.c.v : a.c.k) + a.c.at(page, hh - a.heads - (is_v ? a.c.hkv : 0), slot & (a.c.page_tokens - 1));
      if (turn && !is_v) append_rotate<T>(a.interleaved, cs, va[j], vb[j]);
      *reinterpret_cast<uint4 *>(dst + (is_v ? u * 16 : ia)) = va[j];
      *reinterpret_cast<uint4 *>(dst + (is_v ? u * 16 + 8 : ib)) = vb[j];
    }
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
  int group, budget, keep_first, keep_last;
  float *scores;                           // [row][KV head][pages_per_seq], as k_cache_scores has them ...
  float *off;                              // [row][KV head][score_blocks]: ... each right to so much, by the block that made it
  int score_blocks;
  int *ids;
  int *status;
};

__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return v == v ? u ^ (u & 0x80000000u ? 0xffffffffu : 0x80000000u) : 0u;
}
__device__ __forceinline__ float order_value(uint32_t k) { return __uint_as_float(k ^ (k & 0x80000000u ? 0x80000000u : 0xffffffffu)); }
// Pages up to the row's own; 0 for a row without any.
__device__ __forceinline__ int select_pages(const CacheSelectArgs &a, int seq, int pos) {
  return seq >= 0 && pos >= 0 && a.c.token_ok(seq, pos) ? (pos >> a.c.page_shift) + 1 : 0;
}
// Scores in 32 bits, with a bound on how far they are off.  (Which pages are kept is a matter of the scores in 64 bits, but only for the few near the cut, which
// k_cache_select looks at again; in 64 bits for all, a score took four times the instructions, and 64 rows of 1024 pages 20 us.)  HD / 8 lanes take a page, eight
// channels each; a warp has SCORE_DEEP pages per lane under way at a time, and GC heads of the group: a lane has SCORE_DEEP * GC partial sums,
// which are added up across the lanes by halves, each step with half as many of them, and then compared.
// The bound: a sum is eight fused steps in a lane and up to five additions across lanes, each wrong by 2^-24 of a partial sum, which is no larger than
// sum |q_d| times the largest bound there is; one more such error for the rounding of the exact score, and three for the bound's own.
#define SCORE_DEEP 4
template <typename T> __device__ __forceinline__ float2 widen2(uint32_t w);
template <> __device__ __forceinline__ float2 widen2<bf16>(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
template <> __device__ __forceinline__ float2 widen2<f16>(uint32_t w) { return __half22float2(*reinterpret_cast<__half2 *>(&w)); }

template <typename T, int HD, int GC>
__global__ void __launch_bounds__(CACHE_THREADS, 3)
k_cache_scores(const __grid_constant__ CacheSelectArgs a) {
  constexpr int LANES = HD / 8, PAGES = 32 / LANES, NV = SCORE_DEEP * GC, BLOCK = CACHE_THREADS / 32 * PAGES * SCORE_DEEP;
  constexpr int LEFT = NV > LANES ? NV / LANES : 1, STEPS = NV > LANES ? LANES : NV;
  __shared__ float4 q_s[GC][2][LANES];                      // a lane's eight channels of a head
  __shared__ uint4 m_s[GC][LANES];                          // and where they are negative: a mask for each pair
  __shared__ uint32_t top_s[CACHE_THREADS / 32];
  __shared__ float q1_s;
  kernel_entry(TR_k_cache_scores);
  const int r = blockIdx.x / a.c.hkv, kvh = blockIdx.x % a.c.hkv, seq = a.row_seq[r], pos = a.row_pos[r], n = select_pages(a, seq, pos);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % LANES, end = n - a.keep_last;
  if (n <= a.budget) return;                               // all are kept
  const T *q0 = (const T *)a.q + r * a.q_ld + (long long)kvh * a.group * HD;
  float *scores = a.scores + (long long)blockIdx.x * a.c.pages_per_seq;
  uint32_t top = 0u;                                       // the largest magnitudes met, a pair
  int page[SCORE_DEEP];                                    // of the pages ahead; -1: not asked for, -2: no number
  const auto look_up = [&](int base) {
#pragma unroll
    for (int j = 0; j < SCORE_DEEP; ++j) {
      const int p = base + warp * PAGES * SCORE_DEEP + lane / LANES + j * PAGES;         // pages p0, p0 + PAGES, ...
      page[j] = -1;
      if (p >= a.keep_first && p < end) {
        page[j] = a.c.page(seq, p);
        if (page[j] < 0) { page[j] = -2; cache_bad_index(a.status); }
      }
    }
  };
  look_up(blockIdx.y * BLOCK);
  if (threadIdx.x == 0) q1_s = 0.f;
  for (int base = blockIdx.y * BLOCK; base < end; base += gridDim.y * BLOCK) {
    const int p0 = base + warp * PAGES * SCORE_DEEP + lane / LANES;
    uint4 lo[SCORE_DEEP], hi[SCORE_DEEP];
    unsigned bad = 0, on = 0;                              // pages without a number, pages of this row: bit j
#pragma unroll
    for (int j = 0; j < SCORE_DEEP; ++j) {
      lo[j] = hi[j] = make_uint4(0u, 0u, 0u, 0u);
      if (page[j] >= 0) {
        const uint4 *b = reinterpret_cast<const uint4 *>((const T *)a.c.bounds + ((long long)page[j] * a.c.hkv + kvh) * 2 * HD) + l;
        lo[j] = b[0];
        hi[j] = b[LANES];
      }
      on |= (page[j] != -1) << j;
      bad |= (page[j] == -2) << j;
    }
    look_up(base + gridDim.y * BLOCK);
    if (base == (int)blockIdx.y * BLOCK) {                 // the largest sum |q_d| of the group's heads
      __syncthreads();
      for (int g = warp; g < a.group; g += CACHE_THREADS / 32) {
        float sum = 0.f;
        for (int d = lane; d < HD; d += 32) sum += fabsf(to_f(q0[g * HD + d]));
        sum = warp_sum(sum);
        if (lane == 0) atomicMax(reinterpret_cast<int *>(&q1_s), __float_as_int(sum));      // (floats above zero are ordered as integers are; NaN is above all)
      }
    }
    float best[LEFT];
#pragma unroll
    for (int j = 0; j < LEFT; ++j) best[j] = -INFINITY;
    for (int g0 = 0; g0 < a.group; g0 += GC) {
      if (base == (int)blockIdx.y * BLOCK || a.group > GC) {                             // (heads that fit stay where they are)
        __syncthreads();
        for (int i = threadIdx.x; i < GC * LANES; i += CACHE_THREADS) {
          const int g = i / LANES, c = i % LANES;
          const uint4 w = g0 + g < a.group ? *reinterpret_cast<const uint4 *>(q0 + (g0 + g) * HD + c * 8) : make_uint4(0u, 0u, 0u, 0u);
          const float2 x = widen2<T>(w.x), y = widen2<T>(w.y), z = widen2<T>(w.z), u = widen2<T>(w.w);
          q_s[g][0][c] = make_float4(x.x, x.y, y.x, y.y);
          q_s[g][1][c] = make_float4(z.x, z.y, u.x, u.y);
          const auto mask = [](uint32_t v) { return (v & 0x8000u ? 0xffffu : 0u) | (v & 0x80000000u ? 0xffff0000u : 0u); };
          m_s[g][c] = make_uint4(mask(w.x), mask(w.y), mask(w.z), mask(w.w));
        }
        __syncthreads();
      }
      float v[NV];                                         // v[g * SCORE_DEEP + j]
#pragma unroll
      for (int g = 0; g < GC; ++g) {
        const float4 qa = q_s[g][0][l], qb = q_s[g][1][l];
        const uint4 m = m_s[g][l];
#pragma unroll
        for (int j = 0; j < SCORE_DEEP; ++j) {
          // the lower bound where q is negative, else the upper one
          const float2 x = widen2<T>((lo[j].x & m.x) | (hi[j].x & ~m.x)), y = widen2<T>((lo[j].y & m.y) | (hi[j].y & ~m.y));
          const float2 z = widen2<T>((lo[j].z & m.z) | (hi[j].z & ~m.z)), u = widen2<T>((lo[j].w & m.w) | (hi[j].w & ~m.w));
          float t = qa.x * x.x;
          t = fmaf(qa.y, x.y, t); t = fmaf(qa.z, y.x, t); t = fmaf(qa.w, y.y, t);
          t = fmaf(qb.x, z.x, t); t = fmaf(qb.y, z.y, t); t = fmaf(qb.z, u.x, t);
          v[g * SCORE_DEEP + j] = fmaf(qb.w, u.y, t);
        }
      }
      // across the lanes of a page: at each step a lane gives away one half of its sums and adds to the other
      int width = NV;
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) {
        if (width > 1) {
          width /= 2;
          const bool up = (lane & o) != 0;
#pragma unroll
          for (int j = 0; j < NV / 2; ++j)
            if (j < width) {
              const float give = up ? v[j] : v[j + width], keep = up ? v[j + width] : v[j];
              v[j] = keep + __shfl_xor_sync(0xffffffffu, give, o);
            }
        } else v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
      }
      // A lane is left with the sums own * LEFT + (0 .. LEFT - 1), the bits of own being the lane's highest.  The largest of the group's heads: those past
      // the group have no say, nor has NaN.
      const int own = l / (LANES / STEPS);
#pragma unroll
      for (int j = 0; j < LEFT; ++j) {
        float f = g0 + (own * LEFT + j) / SCORE_DEEP < a.group ? v[j] : -INFINITY;
#pragma unroll
        for (int o = LANES / 2; o >= LANES / STEPS * (SCORE_DEEP / LEFT); o >>= 1) f = fmaxf(f, __shfl_xor_sync(0xffffffffu, f, o));
        best[j] = fmaxf(best[j], f);
      }
    }
#pragma unroll
    for (int j = 0; j < SCORE_DEEP; ++j) {
      const uint32_t w[8] = {lo[j].x, lo[j].y, lo[j].z, lo[j].w, hi[j].x, hi[j].y, hi[j].z, hi[j].w};
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max_pair(top, w[i] & 0x7fff7fffu, T());
    }
    const int own = l / (LANES / STEPS);
#pragma unroll
    for (int j = 0; j < LEFT; ++j) {
      const int i = own * LEFT + j, p = p0 + i % SCORE_DEEP * PAGES;
      if (i < SCORE_DEEP && l % (LANES / STEPS) == 0 && on >> i & 1u) scores[p] = bad >> i & 1u ? __int_as_float(0x7fffffff) : best[j];
    }
  }
  for (int o = 16; o > 0; o >>= 1) top = max_pair(top, __shfl_xor_sync(0xffffffffu, top, o), T());
  if (lane == 0) top_s[warp] = top;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < CACHE_THREADS / 32; ++w) top = max_pair(top, top_s[w], T());
    const float2 t = widen2<T>(top);
    // (and what products below the smallest normal number lose)
    a.off[(long long)blockIdx.x * a.score_blocks + blockIdx.y] = 18.f * 0x1p-24f * q1_s * fmaxf(t.x, t.y) + 0x1p-140f;
  }
}

// A page's score by the whole warp, from 64 bits: products are exact (8 and 8, or 11 and 11, digits), and so is nearly every sum of them.
template <typename T, int HD>
__device__ __forceinline__ float exact_score(const CacheSelectArgs &a, const T *q0, int page, int kvh, int lane) {
  const T *lo = (const T *)a.c.bounds + ((long long)page * a.c.hkv + kvh) * 2 * HD, *hi = lo + HD;
  float best = -INFINITY;
  for (int g = 0; g < a.group; ++g) {
    double s = 0.0;
    for (int d = lane; d < HD; d += 32) {
      const float x = to_f(q0[g * HD + d]);
      s += (double)x * (double)to_f(x < 0.f ? lo[d] : hi[d]);
    }
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    best = fmaxf(best, (float)s);
  }
  return best;
}

// grid (rows * KV heads), the scores in shared memory as 32-bit keys of the same order (0: a page without a number).  The cut, the left-th largest: bins over the range of
// the keys, of equal width, so that they are filled evenly whatever the scores are; the bin in which the cut falls is looked into again until it holds few keys,
// which are compared with each other.  Scores are off by up to E, and so is the cut: what lies above the cut by more than 2 E is kept, what lies below it by more is not, and where what lies
// between (as a rule the cut's own page and nothing else) is not taken as a whole, it gets its exact scores and the cut is looked for again.  Then the kept pages in order: a
// thread has a run of pages.
#define SELECT_THREADS 512
#define SELECT_BINS 1024
#define SELECT_FEW 64
struct SelectShared {
  int hist[SELECT_BINS], scan[SELECT_THREADS / 32], n_few, bin, above, count, ties;
  uint32_t few[SELECT_FEW], lows[SELECT_THREADS / 32], highs[SELECT_THREADS / 32], key;
};
// The left-th largest (1 .. m) of keys[0 .. m - 1] in sh.key, and in sh.ties how many equal to it are among the left largest.
// low, high: the lowest and the highest key of this thread's share.
__device__ __forceinline__ void select_cut(SelectShared &sh, const uint32_t *keys, int m, int left, uint32_t low, uint32_t high) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  low = __reduce_min_sync(0xffffffffu, low);
  high = __reduce_max_sync(0xffffffffu, high);
  if (lane == 0) { sh.lows[warp] = low; sh.highs[warp] = high; }
  for (int i = tid; i < SELECT_BINS; i += SELECT_THREADS) sh.hist[i] = 0;
  if (tid == 0) sh.n_few = 0;
  __syncthreads();
  low = __reduce_min_sync(0xffffffffu, sh.lows[lane % (SELECT_THREADS / 32)]);
  high = __reduce_max_sync(0xffffffffu, sh.highs[lane % (SELECT_THREADS / 32)]);
  for (bool first = true;; first = false) {                     // keys low .. high hold the cut, the left-th largest of them
    int shift = 0;
    while ((high - low) >> shift >= SELECT_BINS) ++shift;
    if (!first) {
      for (int i = tid; i < SELECT_BINS; i += SELECT_THREADS) sh.hist[i] = 0;
      __syncthreads();
    }
    for (int i = tid; i < m; i += SELECT_THREADS)
      if (keys[i] >= low && keys[i] <= high) atomicAdd(sh.hist + ((keys[i] - low) >> shift), 1);
    __syncthreads();
    // from the top: bins PER t .. PER t + PER - 1 with t = SELECT_THREADS - 1 - tid
    constexpr int PER = SELECT_BINS / SELECT_THREADS;
    int own = 0, sum;
#pragma unroll
    for (int k = 0; k < PER; ++k) own += sh.hist[(SELECT_THREADS - 1 - tid) * PER + k];
    sum = own;
    for (int o = 1; o < 32; o <<= 1) { const int t = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += t; }
    if (lane == 31) sh.scan[warp] = sum;
    __syncthreads();
    for (int w = 0; w < warp; ++w) sum += sh.scan[w];
    if (sum >= left && sum - own < left) {
      int above = sum - own, b = (SELECT_THREADS - tid) * PER - 1;
      while (above + sh.hist[b] < left) above += sh.hist[b--];
      sh.bin = b; sh.above = above; sh.count = sh.hist[b];
    }
    __syncthreads();
    left -= sh.above;
    low += (uint32_t)sh.bin << shift;
    high = min(high, low + (1u << shift) - 1u);
    const int count = sh.count;
    if (shift == 0) {                                           // a bin is a key
      if (tid == 0) { sh.key = low; sh.ties = left; }
      break;
    }
    if (count <= SELECT_FEW) {
      for (int i = tid; i < m; i += SELECT_THREADS)
        if (keys[i] >= low && keys[i] <= high) sh.few[atomicAdd(&sh.n_few, 1)] = keys[i];
      __syncthreads();
      if (tid < count) {
        const uint32_t k = sh.few[tid];
        int above = 0, same = 0;
        for (int i = 0; i < count; ++i) { above += sh.few[i] > k; same += sh.few[i] == k; }
        if (above < left && above + same >= left) { sh.key = k; sh.ties = left - above; }              // (equal keys write the same)
      }
      break;
    }
    __syncthreads();
  }
  __syncthreads();
}

template <typename T, int HD>
__global__ void __launch_bounds__(SELECT_THREADS)
k_cache_select(const __grid_constant__ CacheSelectArgs a) {
  extern __shared__ uint32_t sel_keys[];
  __shared__ SelectShared sh;
  __shared__ int n_in, n_border, border[SELECT_FEW], taken[SELECT_FEW];
  __shared__ float offs[SELECT_THREADS / 32];
  kernel_entry(TR_k_cache_select);
  const int r = blockIdx.x / a.c.hkv, kvh = blockIdx.x % a.c.hkv, seq = a.row_seq[r], pos = a.row_pos[r], n = select_pages(a, seq, pos);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int *ids = a.ids + (long long)blockIdx.x * a.budget;
  if (seq >= 0 && pos >= 0 && !n && tid == 0) cache_bad_index(a.status);
  if (n <= a.budget) {
    for (int i = tid; i < a.budget; i += SELECT_THREADS) ids[i] = i < n ? i : -1;
    return;
  }
  const float *scores = a.scores + (long long)blockIdx.x * a.c.pages_per_seq;
  const int p0 = a.keep_first, m = n - a.keep_last - p0;        // candidates p0 .. p0 + m - 1
  const int left = a.budget - a.keep_first - a.keep_last;       // of which so many are taken: fewer than there are
  uint32_t cut = 0u;                                            // what is above it is kept, and of what is equal to it the first so many
  int ties = 0;
  if (tid == 0) n_in = n_border = 0;
  if (left) {
    float off = 0.f;
    uint32_t low = 0xffffffffu, high = 0u;
    for (int i = tid; i < a.score_blocks; i += SELECT_THREADS) {
      const float f = a.off[(long long)blockIdx.x * a.score_blocks + i];
      off = f > off || f != f ? (f != f ? INFINITY : f) : off;
    }
    for (int i = tid; i < m; i += SELECT_THREADS) {
      const uint32_t b = __float_as_uint(scores[p0 + i]);
      const uint32_t k = b == 0x7fffffffu ? 0u : order_key(__uint_as_float(b));
      sel_keys[i] = k;
      low = min(low, k); high = max(high, k);
    }
    off = warp_max(off);
    if (lane == 0) offs[warp] = off;
    select_cut(sh, sel_keys, m, left, low, high);
    cut = sh.key;
    ties = sh.ties;
  }
  if (left && cut) {                                            // (0: pages without a number are needed to fill the budget)
    // ---- what is near the cut
    const float at = order_value(cut), e2 = 2.f * warp_max(offs[lane % (SELECT_THREADS / 32)]);
    const auto side = [&](uint32_t k) {                         // 1: above the border, -1: below, 0: on it
      const float s = order_value(k);
      return k == 0u ? -1 : s - at > e2 ? 1 : at - s > e2 ? -1 : 0;
    };
    int in = 0;
    for (int i = tid; i < m; i += SELECT_THREADS) {
      const int d = side(sel_keys[i]);
      in += d > 0;
      if (d == 0) { const int j = atomicAdd(&n_border, 1); if (j < SELECT_FEW) border[j] = i; }
    }
    in = __reduce_add_sync(0xffffffffu, in);
    if (lane == 0 && in) atomicAdd(&n_in, in);
    __syncthreads();
    const int nb = n_border, take = left - n_in;                // 1 .. nb of those on the border are taken
    const bool few = nb <= SELECT_FEW, open = nb > take;
    if (open && few) {
      const T *q0 = (const T *)a.q + r * a.q_ld + (long long)kvh * a.group * HD;
      for (int j = warp; j < nb; j += SELECT_THREADS / 32) {
        const float s = exact_score<T, HD>(a, q0, a.c.page(seq, p0 + border[j]), kvh, lane);
        if (lane == 0) sh.few[j] = order_key(s);
      }
      __syncthreads();
      if (tid < nb) {
        int before = 0;
        for (int i = 0; i < nb; ++i) before += sh.few[i] > sh.few[tid] || (sh.few[i] == sh.few[tid] && border[i] < border[tid]);
        taken[tid] = before < take;
      }
      __syncthreads();
    }
    if (open) {
      // Pages above become the highest key and those below 0; those on the border either, or their exact score, for which the cut is looked for again.  (Where they are
      // all taken, what is kept is what the cut says already.)
      uint32_t low = 0xffffffffu, high = 0u;
      if (few) {
        for (int i = tid; i < m; i += SELECT_THREADS) sel_keys[i] = side(sel_keys[i]) > 0 ? 0xffffffffu : 0u;
        __syncthreads();
        if (tid < nb && taken[tid]) sel_keys[border[tid]] = 0xffffffffu;
        cut = 0xfffffffeu;
        ties = 0;
      } else {
        const T *q0 = (const T *)a.q + r * a.q_ld + (long long)kvh * a.group * HD;
        for (int i = warp; i < m; i += SELECT_THREADS / 32) {
          const int d = side(sel_keys[i]);
          const uint32_t k = d > 0 ? 0xffffffffu : d < 0 ? 0u : order_key(exact_score<T, HD>(a, q0, a.c.page(seq, p0 + i), kvh, lane));
          __syncwarp();
          if (lane == 0) sel_keys[i] = k;
          low = min(low, k); high = max(high, k);
        }
        __syncthreads();
        select_cut(sh, sel_keys, m, left, low, high);
        cut = sh.key;
        ties = sh.ties;
      }
      __syncthreads();
    }
  }
  // pages i0 .. i1 - 1 are this thread's
  const int run = (m + SELECT_THREADS - 1) / SELECT_THREADS, i0 = min(m, tid * run), i1 = left ? min(m, i0 + run) : i0;
  int above = 0, same = 0;
  for (int i = i0; i < i1; ++i) { above += sel_keys[i] > cut; same += sel_keys[i] == cut; }
  const int both = above | same << 16;                          // (no more than 32768 of each)
  int sum = both;
  for (int o = 1; o < 32; o <<= 1) { const int t = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += t; }
  if (lane == 31) sh.scan[warp] = sum;
  __syncthreads();
  sum -= both;
  for (int w = 0; w < warp; ++w) sum += sh.scan[w];
  int tie = sum >> 16 & 0xffff, at = a.keep_first + (sum & 0xffff) + min(tie, ties);
  for (int i = i0; i < i1; ++i) {
    const uint32_t k = sel_keys[i];
    if (k > cut || (k == cut && tie < ties)) ids[at++] = p0 + i;
    tie += k == cut;
  }
  for (int i = tid; i < a.keep_first; i += SELECT_THREADS) ids[i] = i;
  for (int i = tid; i < a.keep_last; i += SELECT_THREADS) ids[a.budget - a.keep_last + i] = n - a.keep_last + i;
}
