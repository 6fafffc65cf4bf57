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

// A pair in 32 bits.
__device__ __forceinline__ float2 unpack2(uint32_t w, bf16) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ float2 unpack2(uint32_t w, f16) { return __half22float2(*reinterpret_cast<__half2 *>(&w)); }

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

// Whether a row has a position that there are factors for (it is not written otherwise).
__device__ __forceinline__ bool append_position_ok(const CacheAppendArgs &a, int r, int slot) { return !a.rot || (unsigned)(a.positions ? a.positions[r] : slot) < (unsigned)a.n_pos; }
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
    const bool here = rr >= 0 && a.row_seq[rr] == seq && a.slots[rr] == first + t && append_position_ok(a, rr, first + t);
    from[t] = here ? rr : -1;                // -1: it is in the cache already
    missing |= !here;
  }
  if (__syncthreads_or(missing)) {
    // By the page, which another sequence may name too.  Four look-ups of a thread under way together: 16900 rows of 20 sequences, each of which begins inside a page, take 154 us (one by
    // one 178; by the sequence alone, which is not enough, 145).
    constexpr int AT_ONCE = 4;
    for (int r0 = tid; r0 < a.rows; r0 += AT_ONCE * CACHE_THREADS) {
      int other[AT_ONCE], at[AT_ONCE];
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        const int rr = r0 + j * CACHE_THREADS;
        other[j] = rr < a.rows ? a.row_seq[rr] : -1;
        at[j] = rr < a.rows ? a.slots[rr] : 0;
      }
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) other[j] = other[j] >= 0 && a.c.token_ok(other[j], at[j]) && from[at[j] & (pt - 1)] < 0 && append_position_ok(a, r0 + j * CACHE_THREADS, at[j])
                                                          ? a.c.page(other[j], at[j] >> a.c.page_shift) : -1;
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) if (other[j] == page) from[at[j] & (pt - 1)] = r0 + j * CACHE_THREADS;
    }
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
      if (rr >= 0 && u * 16 < a.rot) {
        float cs[16];
        append_factors(a, u, a.positions ? a.positions[rr] : a.slots[rr], cs);
        append_rotate<T>(a.interleaved, cs, va[j], vb[j]);
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
// the unit's rotary factors it looks up once.  Four blocks to an SM, which takes 12 to 36 bytes of a thread's registers to memory and back; with three, and none, 44.0 us for the 42.4
// below, 163 for the 154 above.  Measured with 5871 rows of 16 + 2 x 8 heads of 256, 193 MB: 42.4 us (4.5 TB/s), 37.1 without bounds; with 16 heads
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

// D = A B + 0, 16 x 8 over 16: a lane has of A the pairs 2 j, 2 j + 1 (a[0], a[1]) and 2 j + 8, 2 j + 9 (a[2], a[3]) of rows i and i + 8, of B those of column i, of D
// columns 2 j and 2 j + 1 of both rows (lane = 4 i + j).
__device__ __forceinline__ void score_mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, bf16) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void score_mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, f16) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

// Scores in 32 bits, with a bound on how far they are off.  (Which pages are kept is a matter of the scores in 64 bits, but only for the few near the cut, which
// k_cache_select looks at again.)  sum_d max(q_d lo_d, q_d hi_d) is a product of the bounds with q's positive part and its negative one, [hi | lo] [q+ ; q-]: a
// warp takes 16 pages against up to eight heads of the group (more in another pass) with the warp's own matrix instruction; eight columns are too few for the others, and what
// bounds this is the bounds' way from memory.  A row of A is a page, and its channels come in any order, the same in q, so that a lane reads 16 bytes at a time.
// Selection as a whole, with 64 pages kept, before (a lane had eight channels of a page, multiplied, added one by one and across lanes: six times the instructions) and now: 8 rows
// against 1024 pages, 32 heads over 8 of 128, 23.9 and 17.9 us; 64 rows 93 and 68; one row against 2048 pages 15.2 and 10.6; 9 rows against 1876 pages of 16 tokens, 16 over 8 of 256, 35 and 28.
// (Two or four runs of 32 channels under way in a lane take registers from blocks: 64 rows 91 us and 69, 8 rows 19.0 and 21.6.)
// A sum that is no finite number, as infinite bounds make it or a part of it past the largest number of 32 bits, is formed again from 64 bits.
// The bound.  Each of HD / 8 instructions adds 16 exact products to zero; of each product it may lose 2^-23 of the largest, and of its result, no larger than 16 of these, as much:
// 32 x 2^-23 = 2^-18 of the largest product there may be, max |q_d| times the largest bound there is (met in 2.5 million sums: 2^-21).  The sums are added in 32 bits, each time wrong by
// 2^-24 of a partial sum, which is no larger than sum |q_d| times the largest bound; one more such error for the rounding of the exact score, and four for the bound's own.
#define SCORE_PAGES (CACHE_THREADS / 32 * 16)              // pages that a block has under way
// Blocks to an SM: few registers a thread, 12 to 20 bytes of which go to memory and back, and many blocks (three, and none: 64 rows 82.7 us for 67.7, 8 rows 19.6 for 18.0, 9 rows of
// small pages 32.4 for 28.4).
#define SCORE_BLOCKS 4
template <typename T, int HD>
__global__ void __launch_bounds__(CACHE_THREADS, SCORE_BLOCKS)
k_cache_scores(const __grid_constant__ CacheSelectArgs a) {
  constexpr int CHUNKS = HD / 32;                           // 32 channels: a lane's 16 bytes, four lanes to a page
  __shared__ uint4 q_s[2][CHUNKS][32];                      // positive and negative parts, as the lanes take them
  __shared__ uint32_t top_s[CACHE_THREADS / 32];
  __shared__ float q1_s, q_top_s;
  unsigned long long *tr = trace_open();
  pdl_wait();
  trace_stamp(tr, TR_k_cache_scores);
  const int r = blockIdx.x / a.c.hkv, kvh = blockIdx.x % a.c.hkv, seq = a.row_seq[r], pos = a.row_pos[r], n = select_pages(a, seq, pos);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, end = n - a.keep_last;
  if (n <= a.budget) return;                               // all are kept
  const T *q0 = (const T *)a.q + r * a.q_ld + (long long)kvh * a.group * HD;
  float *scores = a.scores + (long long)blockIdx.x * a.c.pages_per_seq;
  const uint32_t inf = CaInf<T>::BITS * 0x10001u;
  uint32_t high = inf | 0x80008000u, low = inf;            // the largest upper and the smallest lower bound met, a pair
  const int step = gridDim.y * SCORE_PAGES;
  int page;                                                // of the pages ahead, a lane and its neighbour 16 further on have one; -1: not asked for, -2: no number
  const auto look_up = [&](int base) {
    const int p = base + warp * 16 + (lane & 15);
    page = -1;
    if (p >= a.keep_first && p < end) {
      page = a.c.page(seq, p);
      if (page < 0) { page = -2; cache_bad_index(a.status); }
    }
  };
  if (threadIdx.x == 0) q1_s = q_top_s = 0.f;
  for (int g0 = 0; g0 < a.group; g0 += 8) {
    look_up(blockIdx.y * SCORE_PAGES);
    __syncthreads();
    for (int i = threadIdx.x; i < CHUNKS * 32; i += CACHE_THREADS) {
      const int g = g0 + (i & 31) / 4;
      const uint4 w = g < a.group ? *reinterpret_cast<const uint4 *>(q0 + g * HD + (i >> 5) * 32 + (i & 3) * 8) : make_uint4(0u, 0u, 0u, 0u);
      const auto mask = [](uint32_t v) { return (v & 0x8000u ? 0xffffu : 0u) | (v & 0x80000000u ? 0xffff0000u : 0u); };
      const uint4 m = make_uint4(mask(w.x), mask(w.y), mask(w.z), mask(w.w));
      q_s[0][i >> 5][i & 31] = make_uint4(w.x & ~m.x, w.y & ~m.y, w.z & ~m.z, w.w & ~m.w);
      q_s[1][i >> 5][i & 31] = make_uint4(w.x & m.x, w.y & m.y, w.z & m.z, w.w & m.w);
    }
    for (int g = g0 + warp; g < min(g0 + 8, a.group); g += CACHE_THREADS / 32) {
      float sum = 0.f, most = 0.f;                         // sum |q_d| and max |q_d|
      for (int d = lane; d < HD; d += 32) {
        const float x = fabsf(to_f(q0[g * HD + d]));
        sum += x;
        most = fmaxf(most, x);
      }
      sum = warp_sum(sum);
      most = warp_max(most);
      // (floats above zero are ordered as integers are; NaN is above all)
      if (lane == 0) { atomicMax(reinterpret_cast<int *>(&q1_s), __float_as_int(sum)); atomicMax(reinterpret_cast<int *>(&q_top_s), __float_as_int(most)); }
    }
    __syncthreads();
    for (int base = blockIdx.y * SCORE_PAGES; base < end; base += step) {
      const int now = page, p0 = base + warp * 16;
      look_up(base + step);
      const int pa = __shfl_sync(0xffffffffu, now, lane / 4), pb = __shfl_sync(0xffffffffu, now, lane / 4 + 8);
      const uint4 *lo_a = reinterpret_cast<const uint4 *>((const T *)a.c.bounds + ((long long)max(pa, 0) * a.c.hkv + kvh) * 2 * HD) + (lane & 3);
      const uint4 *lo_b = reinterpret_cast<const uint4 *>((const T *)a.c.bounds + ((long long)max(pb, 0) * a.c.hkv + kvh) * 2 * HD) + (lane & 3);
      float v[4] = {};
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        uint4 x[4];                                         // upper and lower bounds of both pages
        x[0] = x[1] = x[2] = x[3] = make_uint4(0u, 0u, 0u, 0u);
        if (pa >= 0) { x[0] = lo_a[HD / 8 + c * 4]; x[2] = lo_a[c * 4]; }
        if (pb >= 0) { x[1] = lo_b[HD / 8 + c * 4]; x[3] = lo_b[c * 4]; }
#pragma unroll
        for (int s = 0; s < 2; ++s) {                       // the positive part with the upper bounds, the negative one with the lower
          const uint4 b = q_s[s][c][lane], &ya = x[2 * s], &yb = x[2 * s + 1];
          float d[4], e[4];
          score_mma(d, ya.x, yb.x, ya.y, yb.y, b.x, b.y, T());
          score_mma(e, ya.z, yb.z, ya.w, yb.w, b.z, b.w, T());
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = (v[i] + d[i]) + e[i];
          if (g0 == 0) {
            const uint32_t w[8] = {ya.x, ya.y, ya.z, ya.w, yb.x, yb.y, yb.z, yb.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              if (s == 0) high = max_pair(high, w[i], T());
              else low = min_pair(low, w[i], T());
            }
          }
        }
      }
      // the largest of the group's heads, across the four lanes of a page
      float best[2];
      bool odd[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int g = g0 + 2 * (lane & 3);
        const float s0 = g < a.group ? v[2 * k] : -INFINITY, s1 = g + 1 < a.group ? v[2 * k + 1] : -INFINITY;
        odd[k] = (g < a.group && !(fabsf(s0) < INFINITY)) || (g + 1 < a.group && !(fabsf(s1) < INFINITY));
        float f = fmaxf(s0, s1);
        f = fmaxf(f, __shfl_xor_sync(0xffffffffu, f, 1));
        best[k] = fmaxf(f, __shfl_xor_sync(0xffffffffu, f, 2));
      }
      const unsigned odd_a = __ballot_sync(0xffffffffu, odd[0] && pa >= 0), odd_b = __ballot_sync(0xffffffffu, odd[1] && pb >= 0);
      if (odd_a | odd_b)
        for (int i = 0; i < 16; ++i)
          if ((i < 8 ? odd_a >> 4 * i : odd_b >> 4 * (i - 8)) & 15u) {
            const float s = exact_score<T, HD>(a, q0, __shfl_sync(0xffffffffu, now, i), kvh, lane);
            if (lane / 4 == i % 8) best[i / 8] = s;
          }
      if ((lane & 3) == 0) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int pg = k ? pb : pa, p = p0 + lane / 4 + 8 * k;
          if (pg != -1) scores[p] = pg == -2 ? __int_as_float(0x7fffffff) : g0 ? fmaxf(scores[p], best[k]) : best[k];
        }
      }
    }
  }
  for (int o = 16; o > 0; o >>= 1) {
    high = max_pair(high, __shfl_xor_sync(0xffffffffu, high, o), T());
    low = min_pair(low, __shfl_xor_sync(0xffffffffu, low, o), T());
  }
  if (lane == 0) top_s[warp] = max_pair(max_pair(high, low ^ 0x80008000u, T()), 0u, T());
  __syncthreads();
  pdl_trigger();                             // (at the start, the blocks of k_cache_select would crowd the SMs that have room then: 8 rows 21 us for 18)
  if (threadIdx.x == 0) {
    uint32_t top = top_s[0];
    for (int w = 1; w < CACHE_THREADS / 32; ++w) top = max_pair(top, top_s[w], T());
    const float2 t = unpack2(top, T());
    // (and what products below the smallest normal number lose)
    a.off[(long long)blockIdx.x * a.score_blocks + blockIdx.y] = ((HD / 8) * 0x1p-18f * q_top_s + (HD / 8 + 5) * 0x1p-24f * q1_s) * fmaxf(t.x, t.y) + 0x1p-116f;
  }
}

// grid (rows * KV heads), the scores in shared memory as 32-bit keys of the same order (0: a page without a number).  The cut, the left-th largest: bins over the range of
// the keys, of equal width, so that they are filled evenly whatever the scores are; the bin in which the cut falls is looked into again until it holds few keys,
// which are compared with each other.  Scores are off by up to E, and so is the cut: what lies above the cut by more than 2 E is kept, what lies below it by more is not, and where what lies
// between (as a rule the cut's own page and nothing else) is not taken as a whole, it gets its exact scores and the cut is looked for again.  Then the kept pages in order: a
// thread has a run of pages.
#define SELECT_THREADS 512
#define SELECT_BITS 10
#define SELECT_BINS (1 << SELECT_BITS)
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
    const int shift = max(0, 32 - __clz(high - low) - SELECT_BITS);
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
    sum += __reduce_add_sync(0xffffffffu, lane < warp ? sh.scan[lane] : 0);
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
  sum += __reduce_add_sync(0xffffffffu, lane < warp ? sh.scan[lane] : 0);
  int tie = sum >> 16 & 0xffff, at = a.keep_first + (sum & 0xffff) + min(tie, ties);
  for (int i = i0; i < i1; ++i) {
    const uint32_t k = sel_keys[i];
    if (k > cut || (k == cut && tie < ties)) ids[at++] = p0 + i;
    tie += k == cut;
  }
  for (int i = tid; i < a.keep_first; i += SELECT_THREADS) ids[i] = i;
  for (int i = tid; i < a.keep_last; i += SELECT_THREADS) ids[a.budget - a.keep_last + i] = n - a.keep_last + i;
}
