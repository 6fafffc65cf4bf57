// Truncated sampling on rows of logits: dream_sample draws a token per row, dream_truncate_logits leaves the kept tokens and
// puts the others at -inf (what the sampling acceptance of Section 2.1 reads when the target samples from a truncated distribution).
//
//   w_i = exp((l_i - max l) / T);  order: larger l first, then lower id;  kept: the first n of the order,
//   n = max(1, min(top_k, tokens until the mass before the next one reaches top_p of the top_k's mass, tokens with w >= min_p)).
//   token: the first kept id, in id order, at which the running sum of w exceeds u * (sum over the kept).
//
// A token is a whole number, so a row's sums have to be exact enough that no rounding moves a border: an error of 1e-7 of the
// total, what 32-bit exponentials leave, moves the token of one row in ten where 100000 tokens share the mass.  Weights are
// therefore taken in double (to 1.3e-12, Weigher).  Lists and histograms add them as 64-bit integers, whose sums do not depend on their order: of
// 2^-53 of the largest weight in a list (512 of them, half a unit off each: 2.8e-14), in histograms of as small a part as lets the row's mass fit (2^-43
// of the mass at most).  The draw and the mass in front of a list add them in double, in one fixed order.  All told a border is good to some
// 2e-12 of the row's mass.
//
// A row is read once into shared memory, by one block or a cluster of up to 16 whose blocks exchange through shared memory.  The cut is
// a logit and the last id kept among its ties.  Ways to it:
//   few tokens (top_k up to 112, greedy): the k-th largest of the threads' own maxima is a bound that little more than k logits pass; those
//     are listed, and one block settles order, masses, cut and draw on the list.  Against the bins below, by top_k alone: one row of 32000 takes
//     9.4 us at 50, 10.5 at 64, 13.5 at 112, 19.2 at 128 and 55.7 at 256, through the bins 11.5 to 12.0; 61 rows 13.2, 15.0, 18.2, 25.0 and 66.4,
//     through the bins 18.2 to 19.7; 64 rows of 131072 30.7, 33.9, 40.3, 53.7 and 132, through the bins 52 to 55.  With a top_p behind it the
//     bins take half as long again, and the list wins up to 112 everywhere (12.7 against 19.6 us at 96 in one row of 32000).
//   many: a pass sorts the row into bins of 1 / 128 nat, with counts (top_k) or approximate masses (top_p); the bin in which the cut falls is
//     listed (a full one is divided once more) and settled exactly, the mass in front of it being summed exactly: the bins only say where to look.
//   neither list fits (masked rows, rows of ties, logits of an odd scale), or the exact mass contradicts the bins: a radix selection over
//     order-preserving keys, eleven bits a level, by count or by exact mass, which assumes nothing about the values.
//
// What bounds it: no unit, but a block's steps one after the other (load, maximum over the cluster, bins, list, weights, draw), of which two blocks
// per SM overlap part.  Warp instructions for 32 logits, all told, and how often a scheduler issued: a temperature alone 52 (29 in the two passes,
// nine of them in double; the other 23 are a warp's 730 around its 1024 logits), 49 % of the time; 244 rows cut by top_p 144, 52 %; a nucleus over
// eight wide rows 185, 32 %.
//   1 row of 32000, top_k 50, top_p 0.9: 9.8 us, a launch and a chain of cluster barriers (44 with radix levels alone)
//   8 rows of 262144 fp32, top_p 0.95: 64 to 95 us, by how often the bins have to be divided
//   61 rows of 32003 bf16, settings mixed by row: 37 to 43 us
//   64 rows of 131072 at top_k 50, top_p 0.9: 31 us, in bf16 19; at top_k 5000: 65 us
//   256 rows of 131072, a temperature alone: 107 us (1.25 TB/s; 159 with weights by series)
//   61 rows of 32000 truncated at top_k 40, top_p 0.95: 13.8 us; 244 rows of 131072 at top_p 0.9, min_p 0.002: 264 to 294 us
// 512 threads and two blocks per SM: one block's barriers pass while the other computes.
#pragma once
#include "common.cuh"
#include "rows.cuh"

#define SAMPLE_MAX_CLUSTER 16          // above 8 for up to 9 rows
#define SAMPLE_MAX_VOCAB 262144
#define SAMPLE_BINS 2048
#define SAMPLE_CHUNKS 32               // of SAMPLE_BINS / 32 bins, a lane each
#define SAMPLE_EXCHANGES 12
#define SAMPLE_LIST 512                // listed tokens one block settles
#define SAMPLE_SMALL_K 112             // above, settling the list takes longer than the bins do
#define SAMPLE_THREADS 512

typedef unsigned long long u64;

struct SampleArgs {
  const void *logits;
  long long ld;                        // elements from one row to the next
  int vocab, cluster, warp_elems;      // logits per warp, a multiple of 32 vectors of 16 bytes
  const float *temperature;            // [rows] each, or null: the values below for every row
  const int *top_k;
  const float *top_p, *min_p, *uniforms;
  float t0, p0, m0;
  int k0;
  int *tokens;
  float *logprob;                      // may be null
  int *kept;                           // may be null
  int *status;                         // of a context, or null: a row without mass then raises it and gives token 0
  void *out;
  long long out_ld;
};

struct SampleShared {
  u64 xch[SAMPLE_EXCHANGES][SAMPLE_MAX_CLUSTER];   // one 64-bit word from every CTA of the cluster
  u64 warp_tot[32];
  u64 coarse[SAMPLE_CHUNKS];
  uint32_t warp_cnt[32];
  float2 warp_f[32];
  // what a selection level found
  int bin, chunk;
  uint32_t bin_cnt;
  u64 before, total;
  // listed tokens (of the whole cluster, in its first CTA) and what they settle
  uint32_t list_n[3];                  // a counter for each list a row may need
  float list_l[SAMPLE_LIST], cut_l;
  int list_id[SAMPLE_LIST], min_id;
  u64 list_w[SAMPLE_LIST];
  double table[32];                    // of the weights (Weigher)
  double c2;                           // of the row
  int cut_id;
  uint32_t cnt[SAMPLE_BINS], lo[SAMPLE_BINS], hi[SAMPLE_BINS];
  __device__ uint32_t *part() { return lo; }       // 64 words from every CTA, where there are no exact masses
};

// Sums and inclusive running sums over a warp, of u64 or double.
template <typename A> __device__ __forceinline__ A warp_total(A v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <typename A> __device__ __forceinline__ A warp_scan(A v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const A t = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += t;
  }
  return v;
}
__device__ __forceinline__ u64 as_bits(u64 v) { return v; }
__device__ __forceinline__ u64 as_bits(double v) { return (u64)__double_as_longlong(v); }
template <typename A> __device__ __forceinline__ A of_bits(u64 v);
template <> __device__ __forceinline__ u64 of_bits<u64>(u64 v) { return v; }
template <> __device__ __forceinline__ double of_bits<double>(u64 v) { return __longlong_as_double((long long)v); }

// exp((l - m) / T), also as an integer.  2^y by table, as in Tang's table-driven exponential: y = n + j / 32 + r, |r| <= 1 / 64, and 2^r by the
// Taylor series of e^(r ln 2) to its fourth power (remainder 1.3e-12).  The rounding to 1 / 32 is an addition of a number so large that its
// last bit is 1 / 32.  Nine operations in double, where a series without a table takes fourteen.
#define SAMPLE_TABLE 32
struct Weigher {
  double m, c2, one;                   // row maximum, log2(e) / T, what a weight of 1 is as an integer
  float cut;                           // below it a weight is less than e^-700 and counts as zero; rounded up: raw() has no weights for what lies
                                       // farther below, at a very low temperature the very next float
  const double *table;                 // 2^(j / 32), in shared memory
  __device__ __forceinline__ double raw(float l) const {
    const double d = (double)fminf(l, 3.402823466e38f) - m;
    const double big = 6755399441055744.0 / SAMPLE_TABLE;       // 1.5 * 2^52 / 32: its last bit is 1 / 32
    const double t = fma(d, c2, big), r = fma(d, c2, -(t - big));
    const int n = __double2loint(t);
    const double e = table[n & (SAMPLE_TABLE - 1)];
    double p = fma(r, 0.009618129107628477, 0.05550410866482158);          // ln(2)^k / k!, k = 4, 3, 2, 1
    p = fma(p, r, 0.2402265069591007);
    p = fma(p, r, 0.6931471805599453);
    p = fma(e, p * r, e);
    return __hiloint2double(__double2hiint(p) + ((n >> 5) << 20), __double2loint(p));
  }
  __device__ __forceinline__ double exact(float l) const { const double p = raw(l); return l >= cut ? p : 0.0; }
  __device__ __forceinline__ u64 units(float l) const {
    const u64 w = __double2ull_rn(raw(l) * one);
    return l >= cut ? w : 0ull;
  }
  // The smallest logit whose weight is above zero in double; beside +inf nothing else has any.
  __device__ __forceinline__ double least(double temp) const { return cut == INFINITY ? (double)INFINITY : m - 744.0 * temp; }
};

// A cut of the order: larger logits stay, and equal ones up to an id; -inf and NaN never do.
struct Cut {
  float l;
  int id;
  __device__ __forceinline__ bool keeps(float x, int i) const { return x > l || (x == l && i <= id); }
};

template <typename T>
struct SampleRow {
  static constexpr int VEC = 16 / sizeof(T);
  const SampleArgs &a;
  SampleShared &sh;
  uint4 *vals;                           // this CTA's logits, as they came
  int rank, nw, warp, lane, steps, base; // base: id of the warp's first logit; vectors lie on 16-byte boundaries, so the row's first may begin below 0

  __device__ __forceinline__ void unpack(const uint4 &q, float (&l)[VEC]) const {
    if constexpr (sizeof(T) == 4) {
      l[0] = __uint_as_float(q.x); l[1] = __uint_as_float(q.y); l[2] = __uint_as_float(q.z); l[3] = __uint_as_float(q.w);
    } else {
      const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) { l[2 * i] = __uint_as_float(u[i] << 16); l[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
    }
  }
  // f(logits, id of the first) for the thread's vectors
  template <typename F> __device__ __forceinline__ void each_vec(F f) const {
    const uint4 *p = vals + (size_t)warp * steps * 32 + lane;
    int i0 = base + lane * VEC;
#pragma unroll 1
    for (int j = 0; j < steps; ++j, p += 32, i0 += 32 * VEC) {
      float l[VEC];
      unpack(*p, l);
      f(l, i0);
    }
  }
  // f(logit, id) for the thread's logits, ascending ids inside a thread
  template <typename F> __device__ __forceinline__ void each(F f) const {
    each_vec([&](const float (&l)[VEC], int i0) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) f(l[e], i0 + e);
    });
  }
  // One word from every CTA to every CTA; ends in a barrier of the cluster.
  __device__ __forceinline__ void exchange(int slot, u64 v) const {
    if (threadIdx.x < a.cluster) st_cluster_u64(mapa_of(a.cluster, smem_u32(&sh.xch[slot][rank]), threadIdx.x), v);
    sync_all_of(a.cluster);
  }

  // The row into shared memory.  own: the thread's largest logit (NaN does not count; past the row's end: -inf); most, least: the
  // largest and the smallest of those that are not -inf.
  __device__ __forceinline__ void load(int row, float &own, float &most, float &least) const {
    const T *src = (const T *)a.logits + row * a.ld;
    uint4 *p = vals + (size_t)warp * steps * 32 + lane;
    float m = -INFINITY;
    const int first = base + lane * VEC;
    constexpr int U = 8;
    int j = 0;
    if (base >= 0) {                                        // whole vectors, as many at once as there are
      const uint4 *s = reinterpret_cast<const uint4 *>(src + first);
      const int whole = max(0, min(steps, (a.vocab - base) / (32 * VEC)));
      for (; j + U <= whole; j += U) {
        uint4 q[U];
#pragma unroll
        for (int k = 0; k < U; ++k) q[k] = s[(j + k) * 32];
#pragma unroll
        for (int k = 0; k < U; ++k) { m = fmaxf(m, max_vec<T, VEC>(q[k])); p[(j + k) * 32] = q[k]; }
      }
    }
#pragma unroll 2
    for (; j < steps; ++j) {
      const int i = first + j * 32 * VEC;
      uint4 q;
      if (i >= 0 && i + VEC <= a.vocab) q = *reinterpret_cast<const uint4 *>(src + i);
      else {
        T t[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) t[e] = i + e >= 0 && i + e < a.vocab ? src[i + e] : from_f<T>(-INFINITY);
        memcpy(&q, t, 16);
      }
      m = fmaxf(m, max_vec<T, VEC>(q));
      p[j * 32] = q;
    }
    own = m;
    most = warp_max(m);
    least = -warp_max(m > -INFINITY ? -m : -INFINITY);
    if (lane == 0) sh.warp_f[warp] = make_float2(most, least);
    if (threadIdx.x == 0) { sh.list_n[0] = sh.list_n[1] = sh.list_n[2] = 0; sh.min_id = 0x7fffffff; }
    __syncthreads();
    cluster_started_wait(a.cluster);
    const float2 w = lane < nw ? sh.warp_f[lane] : make_float2(-INFINITY, INFINITY);
    most = warp_max(w.x);
    least = -warp_max(-w.y);
    exchange(0, (u64)__float_as_uint(most) | (u64)__float_as_uint(least) << 32);
    const u64 x = sh.xch[0][min(lane, a.cluster - 1)];
    most = warp_max(__uint_as_float((uint32_t)x));
    least = -warp_max(-__uint_as_float((uint32_t)(x >> 32)));
  }

  // One level of the selection.  walk(put) hands put(bin, term) the tokens, or one value a thread; of the bins, from the top, that one is
  // found in which the running sum reaches goal(total), and left in sh.bin, with what is in front of it and how much of cnt it holds.  enough: false,
  // and nothing found, where the goal is not below the total.  Bin 0 may hold most of a row, so it is added up in registers first.
  //   COUNT: tokens.  UNITS: exact mass, a 64-bit sum in two words.  NATS: approximate mass; a bin holds weights in 2^-17 of the weight at its upper
  //   edge (slope 1: bins of 1 / 128 nat) or at that of the top bin (0), good to a few 1e-6 of a bin.
  enum { COUNT, UNITS, NATS };
  template <int KIND> __device__ __forceinline__ auto bin_sum(float slope, int i, uint32_t n, uint32_t lo, uint32_t hi) const {
    if constexpr (KIND == COUNT) return n;
    else if constexpr (KIND == UNITS) return (u64)lo + ((u64)hi << 32);
    else return (float)n * ex2((float)(i - (SAMPLE_BINS - 1)) * (slope * (1.44269504f / 128.f)) - 17.f);
  }
  template <int KIND, typename F, typename G> __device__ __forceinline__ bool level(bool first, bool enough, F walk, G goal, float slope = 0.f) const {
    constexpr bool EXACT = KIND == UNITS;
    typedef decltype(bin_sum<KIND>(0.f, 0, 0u, 0u, 0u)) A;
    if (!first) sync_all_of(a.cluster);                     // nobody still reads the bins of the level before
    for (int i = threadIdx.x; i < SAMPLE_BINS; i += SAMPLE_THREADS) {
      sh.cnt[i] = 0;
      if (EXACT) { sh.lo[i] = 0; sh.hi[i] = 0; }
    }
    __syncthreads();
    uint32_t n0 = 0;
    u64 w0 = 0;
    auto add = [&](int bin, uint32_t n, u64 w) {
      atomicAdd(&sh.cnt[bin], n);
      if (EXACT && w) {
        const uint32_t low = (uint32_t)w, old = atomicAdd(&sh.lo[bin], low), up = (uint32_t)(w >> 32) + (old + low < old ? 1u : 0u);
        if (up) atomicAdd(&sh.hi[bin], up);
      }
    };
    walk([&](int bin, u64 w) {
      if (bin > 0 && bin < SAMPLE_BINS) add(bin, KIND == NATS ? (uint32_t)w : 1u, w);
      if (KIND != NATS) n0 += bin == 0 ? 1u : 0u;
      if (EXACT) w0 += bin == 0 ? w : 0ull;
    });
    if (KIND != NATS) {
      n0 = __reduce_add_sync(0xffffffffu, n0);
      if (EXACT) w0 = warp_total<u64>(w0);
      if (lane == 0 && n0) add(0, n0, w0);
    }
    __syncthreads();
    A *coarse = reinterpret_cast<A *>(sh.coarse);
    for (int ch = warp; ch < SAMPLE_CHUNKS; ch += nw) {
      const int i = ch * 64 + lane;
      A w = bin_sum<KIND>(slope, i, sh.cnt[i], EXACT ? sh.lo[i] : 0u, EXACT ? sh.hi[i] : 0u) + bin_sum<KIND>(slope, i + 32, sh.cnt[i + 32], EXACT ? sh.lo[i + 32] : 0u, EXACT ? sh.hi[i + 32] : 0u);
      if constexpr (KIND == COUNT) w = __reduce_add_sync(0xffffffffu, w);
      else w = warp_total<A>(w);
      if (lane == 0) coarse[ch] = w;
    }
    sync_all_of(a.cluster);
    // Each warp reads a CTA's chunks, then its bins of the chunk in question, and the first warp adds them up: read one after the other the
    // round trips to the other CTAs took longer than all else.  (Exact masses, the rare case, are in the way and are read one by one.)
    auto of_chunk = [&](int q) -> A {                       // lane 0 has the top chunk
      const uint32_t from = mapa_of(a.cluster, smem_u32(coarse + SAMPLE_CHUNKS - 1 - lane), q);
      if constexpr (EXACT) return (A)ld_cluster_u64(from);
      else if constexpr (KIND == NATS) return ld_cluster(from);
      else return (A)ld_cluster_u32(from);
    };
    if constexpr (!EXACT) {
      for (int q = warp; q < a.cluster; q += nw) reinterpret_cast<A *>(sh.part())[q * 64 + lane] = of_chunk(q);
      __syncthreads();
    }
    A before = 0, want = 0;
    if (warp == 0) {
      A c = 0;
      for (int q = 0; q < a.cluster; ++q) {
        if constexpr (EXACT) c += of_chunk(q);
        else c += reinterpret_cast<A *>(sh.part())[q * 64 + lane];
      }
      const A run = warp_scan<A>(c), total = __shfl_sync(0xffffffffu, run, 31);
      want = goal(total);
      const unsigned hit = __ballot_sync(0xffffffffu, run >= want);
      const int at = !hit || (enough && want >= total) ? -1 : __ffs(hit) - 1;
      before = __shfl_sync(0xffffffffu, run - c, max(at, 0));
      if (lane == 0) { sh.chunk = at; if (at < 0) sh.bin = -1; if (KIND != NATS) sh.total = (u64)total; }
    }
    __syncthreads();
    const int at = sh.chunk;
    if (at < 0) return false;
    const int top = (SAMPLE_CHUNKS - at) * 64 - 1;          // bins descending from here, two to a lane
    if (!EXACT) {
      for (int q = warp; q < a.cluster; q += nw)
#pragma unroll
        for (int k = 0; k < 2; ++k) sh.part()[q * 64 + 2 * lane + k] = ld_cluster_u32(mapa_of(a.cluster, smem_u32(&sh.cnt[top - 2 * lane - k]), q));
      __syncthreads();
    }
    if (warp == 0) {
      A w[2] = {0, 0};
      uint32_t n[2] = {0, 0};
      for (int q = 0; q < a.cluster; ++q)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int i = top - 2 * lane - k;
          if constexpr (EXACT) {
            n[k] += ld_cluster_u32(mapa_of(a.cluster, smem_u32(&sh.cnt[i]), q));
            w[k] += ld_cluster_u32(mapa_of(a.cluster, smem_u32(&sh.lo[i]), q)) + ((u64)ld_cluster_u32(mapa_of(a.cluster, smem_u32(&sh.hi[i]), q)) << 32);
          } else n[k] += sh.part()[q * 64 + 2 * lane + k];
        }
      if (!EXACT) for (int k = 0; k < 2; ++k) w[k] = bin_sum<KIND>(slope, top - 2 * lane - k, n[k], 0u, 0u);
      const A run = before + warp_scan<A>(w[0] + w[1]);
      const unsigned hit = __ballot_sync(0xffffffffu, run >= want);
      // a sum in float may fall a rounding short of its chunk's: the chunk's last bin then
      if (lane == (hit ? __ffs(hit) - 1 : 31)) {
        const A front = run - w[0] - w[1];
        const int k = front + w[0] >= want ? 0 : 1;
        sh.bin = top - 2 * lane - k;
        if (KIND != NATS) sh.before = (u64)(front + (k ? w[0] : (A)0));
        sh.bin_cnt = n[k];
      }
    }
    __syncthreads();
    return sh.bin >= 0;
  }

  // The first token in id order at which the running sum of vals exceeds goal(total): found(logit, id, total) runs in the one thread that
  // holds it.  vals(logits, first id, v) gives a vector's terms and returns how many tokens they count for.  Two exchange slots (the second
  // carries the count); returns the total.  In double as in integers the sums have one order, and every warp has the same ones.  The blocks' borders
  // are added up one by one and never fall, so the goal is one block's.  The warps' come from a scan, in which a border may fall by a rounding or a warp
  // without a term have room: the goal is the first warp's with terms whose end lies above it.  (Each warp by its own two borders, a goal on one, as
  // half the mass of a row of two equal halves, was two warps' or nobody's; with the warps added up one by one 256 rows of 131072 took 3 us more.)
  template <typename A, typename V, typename G, typename H> __device__ __forceinline__ A locate(int slot, V vals_of, G goal, H found) const {
    A s = 0;
    uint32_t n = 0;
    each_vec([&](const float (&l)[VEC], int i0) {
      A v[VEC];
      n += vals_of(l, i0, v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) s += v[e];
    });
    s = warp_total<A>(s);
    n = __reduce_add_sync(0xffffffffu, n);
    __syncthreads();
    if (lane == 0) { sh.warp_tot[warp] = as_bits(s); sh.warp_cnt[warp] = n; }
    __syncthreads();
    const A term = lane < nw ? of_bits<A>(sh.warp_tot[lane]) : (A)0, inc = warp_scan<A>(term), all = __shfl_sync(0xffffffffu, inc, nw - 1);
    const unsigned some = __ballot_sync(0xffffffffu, term > (A)0);
    n = __reduce_add_sync(0xffffffffu, lane < nw ? sh.warp_cnt[lane] : 0u);
    if (threadIdx.x < a.cluster) st_cluster_u64(mapa_of(a.cluster, smem_u32(&sh.xch[slot + 1][rank]), threadIdx.x), (u64)n);
    exchange(slot, as_bits(all));
    A before = 0, total = 0;
    for (int q = 0; q < a.cluster; ++q) {
      if (q == rank) before = total;
      total += of_bits<A>(sh.xch[slot][q]);
    }
    const A want = goal(total);
    const unsigned above = __ballot_sync(0xffffffffu, before + inc > want) & some;
    if (want >= before && want < before + all && warp == (above ? __ffs(above) - 1 : 31 - __clz(some))) {
      const A up_to = __shfl_sync(0xffffffffu, inc, max(warp, 1) - 1), start = warp ? before + up_to : before;
      A left = want > start ? want - start : (A)0;
      int last = -1;                                        // with a term of its own, for a rounding that puts the goal behind the lane's end or the warp's
      float last_l = 0.f;
      bool done = false;
      const uint4 *p = vals + (size_t)warp * steps * 32 + lane;
#pragma unroll 1
      for (int j = 0; j < steps && !done; ++j) {
        float l[VEC];
        unpack(p[j * 32], l);
        const int i0 = base + (j * 32 + lane) * VEC;
        A v[VEC], sum = 0;
        vals_of(l, i0, v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) { sum += v[e]; if (v[e] > (A)0) { last = i0 + e; last_l = l[e]; } }
        const A in = warp_scan<A>(sum), group = __shfl_sync(0xffffffffu, in, 31);
        const unsigned hit = __ballot_sync(0xffffffffu, in > left);
        if (hit) {
          const A up = __shfl_up_sync(0xffffffffu, in, 1);
          const int at = __ffs(hit) - 1;
          bool mine = false;
          if (lane == at) {
            A run = lane ? up : (A)0;
            int id = -1;
            float x = 0.f;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              run += v[e];
              if (!mine && run > left) { mine = true; id = i0 + e; x = l[e]; }
            }
            if (mine) found(x, id, total);
          }
          // the lanes' sums reach the goal and their terms one by one do not: the last term up to there
          if (!__any_sync(0xffffffffu, mine)) {
            const int id = __reduce_max_sync(0xffffffffu, lane <= at ? last : -1);
            if (lane <= at && id >= 0 && id == last) found(last_l, id, total);
          }
          done = true;
        } else left -= group;
      }
      if (!done) {
        const int id = __reduce_max_sync(0xffffffffu, last);
        if (id >= 0 && id == last) found(last_l, id, total);
      }
    }
    return total;
  }

  // The last of the first r tokens of a logit in id order, to every CTA.
  __device__ __forceinline__ int nth_tie(float tie, u64 r) const {
    locate<u64>(2, [&](const float (&l)[VEC], int, u64 (&v)[VEC]) {
#pragma unroll
                  for (int e = 0; e < VEC; ++e) v[e] = (u64)(l[e] == tie);
                  return 0u;
                }, [&](u64) { return r - 1; },
           [&](float, int id, u64) { for (int q = 0; q < a.cluster; ++q) st_cluster_u64(mapa_of(a.cluster, smem_u32(&sh.xch[10][0]), q), (u64)id); });
    sync_all_of(a.cluster);
    return (int)sh.xch[10][0];
  }

  static __device__ __forceinline__ u64 mass_goal(double top_p, u64 total) {     // masses below it stay; the first token always does
    const u64 g = (u64)ceil(top_p * (double)total);
    return g < 1 ? (u64)1 : g > total ? total : g;
  }
  // Radix selection, three levels down to one key.  By count: the `want` first; by mass: until top_p of the mass is reached.
  template <bool MASS> __device__ __forceinline__ Cut radix(Cut cut, u64 want, double top_p, Weigher weigh, double z = 0.0) const {
    uint32_t prefix = 0;
    if (MASS) {                                             // z, where it is known: the mass within the cut
      if (z == 0.0) {
        each([&](float l, int id) { const double w = weigh.exact(l); z += cut.keeps(l, id) ? w : 0.0; });
        push(8, block_sum(z));
        sync_all_of(a.cluster);
        z = pushed(8);
      }
      weigh.one = __hiloint2double((2 * 1023 + 60 - (__double2hiint(z) >> 20)) << 20, 0);      // z units are below 2^61
    }
    u64 goal = want, ties = 0;
#pragma unroll 1
    for (int lev = 0; lev < 3; ++lev) {
      const int shift = lev == 0 ? 21 : lev == 1 ? 10 : 0, width = lev == 2 ? 1023 : 2047;
      const uint32_t above = lev == 0 ? 0u : lev == 1 ? 0xffe00000u : 0xfffffc00u;
      if (!level<MASS ? UNITS : COUNT>(false, !MASS && lev == 0,
          [&](auto put) {
            each([&](float l, int id) {
              const uint32_t k = topk_key(l);
              if ((k & above) != prefix || !cut.keeps(l, id)) return;
              put((int)((k >> shift) & width), MASS ? weigh.units(l) : 0ull);
            });
          },
          [&](auto total) { return (decltype(total))(MASS && lev == 0 ? mass_goal(top_p, (u64)total) : goal); }))
        return cut;                                         // fewer tokens than top_k
      if (MASS && lev == 0) goal = mass_goal(top_p, sh.total);
      goal -= sh.before;
      prefix |= (uint32_t)sh.bin << shift;
      ties = sh.bin_cnt;
      __syncthreads();
    }
    u64 r = goal;                                           // ties of the key that stay
    if (MASS) {
      const u64 w = weigh.units(topk_value(prefix));
      r = (goal + w - 1) / w;
    }
    Cut found = {topk_value(prefix), 0x7fffffff};
    if (r < ties) {
      found.id = nth_tie(found.l, r);
      __syncthreads();
    }
    if (found.l == cut.l && cut.id < found.id) found.id = cut.id;
    return found;
  }

  // ---- lists.  Tokens that want(logit, id) to the list of the cluster's first CTA; returns how many there are, which may be more than fit.
  template <typename F, typename P> __device__ __forceinline__ uint32_t list(int which, F want, P before_barrier) const {
    const uint32_t counter = mapa_of(a.cluster, smem_u32(&sh.list_n[which]), 0);
    each([&](float l, int id) {
      if (!want(l, id)) return;
      uint32_t at;
      asm volatile("atom.shared::cluster.add.u32 %0, [%1], 1;" : "=r"(at) : "r"(counter) : "memory");
      if (at < SAMPLE_LIST) {
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(mapa_of(a.cluster, smem_u32(sh.list_l + at), 0)), "r"(__float_as_uint(l)) : "memory");
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(mapa_of(a.cluster, smem_u32(sh.list_id + at), 0)), "r"((uint32_t)id) : "memory");
      }
    });
    before_barrier();
    sync_all_of(a.cluster);
    return ld_cluster_u32(counter);
  }
  __device__ __forceinline__ u64 block_sum_u64(u64 v) const {
    v = warp_total<u64>(v);
    __syncthreads();
    if (lane == 0) sh.warp_tot[warp] = v;
    __syncthreads();
    return warp_total<u64>(lane < nw ? sh.warp_tot[lane] : 0ull);
  }
  // What became of the list, in the first CTA.  `share` threads have an entry together, the one with part 0 holds what became of it.
  struct Settled {
    int entry, share, part, id;        // entry: -1 without one
    float l;
    bool stays;
    u64 w, n, mass;                    // its weight (0 if it is cut); how many stay, and their mass
  };
  // Settles the n listed tokens, which follow tokens that all stay: top_k more of them stay, of these those before which the mass is below
  // goal(their mass), of these those with logits from least_l on; the first of the order does in any case if `one`.  Each entry counts the
  // entries in front of it; threads share an entry so that all of the block works.
  template <typename G> __device__ __forceinline__ Settled settle(uint32_t n, u64 top_k, G goal, float least_l, bool one, const Weigher &weigh) const {
    const int tid = threadIdx.x;
    Settled r;
    r.share = SAMPLE_THREADS;
    for (uint32_t m = 1; m < n; m *= 2) r.share /= 2;
    r.share = max(1, min(32, r.share));
    r.part = tid % r.share;
    r.entry = tid / r.share < (int)n ? tid / r.share : -1;
    for (uint32_t i = tid; i < n; i += SAMPLE_THREADS) sh.list_w[i] = weigh.units(sh.list_l[i]);
    __syncthreads();
    r.l = r.entry >= 0 ? sh.list_l[r.entry] : 0.f;
    r.id = r.entry >= 0 ? sh.list_id[r.entry] : 0;
    const u64 w = r.entry >= 0 ? sh.list_w[r.entry] : 0ull;
    uint32_t rank = 0;
    u64 before = 0;
    for (uint32_t j = r.part; j < n; j += r.share) {
      const float lj = sh.list_l[j];
      if (lj > r.l || (lj == r.l && sh.list_id[j] < r.id)) { ++rank; before += sh.list_w[j]; }
    }
    for (int o = r.share >> 1; o > 0; o >>= 1) { rank += __shfl_xor_sync(0xffffffffu, rank, o); before += __shfl_xor_sync(0xffffffffu, before, o); }
    const bool mine = r.entry >= 0 && r.part == 0, in_k = rank < top_k;
    const u64 want = goal(block_sum_u64(mine && in_k ? w : 0ull));
    r.stays = mine && ((in_k && before < want && r.l >= least_l) || (one && rank == 0));
    r.w = r.stays ? w : 0ull;
    r.mass = block_sum_u64(r.w);
    r.n = block_sum_u64(r.stays ? 1ull : 0ull);
    if (r.stays && rank + 1 == r.n) { sh.cut_l = r.l; sh.cut_id = r.id; }
    __syncthreads();
    return r;
  }
  // The kept entry at which the running mass in id order exceeds goal(their mass); u == 0: the first with any mass at all.  found(logit, id, mass)
  // runs in the thread that holds it.
  template <typename G, typename H> __device__ __forceinline__ void draw_settled(const Settled &r, uint32_t n, float u, double least, G goal, H found) const {
    const bool stays = __shfl_sync(0xffffffffu, (int)r.stays, (int)(threadIdx.x & 31) / r.share * r.share);
    if (r.entry >= 0 && r.part == 0) sh.list_w[r.entry] = r.w;             // cut tokens weigh nothing from here on
    if (r.stays && u == 0.f && (double)r.l >= least) atomicMin(&sh.min_id, r.id);
    __syncthreads();
    u64 before = 0;
    if (stays)
      for (uint32_t j = r.part; j < n; j += r.share) if (sh.list_id[j] < r.id) before += sh.list_w[j];
    for (int o = r.share >> 1; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
    const u64 t = goal(r.mass);
    if (r.stays && (u == 0.f ? r.id == sh.min_id : before <= t && t - before < r.w)) found(r.l, r.id, r.mass);
  }
  // The first CTA's cut to all.
  __device__ __forceinline__ Cut share_cut(int slot) const {
    if (rank == 0 && threadIdx.x < a.cluster)
      st_cluster_u64(mapa_of(a.cluster, smem_u32(&sh.xch[slot][0]), threadIdx.x), (u64)__float_as_uint(sh.cut_l) << 32 | (uint32_t)sh.cut_id);
    sync_all_of(a.cluster);
    return {__uint_as_float((uint32_t)(sh.xch[slot][0] >> 32)), (int)(uint32_t)sh.xch[slot][0]};
  }

  __device__ __forceinline__ double block_sum(double v) const {
    v = warp_total<double>(v);
    __syncthreads();
    if (lane == 0) sh.warp_tot[warp] = as_bits(v);
    __syncthreads();
    return warp_total<double>(lane < nw ? of_bits<double>(sh.warp_tot[lane]) : 0.0);
  }
  __device__ __forceinline__ void push(int slot, double v) const {       // to every CTA; there behind the next barrier of the cluster
    if (threadIdx.x < a.cluster) st_cluster_u64(mapa_of(a.cluster, smem_u32(&sh.xch[slot][rank]), threadIdx.x), as_bits(v));
  }
  __device__ __forceinline__ double pushed(int slot) const {
    double v = 0.0;
    for (int q = 0; q < a.cluster; ++q) v += of_bits<double>(sh.xch[slot][q]);
    return v;
  }
  // Many tokens, by count (top_k) or by mass (top_p) within the cut.  Bins of 1 / 128 nat below the row's maximum, up to 16 nats; where the bin in
  // which the cut falls holds too many to list, once more with bins a fraction as wide.  By mass the bins are approximate and only
  // say where to look: the mass in front of the bin's upper neighbour is then summed exactly, and the three bins are listed.
  // fresh: nobody has used the bins yet.
  template <bool MASS> __device__ __forceinline__ Cut select(bool fresh, Cut cut, u64 top_k, double top_p, const Weigher &weigh, float m, float temp) const {
    constexpr int LAST = SAMPLE_BINS - 1;
    const float scale = 128.f / temp;
    float x0 = 0.f, fine = 1.f;                             // where the bins begin, and how many to 1 / 128 nat
    // Product and difference rounded apart: both looks then see one product, and where it is x0 or more the difference is exact.  Fused, the second
    // look would take a product that rounds up to x0 for less, and its token, which the first look did not count in front, would be lost to the count.
    auto depth = [&](float l) { return __fsub_rn(__fmul_rn(m - l, scale), x0); };
    auto place = [&](float x) { return (int)floorf(fminf(x * fine, (float)LAST)); };       // NaN: the last
    double z = 0.0;
    u64 left = top_k;
    int at = 0;
    if (!(scale < INFINITY)) return radix<MASS>(cut, top_k, top_p, weigh);      // everything in one place
#pragma unroll 1
    for (int lev = 0;; ++lev) {
      const bool found_bin = level<MASS ? NATS : COUNT>(fresh && lev == 0, !MASS && lev == 0,
            [&](auto put) {
              if (!MASS) {
                each([&](float l, int id) {
                  const int i = place(depth(l));
                  if (cut.keeps(l, id) && i >= 0) put(LAST - i, 0ull);
                });
                return;
              }
              double s = 0.0;                               // of the row; then of what lies in front of the finer bins
              each_vec([&](const float (&l)[VEC], int i0) {
                bool sum[VEC], any = false;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                  const bool on = cut.keeps(l[e], i0 + e);
                  const float x = depth(l[e]);
                  const int i = place(x);
                  sum[e] = on && (lev == 0 || i < 0);
                  any = any || sum[e];
                  if (on && i >= 0 && i < LAST) {
                    const float y = (lev ? x : x - (float)i) * (1.f / 128.f);
                    put(LAST - i, (u64)(uint32_t)(131072.5f - 131072.f * y * (1.f - y * (0.5f - y * (1.f / 6.f)))));
                  }
                }
                if (any) {
#pragma unroll
                  for (int e = 0; e < VEC; ++e) { const double w = weigh.exact(l[e]); s += sum[e] ? w : 0.0; }
                }
              });
              push(lev ? 9 : 8, block_sum(s));
            },
            [&](auto total) {
              typedef decltype(total) A;
              if (!MASS) return (A)left;
              z = pushed(8);
              return (A)fmax(1e-30, lev ? (top_p * z - pushed(9)) * exp((double)x0 / 128.0) : top_p * z);
            }, lev ? 0.f : 1.f);
      if (!MASS && lev == 0 && !found_bin) return cut;      // no more tokens than top_k
      if (MASS) z = pushed(8);
      at = LAST - sh.bin;
      const uint32_t n = MASS ? 3 * (sh.bin_cnt >> 17) : sh.bin_cnt;
      if (!found_bin || at >= LAST) return radix<MASS>(cut, top_k, top_p, weigh, z);
      if (!MASS) left -= sh.before;
      __syncthreads();
      if (lev || n <= SAMPLE_LIST - 100) break;
      x0 = MASS ? fmaxf((float)(at - 1), 0.f) : (float)at;
      fine = MASS ? (float)LAST / 3.f : (float)LAST;
    }
    // the mass in front of the list: after a second look only what lies between the finer bins' first and the list is new
    const bool twice = x0 > 0.f || fine != 1.f;
    double s = 0.0;
    const uint32_t n = list(MASS ? 2 : 1, [&](float l, int id) {
          if (!cut.keeps(l, id)) return false;
          const int i = place(depth(l));
          if (MASS && i < at - 1 && (!twice || i >= 0)) s += weigh.exact(l);
          return MASS ? i >= max(at - 1, 0) && i <= at + 1 : i == at;          // what lies in front of the bins is in the mass in front already
        }, [&] { if (MASS) push(11, block_sum(s)); });
    if (rank == 0) {
      bool good = n <= SAMPLE_LIST;
      if (good) {
        const double rest = MASS ? top_p * z - (twice ? pushed(9) + pushed(11) : pushed(11)) : 0.0;        // of the listed tokens' mass
        const u64 units = MASS ? (u64)fmax(0.0, ceil(rest * weigh.one)) : 0ull;
        const auto r = settle(n, MASS ? (u64)n : left, [&](u64 mass) {
            if (MASS && (rest <= 0.0 || units > mass)) sh.bin = -2;        // the bins were too coarse: the cut is not among them
            return MASS ? units : ~0ull;
          }, -INFINITY, false, weigh);
        good = sh.bin != -2 && r.n > 0;
      }
      __syncthreads();
      if (!good && threadIdx.x == 0) { sh.cut_l = INFINITY; sh.cut_id = -1; }
      __syncthreads();
    }
    const Cut found = share_cut(MASS ? 7 : 6);
    if (found.l == INFINITY && found.id < 0) return radix<MASS>(cut, top_k, top_p, weigh, z);
    return found;
  }
};

template <typename T, bool TRUNCATE>
__global__ void __launch_bounds__(SAMPLE_THREADS, 2)
k_sample(const __grid_constant__ SampleArgs a) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  SampleShared &sh = *reinterpret_cast<SampleShared *>(smem_raw);
  constexpr int VEC = SampleRow<T>::VEC;
  cluster_started_arrive(a.cluster);
  kernel_entry(TRUNCATE ? TR_k_truncate : TR_k_sample);
  const int rank = a.cluster > 1 ? (int)cluster_ctarank() : 0, row = blockIdx.x / a.cluster, nw = SAMPLE_THREADS / 32, warp = threadIdx.x >> 5;
  const SampleRow<T> R = {a, sh, reinterpret_cast<uint4 *>(smem_raw + (sizeof(SampleShared) + 15) / 16 * 16), rank, nw, warp, (int)(threadIdx.x & 31),
                          a.warp_elems / (32 * VEC),
                          (rank * nw + warp) * a.warp_elems - (int)((uintptr_t)((const T *)a.logits + row * a.ld) / sizeof(T) % VEC)};
  float temp = a.temperature ? a.temperature[row] : a.t0;
  int k = a.top_k ? a.top_k[row] : a.k0;
  float top_p = a.top_p ? a.top_p[row] : a.p0;
  const float min_p = a.min_p ? a.min_p[row] : a.m0, u = TRUNCATE ? 0.f : fmaxf(a.uniforms[row], 0.f);
  if (!(temp > 0.f)) { temp = 1.f; k = 1; }                 // greedy
  // what takes many instructions is one warp's
  if (warp == 0) sh.table[threadIdx.x] = exp2((double)threadIdx.x / SAMPLE_TABLE);
  else if (warp == 1) { const double c2 = 1.4426950408889634 / (double)temp; if (threadIdx.x == 32) sh.c2 = c2; }
  float own, m, lowest;
  R.load(row, own, m, lowest);
  Cut cut = {-INFINITY, (int)0x80000000};                   // every token above -inf
  Weigher weigh;
  const bool infinite = m == INFINITY;                      // the infinite ones share the mass
  weigh.table = sh.table;
  weigh.m = (double)m; weigh.c2 = sh.c2; weigh.one = 0x1p53;      // SAMPLE_LIST ones fit
  weigh.cut = fmaxf(__double2float_ru(weigh.m - 700.0 * (double)temp), -3.402823466e38f);
  if (infinite) { weigh.m = (double)3.402823466e38f; weigh.cut = INFINITY; }
  auto target = [&](u64 total) { const u64 t = (u64)((double)u * (double)total); return t < total ? t : total - 1; };
  auto draw = [&](float l, int id, double total) {
    a.tokens[row] = id;
    if (a.logprob) a.logprob[row] = (float)((infinite ? 0.0 : ((double)l - weigh.m) / (double)temp) - log(total));
  };
  if (m > -INFINITY) {
    float least_l = -INFINITY;
    bool tried = false;                                     // the bins have been used
    if (min_p > 0.f) {                                      // w >= min_p
      if (min_p > 1.f) k = 1;                               // nothing but the first of the order
      else if (infinite) least_l = m;
      else if (temp < INFINITY) least_l = fminf(__double2float_ru(weigh.m + log((double)min_p) * (double)temp), m);      // beyond, all weigh 1
    }
    if (k > 0 && k < a.vocab) {
      // Few tokens: a bin of the threads' own maxima, in 2047 steps from the smallest (or 256 below the largest) to the largest, down to which
      // there are k of them.
      const float low = fmaxf(lowest, m - 256.f), scale = (float)(SAMPLE_BINS - 1) / (m - low);
      auto bin_of = [&](float l) { return l >= low ? (int)((l - low) * scale) : 0; };
      bool listed = false;
      if (k <= SAMPLE_SMALL_K && scale > 0.f && scale < INFINITY) {
        tried = true;
        R.template level<SampleRow<T>::COUNT>(true, false, [&](auto put) { put(bin_of(own), 0ull); }, [&](uint32_t) { return (uint32_t)k; });
        const int bin = sh.bin;
        __syncthreads();
        uint32_t n = SAMPLE_LIST + 1;
        if (bin > 0) n = R.list(0, [&](float l, int) { return bin_of(l) >= bin; }, [] {});
        listed = n <= SAMPLE_LIST;
        if (listed) {
          if (rank == 0) {
            const auto r = R.settle(n, (u64)k, [&](u64 mass) { return top_p < 1.f ? SampleRow<T>::mass_goal((double)top_p, mass) : ~0ull; }, least_l, true, weigh);
            if (!TRUNCATE) {
              R.draw_settled(r, n, u, weigh.least((double)temp), target, [&](float l, int id, u64 total) { draw(l, id, (double)total * 0x1p-53); });
              if (threadIdx.x == 0 && a.kept) a.kept[row] = (int)r.n;
            }
          }
          if (!TRUNCATE) {                                  // the first CTA stays until the others have read how long its list is
            sync_all_of(a.cluster);
            return;
          }
          cut = R.share_cut(6);
          top_p = 1.f; least_l = -INFINITY;                      // settled with the list
        }
      }
      if (!listed) {
        cut = R.template select<false>(!tried, cut, (u64)k, 0.0, weigh, m, temp);
        tried = true;
      }
    }
    if (top_p < 1.f) cut = R.template select<true>(!tried, cut, 0, fmax((double)top_p, 1e-30), weigh, m, temp);
    if (least_l > cut.l) cut = {least_l, 0x7fffffff};       // the largest logit passes it: a first one always stays
  }
  uint32_t n = 0;
  if (TRUNCATE) {
    T *dst = (T *)a.out + row * a.out_ld;
    const bool out_vec = ((uintptr_t)(dst + R.base) & 15) == 0;          // the output lies on its boundaries like the row
    const uint4 *p = R.vals + (size_t)warp * R.steps * 32 + R.lane;
#pragma unroll 1
    for (int j = 0; j < R.steps; ++j) {
      const int i0 = R.base + (j * 32 + R.lane) * VEC;
      float l[VEC];
      R.unpack(p[j * 32], l);
      T t[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const bool on = cut.keeps(l[e], i0 + e);
        n += on ? 1u : 0u;
        t[e] = from_f<T>(on ? l[e] : -INFINITY);
      }
      if (out_vec && i0 >= 0 && i0 + VEC <= a.vocab) {
        uint4 q;
        memcpy(&q, t, 16);
        *reinterpret_cast<uint4 *>(dst + i0) = q;
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) if (i0 + e >= 0 && i0 + e < a.vocab) dst[i0 + e] = t[e];
      }
    }
    if (a.kept) {
      n = __reduce_add_sync(0xffffffffu, n);
      __syncthreads();
      if (R.lane == 0) sh.warp_cnt[warp] = n;
      __syncthreads();
      n = __reduce_add_sync(0xffffffffu, R.lane < nw ? sh.warp_cnt[R.lane] : 0u);
      R.exchange(1, (u64)n);
      if (rank == 0 && threadIdx.x == 0) {
        u64 all = 0;
        for (int q = 0; q < a.cluster; ++q) all += sh.xch[1][q];
        a.kept[row] = (int)all;
      }
    } else sync_all_of(a.cluster);                          // no CTA leaves while another may still read its histograms
    return;
  }
  if (!(m > -INFINITY)) {                                   // nothing to draw from
    if (rank == 0 && threadIdx.x == 0) {
      a.tokens[row] = a.status ? 0 : -1;
      if (a.status) atomicMax(a.status, DREAM_DEV_BAD_INDEX);
      if (a.logprob) a.logprob[row] = -INFINITY;
      if (a.kept) a.kept[row] = 0;
    }
    return;
  }
  auto whole = [&](const float (&l)[VEC], int, double (&v)[VEC]) {         // nothing is cut: no comparison and no branch among the weights
    uint32_t n = 0;
#pragma unroll
    for (int e = 0; e < VEC; ++e) { v[e] = weigh.exact(l[e]); n += l[e] > -INFINITY ? 1u : 0u; }
    return n;
  };
  auto weights = [&](const float (&l)[VEC], int i0, double (&v)[VEC]) {
    uint32_t n = 0;
    {
      bool on[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) { on[e] = cut.keeps(l[e], i0 + e); v[e] = 0.0; n += on[e] ? 1u : 0u; }
      if (n) {                                              // all of a vector: a branch per token would cost more
#pragma unroll
        for (int e = 0; e < VEC; ++e) { const double w = weigh.exact(l[e]); v[e] = on[e] ? w : 0.0; }
      }
    }
    return n;
  };
  auto goal = [&](double total) { return fmin((double)u * total, total * 0.9999999999999999); };
  auto found = [&](float l, int id, double total) { if (u > 0.f) draw(l, id, total); };
  const double total = cut.l == -INFINITY ? R.template locate<double>(4, whole, goal, found) : R.template locate<double>(4, weights, goal, found);
  if (u == 0.f)                                             // the first kept id with any mass in double, be it below e^-700
    R.template locate<u64>(2, [&](const float (&l)[VEC], int i0, u64 (&v)[VEC]) {
                             const double least = weigh.least((double)temp);
#pragma unroll
                             for (int e = 0; e < VEC; ++e) v[e] = (u64)(cut.keeps(l[e], i0 + e) && (double)l[e] >= least);
                             return 0u;
                           }, [](u64) { return 0ull; }, [&](float l, int id, u64) { draw(l, id, total); });
  if (rank == 0 && threadIdx.x == 0 && a.kept) {
    u64 all = 0;
    for (int q = 0; q < a.cluster; ++q) all += sh.xch[5][q];
    a.kept[row] = (int)all;
  }
}
