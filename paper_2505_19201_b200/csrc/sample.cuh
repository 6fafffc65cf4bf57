// Truncated sampling on rows of logits: dream_sample draws a token per row, dream_truncate_logits leaves the kept tokens and
// puts the others at -inf (what the sampling acceptance of Section 2.1 reads when the target samples from a truncated distribution).
//
//   w_i = exp((l_i - max l) / T);  order: larger l first, then lower id;  kept: the first n of the order,
//   n = max(1, min(top_k, tokens until the mass before the next one reaches top_p of the top_k's mass, tokens with w >= min_p)).
//   token: the first kept id, in id order, at which the running sum of w exceeds u * (sum over the kept).
//
// A token is a whole number, so a row's sums have to be exact enough that no rounding moves a border: an error of 1e-7 of the
// total, what 32-bit exponentials leave, moves the token of one row in ten where 100000 tokens share the mass.  Weights are
// therefore taken in double (to 3e-13) and summed as 64-bit integers of 2^-s (s such that a whole row of ones fits), whose sums do
// not depend on their order: histograms by atomics, shares of a cluster and scans all agree bit for bit.
//
// The cut is a pair (key, id): an order-preserving 32-bit key of the logit and the last id kept among its ties.  It is found by a radix
// selection over the keys, eleven bits a level, by count (top_k) or by mass (top_p), so it needs no sort and no assumption on the
// values: rows masked with the type's lowest value, infinities and rows of ties take the same three levels.
#pragma once
#include "common.cuh"
#include "rows.cuh"

#define SAMPLE_MAX_CLUSTER 8
#define SAMPLE_CTA_MAX 32768           // logits of a row one CTA holds (128 KB as fp32)
#define SAMPLE_MAX_VOCAB (SAMPLE_MAX_CLUSTER * SAMPLE_CTA_MAX)
#define SAMPLE_BINS 2048
#define SAMPLE_CHUNKS 32               // of SAMPLE_BINS / 32 bins, a lane each
#define SAMPLE_EXCHANGES 8

typedef unsigned long long u64;

struct SampleArgs {
  const void *logits;
  long long ld;                        // elements from one row to the next
  int vocab, cluster, warp_elems;      // logits per warp, a multiple of 32 vectors of 16 bytes
  int frac_bits;                       // s: weights are integers of 2^-s
  int vec, out_vec;                    // rows (of the output) start on 16-byte boundaries
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
  u64 coarse_mass[2][SAMPLE_CHUNKS];
  uint32_t coarse_cnt[2][SAMPLE_CHUNKS];
  uint32_t warp_cnt[32];
  float warp_f[32];
  // what a selection level found
  int bin;
  uint32_t bin_cnt;
  u64 before_cnt, before_mass, total;
  // histograms of two levels: while one is read by the cluster the next is filled
  uint32_t cnt[2][SAMPLE_BINS], lo[2][SAMPLE_BINS], hi[2][SAMPLE_BINS];
};

__device__ __forceinline__ u64 warp_sum_u64(u64 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ u64 warp_scan_u64(u64 v) {            // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 t = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += t;
  }
  return v;
}

// exp((l - m) / T) as an integer of 2^-s.  2^y by the textbook reduction y = n + r, |r| <= 1/2, and the Taylor series of
// e^(r ln 2) to its tenth power (remainder 2.2e-13 at the ends); both roundings to integers are additions of a number so large that its
// last bit is the unit wanted.
struct Weigher {
  double m, c2, unit;                  // row maximum, log2(e) / T, 2^(52 - s)
  float cut;                           // below it a weight is less than half a unit
  __device__ __forceinline__ u64 operator()(float l) const {
    const double d = (double)fminf(fmaxf(l, cut), 3.402823466e38f) - m;
    const double big = 6755399441055744.0;         // 1.5 * 2^52
    const double t = fma(d, c2, big), r = fma(d, c2, -(t - big));
    double p = 7.054911620801121e-09;              // ln(2)^k / k!, k = 10 .. 0
    p = fma(p, r, 1.0178086009239696e-07);
    p = fma(p, r, 1.3215486790144305e-06);
    p = fma(p, r, 1.5252733804059838e-05);
    p = fma(p, r, 1.5403530393381606e-04);
    p = fma(p, r, 1.3333558146428441e-03);
    p = fma(p, r, 9.618129107628477e-03);
    p = fma(p, r, 5.5504108664821576e-02);
    p = fma(p, r, 2.402265069591007e-01);
    p = fma(p, r, 6.931471805599453e-01);
    p = fma(p, r, 1.0);
    p = __hiloint2double(__double2hiint(p) + (__double2loint(t) << 20), __double2loint(p));
    const u64 w = (u64)__double_as_longlong(p + unit) - (u64)__double_as_longlong(unit);
    return l >= cut ? w : 0ull;
  }
  // The smallest logit whose weight is above zero in double.
  __device__ __forceinline__ double least(double temp) const { return cut == INFINITY ? INFINITY : m - 744.0 * temp; }
};

// A cut of the order: tokens in front of it stay.  Its key is never below that of -inf, which no cut keeps (nor NaN).
struct Cut {
  uint32_t key;
  int id;
  __device__ __forceinline__ bool keeps(uint32_t k, int i) const { return k > key || (k == key && i <= id); }
};
#define KEY_NEG_INF 0x007fffffu          // topk_key(-inf); NaN is 0

template <typename T>
struct SampleRow {
  static constexpr int VEC = 16 / sizeof(T);
  const SampleArgs &a;
  SampleShared &sh;
  uint4 *vals;                           // this CTA's logits, as they came
  int rank, nw, warp, lane, steps, base; // base: id of the warp's first logit
  mutable int turn;                      // which of the two histograms is next

  __device__ __forceinline__ void unpack(const uint4 &q, float (&l)[VEC]) const {
    if constexpr (sizeof(T) == 4) {
      l[0] = __uint_as_float(q.x); l[1] = __uint_as_float(q.y); l[2] = __uint_as_float(q.z); l[3] = __uint_as_float(q.w);
    } else {
      const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) { l[2 * i] = __uint_as_float(u[i] << 16); l[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
    }
  }
  // f(logit, id) for the thread's logits, ascending ids inside a thread
  template <typename F> __device__ __forceinline__ void each(F f) const {
    const uint4 *p = vals + (size_t)warp * steps * 32 + lane;
#pragma unroll 1
    for (int j = 0; j < steps; ++j) {
      float l[VEC];
      unpack(p[j * 32], l);
#pragma unroll
      for (int e = 0; e < VEC; ++e) f(l[e], base + (j * 32 + lane) * VEC + e);
    }
  }
  // One word from every CTA to every CTA; ends in a barrier of the cluster.
  __device__ __forceinline__ void exchange(int slot, u64 v) const {
    if (threadIdx.x < a.cluster) st_cluster_u64(mapa_of(a.cluster, smem_u32(&sh.xch[slot][rank]), threadIdx.x), v);
    sync_all_of(a.cluster);
  }

  // The row into shared memory; returns its maximum (NaN does not count).  Past the row's end: -inf.
  __device__ __forceinline__ float load(int row) const {
    const T *src = (const T *)a.logits + row * a.ld;
    const T neg = from_f<T>(-INFINITY);
    uint4 *p = vals + (size_t)warp * steps * 32 + lane;
    float m = -INFINITY;
    constexpr int U = 8;
    for (int j0 = 0; j0 < steps; j0 += U) {
      uint4 q[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int i = base + ((j0 + k) * 32 + lane) * VEC;
        if (j0 + k < steps && a.vec && i + VEC <= a.vocab) q[k] = __ldg(reinterpret_cast<const uint4 *>(src + i));
        else {
          T t[VEC];
#pragma unroll
          for (int e = 0; e < VEC; ++e) t[e] = j0 + k < steps && i + e < a.vocab ? src[i + e] : neg;
          memcpy(&q[k], t, 16);
        }
      }
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (j0 + k < steps) {
          float l[VEC];
          unpack(q[k], l);
#pragma unroll
          for (int e = 0; e < VEC; ++e) m = fmaxf(m, l[e]);
          p[(j0 + k) * 32] = q[k];
        }
    }
    m = warp_max(m);
    if (lane == 0) sh.warp_f[warp] = m;
    __syncthreads();
    m = warp_max(lane < nw ? sh.warp_f[lane] : -INFINITY);
    cluster_started_wait(a.cluster);
    exchange(0, (u64)__float_as_uint(m));
    for (int q = 0; q < a.cluster; ++q) m = fmaxf(m, __uint_as_float((uint32_t)sh.xch[0][q]));
    return m;
  }

  // One level of the selection: among the tokens that f gives a bin (>= 0) and a mass, the bin, from the top, in which the running
  // count (MASS false) or mass reaches `goal(total)`.  Leaves it in sh.bin .. sh.total; false, and nothing found, where the total is not
  // above the goal by count.
  template <bool MASS, typename F, typename G> __device__ __forceinline__ bool level(int lev, F f, G goal) const {
    const int b = turn++ & 1;
    for (int i = threadIdx.x; i < SAMPLE_BINS; i += blockDim.x) {
      sh.cnt[b][i] = 0;
      if (MASS) { sh.lo[b][i] = 0; sh.hi[b][i] = 0; }
    }
    __syncthreads();
    each([&](float l, int id) {
      u64 w = 0;
      const int bin = f(l, id, w);
      if (bin < 0) return;
      atomicAdd(&sh.cnt[b][bin], 1u);
      if (MASS && w) {
        const uint32_t add = (uint32_t)w, old = atomicAdd(&sh.lo[b][bin], add), carry = old + add < old ? 1u : 0u;
        const uint32_t up = (uint32_t)(w >> 32) + carry;
        if (up) atomicAdd(&sh.hi[b][bin], up);
      }
    });
    __syncthreads();
    for (int ch = warp; ch < SAMPLE_CHUNKS; ch += nw) {
      const int i = ch * (SAMPLE_BINS / SAMPLE_CHUNKS) + lane;
      uint32_t c = sh.cnt[b][i] + sh.cnt[b][i + 32];
      c = __reduce_add_sync(0xffffffffu, c);
      u64 w = 0;
      if (MASS) w = warp_sum_u64(bin_mass(b, i) + bin_mass(b, i + 32));
      if (lane == 0) { sh.coarse_cnt[b][ch] = c; if (MASS) sh.coarse_mass[b][ch] = w; }
    }
    sync_all_of(a.cluster);
    if (warp == 0) {
      // lane 0 has the top chunk
      const int ch = SAMPLE_CHUNKS - 1 - lane;
      u64 c = 0, w = 0;
      for (int q = 0; q < a.cluster; ++q) {
        c += ld_cluster_u32(mapa_of(a.cluster, smem_u32(&sh.coarse_cnt[b][ch]), q));
        if (MASS) w += ld_cluster_u64(mapa_of(a.cluster, smem_u32(&sh.coarse_mass[b][ch]), q));
      }
      const u64 ic = warp_scan_u64(c), iw = MASS ? warp_scan_u64(w) : 0;
      const u64 total = __shfl_sync(0xffffffffu, MASS ? iw : ic, 31), want = goal(total);
      const unsigned hit = __ballot_sync(0xffffffffu, (MASS ? iw : ic) >= want);
      if (!hit || (!MASS && want >= total && lev == 0)) { if (lane == 0) sh.bin = -1; }
      else {
        const int at = __ffs(hit) - 1;                                   // the chunk
        const u64 bc = __shfl_sync(0xffffffffu, ic - c, at), bw = __shfl_sync(0xffffffffu, iw - w, at);
        const int top = (SAMPLE_CHUNKS - at) * (SAMPLE_BINS / SAMPLE_CHUNKS) - 1;
        u64 c2[2] = {0, 0}, w2[2] = {0, 0};
        for (int q = 0; q < a.cluster; ++q)
#pragma unroll
          for (int k = 0; k < 2; ++k) {                                  // lane's bins, descending: top - 2 lane, then the next
            const int i = top - 2 * lane - k;
            c2[k] += ld_cluster_u32(mapa_of(a.cluster, smem_u32(&sh.cnt[b][i]), q));
            if (MASS) w2[k] += (u64)ld_cluster_u32(mapa_of(a.cluster, smem_u32(&sh.lo[b][i]), q)) + ((u64)ld_cluster_u32(mapa_of(a.cluster, smem_u32(&sh.hi[b][i]), q)) << 32);
          }
        const u64 sc = bc + warp_scan_u64(c2[0] + c2[1]), sw = bw + (MASS ? warp_scan_u64(w2[0] + w2[1]) : 0);
        const unsigned h2 = __ballot_sync(0xffffffffu, (MASS ? sw : sc) >= want);
        if (lane == __ffs(h2) - 1) {
          const u64 c0 = sc - c2[0] - c2[1], w0 = sw - w2[0] - w2[1];
          const int k = (MASS ? w0 + w2[0] : c0 + c2[0]) >= want ? 0 : 1;
          sh.bin = top - 2 * lane - k;
          sh.before_cnt = c0 + (k ? c2[0] : 0);
          sh.before_mass = w0 + (k ? w2[0] : 0);
          sh.bin_cnt = (uint32_t)c2[k];
          sh.total = total;
        }
      }
    }
    __syncthreads();
    return sh.bin >= 0;
  }
  __device__ __forceinline__ u64 bin_mass(int b, int i) const { return (u64)sh.lo[b][i] + ((u64)sh.hi[b][i] << 32); }

  // The first token in id order at which the running sum of val exceeds goal(total): found(logit, id, total) runs in the one thread that
  // holds it.  Two exchange slots (the second carries `side`, summed over the threads); returns the total.
  template <typename V, typename G, typename H> __device__ __forceinline__ u64 locate(int slot, V val, G goal, uint32_t side, H found) const {
    u64 s = 0;
    each([&](float l, int id) { s += val(l, id); });
    s = warp_sum_u64(s);
    side = __reduce_add_sync(0xffffffffu, side);
    __syncthreads();
    if (lane == 0) { sh.warp_tot[warp] = s; sh.warp_cnt[warp] = side; }
    __syncthreads();
    const u64 mine = lane < nw ? sh.warp_tot[lane] : 0, inc = warp_scan_u64(mine), all = __shfl_sync(0xffffffffu, inc, 31);
    const u64 n = __reduce_add_sync(0xffffffffu, lane < nw ? sh.warp_cnt[lane] : 0u);
    if (threadIdx.x < a.cluster) st_cluster_u64(mapa_of(a.cluster, smem_u32(&sh.xch[slot + 1][rank]), threadIdx.x), n);
    exchange(slot, all);
    u64 before = 0, total = 0;
    for (int q = 0; q < a.cluster; ++q) { const u64 x = sh.xch[slot][q]; total += x; if (q < rank) before += x; }
    const u64 want = goal(total);
    before += __shfl_sync(0xffffffffu, inc - mine, warp);
    if (total && want >= before && want - before < s) {                 // a warp at most
      u64 left = want - before;
      const uint4 *p = vals + (size_t)warp * steps * 32 + lane;
#pragma unroll 1
      for (int j = 0; j < steps; ++j) {
        float l[VEC];
        unpack(p[j * 32], l);
        const int i0 = base + (j * 32 + lane) * VEC;
        u64 v[VEC], sum = 0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) { v[e] = val(l[e], i0 + e); sum += v[e]; }
        const u64 in = warp_scan_u64(sum), group = __shfl_sync(0xffffffffu, in, 31);
        if (left < group) {
          const unsigned hit = __ballot_sync(0xffffffffu, in > left);
          if (lane == __ffs(hit) - 1) {
            u64 run = in - sum;
            bool done = false;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              run += v[e];
              if (!done && run > left) { done = true; found(l[e], i0 + e, total); }
            }
          }
          break;
        }
        left -= group;
      }
    }
    return total;
  }

  // The last of the first r ties of `key` in id order, to every CTA.
  __device__ __forceinline__ int nth_tie(uint32_t key, u64 r) const {
    locate(2, [&](float l, int) { return (u64)(topk_key(l) == key); }, [&](u64) { return r - 1; }, 0u,
           [&](float, int id, u64) { for (int q = 0; q < a.cluster; ++q) st_cluster_u64(mapa_of(a.cluster, smem_u32(&sh.xch[4][0]), q), (u64)id); });
    sync_all_of(a.cluster);
    return (int)sh.xch[4][0];
  }

  // Three levels down to one key.  By count: the `want` first; by mass: until top_p of the mass is reached.
  template <bool MASS> __device__ __forceinline__ Cut select(Cut cut, u64 want, double top_p, const Weigher &weigh) const {
    uint32_t prefix = 0;
    u64 goal = want, ties = 0;
    for (int lev = 0; lev < 3; ++lev) {
      const int shift = lev == 0 ? 21 : lev == 1 ? 10 : 0, width = lev == 2 ? 1023 : 2047;
      const uint32_t above = lev == 0 ? 0u : lev == 1 ? 0xffe00000u : 0xfffffc00u;
      const bool any = level<MASS>(lev,
          [&](float l, int id, u64 &w) {
            const uint32_t k = topk_key(l);
            if ((k & above) != prefix || !cut.keeps(k, id)) return -1;
            if (MASS) w = weigh(l);
            return (int)((k >> shift) & width);
          },
          [&](u64 total) {
            if (MASS && lev == 0) { const u64 g = (u64)ceil(top_p * (double)total); return g < 1 ? (u64)1 : g > total ? total : g; }
            return goal;
          });
      if (!any) return cut;                                 // fewer tokens than top_k
      if (MASS && lev == 0) { const u64 g = (u64)ceil(top_p * (double)sh.total); goal = g < 1 ? (u64)1 : g > sh.total ? sh.total : g; }
      goal -= MASS ? sh.before_mass : sh.before_cnt;
      prefix |= (uint32_t)sh.bin << shift;
      ties = sh.bin_cnt;
      __syncthreads();
    }
    u64 r = goal;                                           // ties of the key that stay
    if (MASS) {
      const u64 w = weigh(topk_value(prefix));
      r = (goal + w - 1) / w;
    }
    Cut found = {prefix, 0x7fffffff};
    if (r < ties) {
      found.id = nth_tie(prefix, r);
      __syncthreads();
    }
    if (prefix == cut.key && cut.id < found.id) found.id = cut.id;
    return found;
  }
};

template <typename T, bool TRUNCATE>
__global__ void __launch_bounds__(1024)
k_sample(const __grid_constant__ SampleArgs a) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  SampleShared &sh = *reinterpret_cast<SampleShared *>(smem_raw);
  constexpr int VEC = SampleRow<T>::VEC;
  cluster_started_arrive(a.cluster);
  kernel_entry(TRUNCATE ? TR_k_truncate : TR_k_sample);
  const int rank = a.cluster > 1 ? (int)cluster_ctarank() : 0, row = blockIdx.x / a.cluster, nw = blockDim.x >> 5, warp = threadIdx.x >> 5;
  const SampleRow<T> R = {a, sh, reinterpret_cast<uint4 *>(smem_raw + sizeof(SampleShared)), rank, nw, warp, (int)(threadIdx.x & 31),
                          a.warp_elems / (32 * VEC), (rank * nw + warp) * a.warp_elems, 0};
  float temp = a.temperature ? a.temperature[row] : a.t0;
  int k = a.top_k ? a.top_k[row] : a.k0;
  const float top_p = a.top_p ? a.top_p[row] : a.p0, min_p = a.min_p ? a.min_p[row] : a.m0;
  if (!(temp > 0.f)) { temp = 1.f; k = 1; }                 // greedy
  const float m = R.load(row);
  Cut cut = {KEY_NEG_INF, -1};                              // every token above -inf
  Weigher weigh;
  weigh.m = (double)m; weigh.c2 = 1.4426950408889634 / (double)temp; weigh.unit = __longlong_as_double((long long)(1023 + 52 - a.frac_bits) << 52);
  weigh.cut = fmaxf(__double2float_rd(weigh.m - (double)(a.frac_bits + 2) * 0.69314718055994531 * (double)temp), -3.402823466e38f);
  if (m == INFINITY) { weigh.m = (double)3.402823466e38f; weigh.cut = INFINITY; }   // the infinite ones share the mass
  if (m > -INFINITY) {
    if (k > 0 && k < a.vocab) cut = R.template select<false>(cut, (u64)k, 0.0, weigh);
    if (top_p < 1.f) cut = R.template select<true>(cut, 0, (double)top_p, weigh);
    if (min_p > 0.f) {                      // w >= min_p; the first of the order always stays
      const double least = weigh.m + log((double)min_p) * (double)temp;
      const float edge = m == INFINITY ? m : fminf(__double2float_ru(least), m);
      Cut c = {topk_key(edge), 0x7fffffff};
      if (min_p > 1.f) c = R.template select<false>(cut, 1, 0.0, weigh);
      if (c.key > cut.key) cut = c;
      else if (c.key == cut.key && c.id < cut.id) cut = c;
    }
  }
  uint32_t n = 0;
  if (TRUNCATE) {
    T *dst = (T *)a.out + row * a.out_ld;
    const uint4 *p = R.vals + (size_t)warp * R.steps * 32 + R.lane;
#pragma unroll 1
    for (int j = 0; j < R.steps; ++j) {
      const int i0 = R.base + (j * 32 + R.lane) * VEC;
      float l[VEC];
      R.unpack(p[j * 32], l);
      T t[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const bool on = cut.keeps(topk_key(l[e]), i0 + e);
        n += on ? 1u : 0u;
        t[e] = from_f<T>(on ? l[e] : -INFINITY);
      }
      if (a.out_vec && i0 + VEC <= a.vocab) {
        uint4 q;
        memcpy(&q, t, 16);
        *reinterpret_cast<uint4 *>(dst + i0) = q;
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) if (i0 + e < a.vocab) dst[i0 + e] = t[e];
      }
    }
    if (a.kept) {
      n = __reduce_add_sync(0xffffffffu, n);
      __syncthreads();
      if (R.lane == 0) sh.warp_cnt[warp] = n;
      __syncthreads();
      n = __reduce_add_sync(0xffffffffu, R.lane < nw ? sh.warp_cnt[R.lane] : 0u);
      R.exchange(6, (u64)n);
      if (rank == 0 && threadIdx.x == 0) {
        u64 all = 0;
        for (int q = 0; q < a.cluster; ++q) all += sh.xch[6][q];
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
  R.each([&](float l, int id) { n += cut.keeps(topk_key(l), id) ? 1u : 0u; });
  const float u = fmaxf(a.uniforms[row], 0.f);
  auto draw = [&](float l, int id, u64 total) {
    a.tokens[row] = id;
    if (a.logprob) a.logprob[row] = (float)((m == INFINITY ? 0.0 : ((double)l - weigh.m) / (double)temp) - log(ldexp((double)total, -a.frac_bits)));
  };
  const u64 total = R.locate(6, [&](float l, int id) { return cut.keeps(topk_key(l), id) ? weigh(l) : 0ull; },
                             [&](u64 total) { const u64 t = (u64)((double)u * (double)total); return t < total ? t : total - 1; }, n,
                             [&](float l, int id, u64 total) { if (u > 0.f) draw(l, id, total); });
  if (u == 0.f)                                             // the first kept id with any mass, be it less than a unit
    R.locate(2, [&](float l, int id) { return (u64)(cut.keeps(topk_key(l), id) && l >= weigh.least((double)temp)); }, [](u64) { return 0ull; }, 0u,
             [&](float l, int id, u64) { draw(l, id, total); });
  if (rank == 0 && threadIdx.x == 0 && a.kept) {
    u64 all = 0;
    for (int q = 0; q < a.cluster; ++q) all += sh.xch[7][q];
    a.kept[row] = (int)all;
  }
}
