// Distillation of rows of logits from a teacher's top logits (the training signal of a draft: the target's distribution, Section 3,
// of which the top K logits were kept).
//
//   z_i = s_i / tau, lse = ln sum_i e^z_i, p_i = e^(z_i - lse)
//   teacher: without its log-sum-exp  q_j = softmax over the K valid entries of t_j / tau, q_r = 0;
//            with it                  q_j = e^(t_j / tau - teacher_lse), q_r = max(0, 1 - sum_j q_j): the rest is one bucket.
//   loss = sum_j q_j (ln q_j - ln p_j) + q_r (ln q_r - ln p_r),  p_r = sum of p over the ids that are not listed
//   d loss / d s_i = (1 / tau) (Q p_i - q_i) for listed ids, (1 / tau) p_i (Q - q_r / p_r) for the others,  Q = sum_j q_j + q_r.
//
// Bound by memory: a row is read once (and its gradient written once).  p_r would lose its digits as a difference of sums where the
// listed ids hold nearly everything, so the ids are marked in a bitmap and the others summed by themselves; the few numbers of the listed
// ids and of the row are in double.
#pragma once
#include "common.cuh"

#define DISTILL_MAX_TOP 128
#define DISTILL_MAX_CLUSTER 8
#define DISTILL_CTA_MAX 32768          // logits of a row one CTA holds
#define DISTILL_MAX_VOCAB (DISTILL_MAX_CLUSTER * DISTILL_CTA_MAX)

struct DistillArgs {
  const void *logits;
  long long ld;
  int vocab, cluster, cta_elems, top, vec, grad_vec;
  const int *ids;                      // [rows][top]; outside [0, vocab): no entry
  const float *teacher;                // [rows][top]
  const float *teacher_lse;            // [rows] or null
  double inv_tau;
  float *loss, *lse, *log_rest;        // [rows]; log_rest with teacher_lse only
  const float *row_scale;              // [rows] or null (1)
  void *grad;                          // or null
  long long grad_ld;
};

template <typename T, int VEC> __device__ __forceinline__ void unpack_vec(const uint4 &q, float (&l)[VEC]) {
  if constexpr (sizeof(T) == 4) {
    l[0] = __uint_as_float(q.x); l[1] = __uint_as_float(q.y); l[2] = __uint_as_float(q.z); l[3] = __uint_as_float(q.w);
  } else {
    const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { l[2 * i] = __uint_as_float(u[i] << 16); l[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
  }
}
template <typename T, int VEC> __device__ __forceinline__ uint4 pack_vec(const float (&g)[VEC]) {
  uint4 q;
  if constexpr (sizeof(T) == 4) q = make_uint4(__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3]));
  else {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(g[2 * i], g[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    q = make_uint4(u[0], u[1], u[2], u[3]);
  }
  return q;
}
// A vector of 16 bytes of a row of n elements at element i, `fill` behind the row's end.
template <typename T, int VEC> __device__ __forceinline__ uint4 load_vec(const T *row, int i, int n, bool vec, float fill) {
  if (vec && i + VEC <= n) return *reinterpret_cast<const uint4 *>(row + i);
  T t[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) t[e] = i + e < n ? row[i + e] : from_f<T>(fill);
  uint4 q;
  memcpy(&q, t, 16);
  return q;
}
template <typename T, int VEC> __device__ __forceinline__ void store_vec(T *row, int i, int n, bool vec, const uint4 &q) {
  if (vec && i + VEC <= n) { *reinterpret_cast<uint4 *>(row + i) = q; return; }
  T t[VEC];
  memcpy(t, &q, 16);
#pragma unroll
  for (int e = 0; e < VEC; ++e) if (i + e < n) row[i + e] = t[e];
}

// The teacher's side of a row, by the first DISTILL_MAX_TOP threads of a block of at least as many.
struct Teacher {
  double q[DISTILL_MAX_TOP];           // 0 for no entry
  int id[DISTILL_MAX_TOP];             // -1 for no entry
  double part[4][2];
  double rest, total;                  // q_r and Q
};
// Ends in a barrier: q, id, rest and total are there.
__device__ __forceinline__ void teacher_row(const DistillArgs &a, int row, Teacher &t) {
  const int j = threadIdx.x, lane = j & 31, warp = j >> 5;
  double x = -INFINITY, e = 0.0;
  int id = -1;
  if (j < DISTILL_MAX_TOP) {
    if (j < a.top) {
      id = a.ids[(long long)row * a.top + j];
      if (id < 0 || id >= a.vocab) id = -1;
      else x = (double)a.teacher[(long long)row * a.top + j] * a.inv_tau;
    }
    t.id[j] = id;
    if (a.teacher_lse) e = exp(x - (double)a.teacher_lse[row]);
    else {
      double m = x;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) m = fmax(m, __shfl_xor_sync(0xffffffffu, m, o));
      if (lane == 0) t.part[warp][0] = m;
    }
  }
  if (!a.teacher_lse) {
    __syncthreads();
    if (j < DISTILL_MAX_TOP) {
      const double m = fmax(fmax(t.part[0][0], t.part[1][0]), fmax(t.part[2][0], t.part[3][0]));
      e = x > -INFINITY ? exp(x - m) : 0.0;
    }
  }
  if (j < DISTILL_MAX_TOP) {
    if (id < 0) e = 0.0;
    double s = e;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) t.part[warp][1] = s;
  }
  __syncthreads();
  const double s = t.part[0][1] + t.part[1][1] + t.part[2][1] + t.part[3][1];
  const bool tail = a.teacher_lse != nullptr;
  const bool any = !(s == 0.0);                              // a row with no valid entry has no loss, with or without the rest
  if (j < DISTILL_MAX_TOP) t.q[j] = tail || !any ? e : e / s;
  if (j == 0) {
    t.rest = tail && any ? fmax(0.0, 1.0 - s) : 0.0;
    t.total = tail ? (any ? s + t.rest : 0.0) : any ? 1.0 : 0.0;
  }
  __syncthreads();
}

struct DistillShared {
  Teacher teacher;
  uint32_t bits[DISTILL_CTA_MAX / 32];     // ids of this CTA's share that are listed
  float warp_m[32], warp_s[32];
  double share[DISTILL_MAX_CLUSTER][4];    // of every CTA: maximum, sum over the others, sum over the listed, sum of q s
  uint32_t first[DISTILL_MAX_TOP];         // entry j is the one that stands for its id here
  float m, d2, coef;                       // row maximum, (lse - m / tau) log2 e, factor of e of an id that is not listed
  double lse, scale;
  int repeated;
};

// GRAD: the row stays in shared memory and its gradient leaves in the same pass.
template <typename T, bool GRAD>
__global__ void __launch_bounds__(1024)
k_distill(const __grid_constant__ DistillArgs a) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  DistillShared &sh = *reinterpret_cast<DistillShared *>(smem_raw);
  uint4 *vals = reinterpret_cast<uint4 *>(smem_raw + (sizeof(DistillShared) + 15) / 16 * 16);
  constexpr int VEC = 16 / sizeof(T);
  cluster_started_arrive(a.cluster);
  kernel_entry(TR_k_distill);
  const int rank = a.cluster > 1 ? (int)cluster_ctarank() : 0, row = blockIdx.x / a.cluster, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5,
            nw = blockDim.x >> 5, base = rank * a.cta_elems, n = min(a.cta_elems, a.vocab - base);   // n may be negative: an empty share
  const T *src = (const T *)a.logits + row * a.ld + base;
  T *dst = GRAD ? (T *)a.grad + row * a.grad_ld + base : nullptr;
  const float c2 = (float)(a.inv_tau * 1.4426950408889634), scale = a.row_scale ? a.row_scale[row] : 1.f;
  for (int i = tid; i < a.cta_elems / 32; i += blockDim.x) sh.bits[i] = 0;
  if (tid == 0) sh.repeated = 0;
  teacher_row(a, row, sh.teacher);
  if (tid < DISTILL_MAX_TOP) {
    const int id = sh.teacher.id[tid] - base;
    bool mine = sh.teacher.id[tid] >= 0 && id >= 0 && id < n;
    if (mine && (atomicOr(&sh.bits[id >> 5], 1u << (id & 31)) >> (id & 31) & 1u)) { mine = false; sh.repeated = 1; }
    sh.first[tid] = mine;
  }
  __syncthreads();
  // running maximum and sum of the ids that are not listed
  float m = -INFINITY, s = 0.f;
  const int steps = (max(n, 0) + blockDim.x * VEC - 1) / (blockDim.x * VEC);
  constexpr int U = 4;
  for (int j0 = 0; j0 < steps; j0 += U) {
    uint4 q[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int i = ((j0 + k) * blockDim.x + tid) * VEC;
      if (j0 + k < steps) q[k] = load_vec<T, VEC>(src, i, n, a.vec, -INFINITY);
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (j0 + k >= steps) break;
      const int i = ((j0 + k) * blockDim.x + tid) * VEC;
      float l[VEC];
      unpack_vec<T, VEC>(q[k], l);
      if (GRAD) vals[(j0 + k) * blockDim.x + tid] = q[k];
      if (i < n) {
        const uint32_t b = sh.bits[i >> 5] >> (i & 31);
        if (b & ((1u << VEC) - 1u)) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) if (b >> e & 1u) l[e] = -INFINITY;
        }
        float v = l[0];
#pragma unroll
        for (int e = 1; e < VEC; ++e) v = fmaxf(v, l[e]);
        if (v > m) { s *= ex2((m - v) * c2); m = v; }
        if (m > -INFINITY) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) s += ex2((l[e] - m) * c2);
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) if (l[e] != l[e]) s = l[e];      // NaN is not lost where nothing else is there
        }
      }
    }
  }
  {
    const float wm = warp_max(m);
    s = warp_sum(m > -INFINITY ? s * ex2((m - wm) * c2) : s);          // s is 0, or NaN, without a maximum
    if (lane == 0) { sh.warp_m[warp] = wm; sh.warp_s[warp] = s; }
  }
  __syncthreads();
  cluster_started_wait(a.cluster);
  if (warp == 0) {
    float wm = lane < nw ? sh.warp_m[lane] : -INFINITY, ws = lane < nw ? sh.warp_s[lane] : 0.f;
    float cm = warp_max(wm), z[DISTILL_MAX_TOP / 32];
    double qs = 0.0, tops = 0.0;
#pragma unroll
    for (int k = 0; k < DISTILL_MAX_TOP / 32; ++k) {
      const int id = sh.teacher.id[k * 32 + lane] - base;
      const bool mine = sh.teacher.id[k * 32 + lane] >= 0 && id >= 0 && id < n;
      z[k] = -INFINITY;
      if (mine) {
        z[k] = to_f(src[id]);
        if (sh.teacher.q[k * 32 + lane] > 0.0) qs += sh.teacher.q[k * 32 + lane] * (double)z[k];
      }
    }
#pragma unroll
    for (int k = 0; k < DISTILL_MAX_TOP / 32; ++k) cm = fmaxf(cm, warp_max(z[k]));
#pragma unroll
    for (int k = 0; k < DISTILL_MAX_TOP / 32; ++k)
      if (z[k] > -INFINITY && sh.first[k * 32 + lane]) tops += exp(((double)z[k] - (double)cm) * a.inv_tau);
    double others = wm > -INFINITY ? (double)ws * exp(((double)wm - (double)cm) * a.inv_tau) : (double)ws;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      qs += __shfl_xor_sync(0xffffffffu, qs, o);
      tops += __shfl_xor_sync(0xffffffffu, tops, o);
      others += __shfl_xor_sync(0xffffffffu, others, o);
    }
    if (lane < a.cluster) {
      const uint32_t to = mapa_of(a.cluster, smem_u32(&sh.share[rank][0]), lane);
      st_cluster_u64(to, __double_as_longlong((double)cm)); st_cluster_u64(to + 8, __double_as_longlong(others));
      st_cluster_u64(to + 16, __double_as_longlong(tops)); st_cluster_u64(to + 24, __double_as_longlong(qs));
    }
  }
  sync_all_of(a.cluster);
  const Teacher &t = sh.teacher;
  if (warp == 0) {
    double qlq = 0.0;
    if (rank == 0) {
#pragma unroll
      for (int k = 0; k < DISTILL_MAX_TOP / 32; ++k) { const double q = t.q[k * 32 + lane]; if (q > 0.0) qlq += q * log(q); }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) qlq += __shfl_xor_sync(0xffffffffu, qlq, o);
    }
    if (lane == 0) {
      double rm = -INFINITY, others = 0.0, tops = 0.0, qs = 0.0;
      for (int q = 0; q < a.cluster; ++q) rm = fmax(rm, sh.share[q][0]);
      for (int q = 0; q < a.cluster; ++q) {
        const double f = sh.share[q][0] > -INFINITY ? exp((sh.share[q][0] - rm) * a.inv_tau) : 1.0;
        others += sh.share[q][1] * f; tops += sh.share[q][2] * f; qs += sh.share[q][3];
      }
      const double total = others + tops, lz = log(total);               // relative to the row's maximum
      const double lse = rm * a.inv_tau + lz;
      const double log_rest = others > 0.0 ? -log1p(tops / others) : others == 0.0 ? -INFINITY : others;
      const bool none = total == 0.0;                                    // no finite logit
      if (rank == 0) {
        double loss = qlq - qs * a.inv_tau + (t.total - t.rest) * lse;
        if (t.rest > 0.0) loss += t.rest * (log(t.rest) - log_rest);
        if (none) loss = t.total > 0.0 ? INFINITY : 0.0;
        if (t.total == 0.0) loss = 0.0;
        a.loss[row] = (float)loss;
        a.lse[row] = none ? -INFINITY : (float)lse;
        if (a.teacher_lse) a.log_rest[row] = none ? -INFINITY : (float)log_rest;
      }
      if (GRAD) {
        const double sc = none ? 0.0 : (double)scale * a.inv_tau;
        sh.m = none ? 0.f : (float)rm;
        sh.d2 = none ? 0.f : (float)(lz * 1.4426950408889634);
        sh.lse = lse;
        sh.scale = t.total == 0.0 ? 0.0 : sc;
        sh.coef = t.total == 0.0 || sc == 0.0 ? 0.f : (float)(sc * (t.total - (t.rest > 0.0 && others > 0.0 ? t.rest * (total / others) : 0.0)));
      }
    }
  }
  if (!GRAD) return;
  __syncthreads();
  const float rm = sh.m, d2 = sh.d2, coef = sh.coef;
  const bool zero = sh.scale == 0.0;                                     // padding: zeros, whatever the logits hold
  for (int j = 0; j < steps; ++j) {
    const int i = (j * blockDim.x + tid) * VEC;
    float l[VEC], g[VEC];
    unpack_vec<T, VEC>(vals[j * blockDim.x + tid], l);
#pragma unroll
    for (int e = 0; e < VEC; ++e) g[e] = zero ? 0.f : coef * ex2(fmaf(l[e] - rm, c2, -d2));
    if (i < n) store_vec<T, VEC>(dst, i, n, a.grad_vec, pack_vec<T, VEC>(g));
  }
  if (zero) return;
  __syncthreads();                                                       // the listed ids' own gradients replace what was written
  if (tid < DISTILL_MAX_TOP && sh.first[tid]) {
    const int id = t.id[tid];
    double q = t.q[tid];
    if (sh.repeated) {
      q = 0.0;
      for (int j = 0; j < a.top; ++j) if (t.id[j] == id) q += t.q[j];
    }
    const double z = (double)to_f(reinterpret_cast<const T *>(vals)[id - base]) * a.inv_tau;
    dst[id - base] = from_f<T>((float)(sh.scale * (t.total * exp(z - sh.lse) - q)));
  }
}

// The gradient from a saved log-sum-exp (and, with teacher_lse, log_rest): a CTA takes DISTILL_GRAD_VECS vectors per thread of a row.
#define DISTILL_GRAD_THREADS 256
#define DISTILL_GRAD_VECS 4
template <typename T>
__global__ void __launch_bounds__(DISTILL_GRAD_THREADS)
k_distill_grad(const __grid_constant__ DistillArgs a) {
  __shared__ Teacher t;
  constexpr int VEC = 16 / sizeof(T), CHUNK = DISTILL_GRAD_THREADS * DISTILL_GRAD_VECS * VEC;
  kernel_entry(TR_k_distill_grad);
  const int chunks = (a.vocab + CHUNK - 1) / CHUNK, row = blockIdx.x / chunks, base = (blockIdx.x - row * chunks) * CHUNK,
            n = min(CHUNK, a.vocab - base), tid = threadIdx.x;
  const T *src = (const T *)a.logits + row * a.ld + base;
  T *dst = (T *)a.grad + row * a.grad_ld + base;
  const bool pad = a.row_scale && a.row_scale[row] == 0.f;               // a row of padding is not read
  const double lse = (double)a.lse[row], scale = (a.row_scale ? (double)a.row_scale[row] : 1.0) * a.inv_tau;
  const float c2 = (float)(a.inv_tau * 1.4426950408889634);
  uint4 q[DISTILL_GRAD_VECS];
#pragma unroll
  for (int k = 0; k < DISTILL_GRAD_VECS; ++k) q[k] = load_vec<T, VEC>(src, (k * DISTILL_GRAD_THREADS + tid) * VEC, pad ? 0 : n, a.vec, -INFINITY);
  teacher_row(a, row, t);
  const bool zero = scale == 0.0 || t.total == 0.0 || lse == -INFINITY;
  const double tail = t.rest > 0.0 ? t.rest * exp(-(double)a.log_rest[row]) : 0.0;
  // s near tau lse, so that the difference that the exponential sees is small where p is not
  const float ref = (float)(lse / a.inv_tau), d2 = (float)((lse - (double)ref * a.inv_tau) * 1.4426950408889634), coef = (float)(scale * (t.total - tail));
  // listed ids of this chunk: their logits are read before any gradient is written (the two may be one buffer)
  const int id = tid < DISTILL_MAX_TOP ? t.id[tid] - base : -1;
  const bool mine = tid < DISTILL_MAX_TOP && t.id[tid] >= 0 && id >= 0 && id < n && !zero;
  float g_top = 0.f;
  if (mine) {
    double qj = 0.0;
    for (int j = 0; j < a.top; ++j) if (t.id[j] == t.id[tid]) qj += t.q[j];     // every entry of an id computes the same value
    g_top = (float)(scale * (t.total * exp((double)to_f(src[id]) * a.inv_tau - lse) - qj));
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < DISTILL_GRAD_VECS; ++k) {
    const int i = (k * DISTILL_GRAD_THREADS + tid) * VEC;
    float l[VEC], g[VEC];
    unpack_vec<T, VEC>(q[k], l);
#pragma unroll
    for (int e = 0; e < VEC; ++e) g[e] = zero ? 0.f : coef * ex2(fmaf(l[e] - ref, c2, -d2));
    if (i < n) store_vec<T, VEC>(dst, i, n, a.grad_vec, pack_vec<T, VEC>(g));
  }
  __syncthreads();
  if (mine) dst[id] = from_f<T>(g_top);
}
