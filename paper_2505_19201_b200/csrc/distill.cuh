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

// Two sums, products and both at once per instruction.
__device__ __forceinline__ unsigned long long pair_bits(float2 v) {
  unsigned long long u;
  asm("mov.b64 %0, {%1, %2};" : "=l"(u) : "f"(v.x), "f"(v.y));
  return u;
}
__device__ __forceinline__ float2 pair_of(unsigned long long u) {
  float2 v;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(u));
  return v;
}
__device__ __forceinline__ float2 add_pair(float2 a, float2 b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)));
  return pair_of(r);
}
__device__ __forceinline__ float2 mul_pair(float2 a, float2 b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)));
  return pair_of(r);
}
__device__ __forceinline__ float2 fma_pair(float2 a, float2 b, float2 c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)), "l"(pair_bits(c)));
  return pair_of(r);
}
// The largest of a vector's elements (NaN does not count).
template <typename T, int VEC> __device__ __forceinline__ float max_vec(const uint4 &q) {
  if constexpr (sizeof(T) == 4)
    return fmaxf(fmaxf(__uint_as_float(q.x), __uint_as_float(q.y)), fmaxf(__uint_as_float(q.z), __uint_as_float(q.w)));
  else {
    const __nv_bfloat162 *h = reinterpret_cast<const __nv_bfloat162 *>(&q);
    const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return fmaxf(__low2float(m), __high2float(m));
  }
}
__device__ __forceinline__ double warp_sum_d(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The teacher's side of a row: entry j belongs to thread j of the first DISTILL_TOP_WARPS warps.  Each warp leaves its sums relative to its
// own largest entry, and whoever needs the row's puts the four together.
#define DISTILL_TOP_WARPS (DISTILL_MAX_TOP / 32)
struct Entry {
  int id;                              // -1: no entry
  double x, e;                         // t / tau; e^(x - the warp's reference), with teacher_lse q itself
};
struct TeacherSums {                   // by warp: reference, sum of e, sum of e ln e (with teacher_lse) or e x
  double ref[DISTILL_TOP_WARPS], sum[DISTILL_TOP_WARPS], log[DISTILL_TOP_WARPS];
};
struct TeacherRow {
  double f[DISTILL_TOP_WARPS];         // q_j = e_j f of its warp
  double rest, total, shift;           // q_r; Q; sum q ln q = sum of f log, minus shift
  __device__ __forceinline__ double mine() const {
    double v = 0.0;
#pragma unroll
    for (int w = 0; w < DISTILL_TOP_WARPS; ++w) if (w == (int)(threadIdx.x >> 5)) v = f[w];
    return v;
  }
};
__device__ __forceinline__ Entry load_entry(const DistillArgs &a, int row) {
  const int j = threadIdx.x;
  Entry t = {-1, -INFINITY, 0.0};
  if (j < a.top) {
    const int id = a.ids[(long long)row * a.top + j];
    const float x = a.teacher[(long long)row * a.top + j];
    if (id >= 0 && id < a.vocab) { t.id = id; t.x = (double)x * a.inv_tau; }
  }
  return t;
}
// By the first DISTILL_TOP_WARPS warps.
__device__ __forceinline__ void teacher_sums(const DistillArgs &a, int row, Entry &t, TeacherSums &sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  double ref, y = t.x;
  if (a.teacher_lse) {
    ref = (double)a.teacher_lse[row];
    y = t.x - ref;
  } else {
    ref = t.x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ref = fmax(ref, __shfl_xor_sync(0xffffffffu, ref, o));
  }
  if (t.id >= 0 && t.x != -INFINITY) t.e = exp(t.x - ref);
  const double s = warp_sum_d(t.e), l = warp_sum_d(t.e == 0.0 ? 0.0 : t.e * y);
  if (lane == 0) { sh.ref[warp] = ref; sh.sum[warp] = s; sh.log[warp] = l; }
}
__device__ __forceinline__ TeacherRow teacher_row(const DistillArgs &a, const TeacherSums &sh) {
  TeacherRow r;
  double s = 0.0, m = -INFINITY;
#pragma unroll
  for (int w = 0; w < DISTILL_TOP_WARPS; ++w) {
    r.f[w] = 1.0;
    if (!a.teacher_lse) m = fmax(m, sh.ref[w]);
  }
#pragma unroll
  for (int w = 0; w < DISTILL_TOP_WARPS; ++w) {
    if (!a.teacher_lse && sh.ref[w] != m) r.f[w] = exp(sh.ref[w] - m);
    s += sh.sum[w] * r.f[w];
  }
  const bool any = !(s == 0.0);                             // a row with no valid entry has no loss, with or without the rest
  if (a.teacher_lse) {
    r.rest = any ? fmax(0.0, 1.0 - s) : 0.0;
    r.total = any ? s + r.rest : 0.0;
    r.shift = 0.0;
  } else {
#pragma unroll
    for (int w = 0; w < DISTILL_TOP_WARPS; ++w) r.f[w] = any ? r.f[w] / s : 0.0;
    r.rest = 0.0;
    r.total = any ? 1.0 : 0.0;
    r.shift = any ? m + log(s) : 0.0;
  }
  return r;
}

// A CTA's part in the row's sums, which are of 2^((l - m) ch), ch = log2(e) / tau.  (l ch - m ch in one instruction would overflow on rows
// masked with the type's lowest value.)
struct DistillPart {
  float m, unused;                     // largest logit, -inf without one
  double others, tops, qz;             // sums over the ids that are not listed, that are; sum of q_j z_j tau
};
struct DistillShared {
  DistillPart part[DISTILL_MAX_CLUSTER];
  TeacherSums teacher;
  double q[DISTILL_MAX_TOP], qz[DISTILL_TOP_WARPS], scale, total;
  float top_m[DISTILL_TOP_WARPS], top_s[DISTILL_TOP_WARPS], warp_m[32], warp_s[32], m, d, coef;
  int id[DISTILL_MAX_TOP], repeated;
  uint32_t bits[1];                    // one per id of this CTA's share: is it listed?
};
__host__ __device__ inline size_t distill_row_offset(int cta_elems) { return (sizeof(DistillShared) + (size_t)cta_elems / 8 + 15) / 16 * 16; }

// GRAD: the row stays in shared memory and its gradient leaves in the same pass.
#define DISTILL_THREADS 512
template <typename T, bool GRAD>
__global__ void __launch_bounds__(DISTILL_THREADS, 3)
k_distill(const __grid_constant__ DistillArgs a) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  DistillShared &sh = *reinterpret_cast<DistillShared *>(smem_raw);
  uint4 *vals = reinterpret_cast<uint4 *>(smem_raw + distill_row_offset(a.cta_elems));
  constexpr int VEC = 16 / sizeof(T), U = 4;
  cluster_started_arrive(a.cluster);
  kernel_entry(TR_k_distill);
  const int rank = a.cluster > 1 ? (int)cluster_ctarank() : 0, row = blockIdx.x / a.cluster, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5,
            nt = blockDim.x, nw = nt >> 5, base = rank * a.cta_elems, n = max(0, min(a.cta_elems, a.vocab - base));
  const T *src = (const T *)a.logits + row * a.ld + base;
  const float ch = (float)(a.inv_tau * 1.4426950408889634);
  const bool tail = a.teacher_lse != nullptr, top_warp = warp < DISTILL_TOP_WARPS;
  const int steps = (n + nt * VEC - 1) / (nt * VEC);
  uint4 q[U];
#pragma unroll
  for (int k = 0; k < U; ++k) q[k] = load_vec<T, VEC>(src, (k * nt + tid) * VEC, n, a.vec, -INFINITY);
  Entry t = {-1, -INFINITY, 0.0};
  if (top_warp) { t = load_entry(a, row); sh.id[tid] = t.id; }
  for (int i = tid; i < a.cta_elems / 32; i += nt) sh.bits[i] = 0;
  if (tid == 0) sh.repeated = 0;
  __syncthreads();
  const bool mine = top_warp && t.id >= base && t.id < base + n;
  float z = -INFINITY;
  if (mine) {
    const int i = t.id - base;
    z = to_f(src[i]);
    if (atomicOr(&sh.bits[i >> 5], 1u << (i & 31)) >> (i & 31) & 1u) sh.repeated = 1;
  }
  __syncthreads();
  bool first = mine;                                        // of the entries of one id the first stands for it
  if (mine && sh.repeated)
    for (int j = 0; j < tid; ++j) if (sh.id[j] == t.id) first = false;
  // running maximum m (ref: the same, 0 without one) and sum of 2^((l - ref) ch); listed ids stay out where the rest is a bucket
  float m = -INFINITY, ref = 0.f, s = 0.f, s1 = 0.f;
  for (int j0 = 0; j0 < steps; j0 += U) {
    if (j0) {
#pragma unroll
      for (int k = 0; k < U; ++k) q[k] = load_vec<T, VEC>(src, ((j0 + k) * nt + tid) * VEC, n, a.vec, -INFINITY);
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int i = ((j0 + k) * nt + tid) * VEC;
      if (i >= n) break;
      if (GRAD) vals[(j0 + k) * nt + tid] = q[k];
      float l[VEC], v;
      const uint32_t b = tail ? sh.bits[i >> 5] >> (i & 31) & ((1u << VEC) - 1u) : 0u;
      unpack_vec<T, VEC>(q[k], l);
      if (b) {
        v = -INFINITY;
#pragma unroll
        for (int e = 0; e < VEC; ++e) { if (b >> e & 1u) l[e] = -INFINITY; v = fmaxf(v, l[e]); }
      } else v = max_vec<T, VEC>(q[k]);
      if (v > m) {
        if (m > -INFINITY) { const float f = ex2((m - v) * ch); s *= f; s1 *= f; }
        m = ref = v;
      }
#pragma unroll
      for (int e = 0; e < VEC; e += 2) {
        const float2 y = mul_pair(add_pair(make_float2(l[e], l[e + 1]), make_float2(-ref, -ref)), make_float2(ch, ch));
        s += ex2(y.x); s1 += ex2(y.y);
      }
    }
  }
  if (top_warp) {
    teacher_sums(a, row, t, sh.teacher);
    const float tm = warp_max(z);
    const float ts = warp_sum(first ? ex2((z - (tm > -INFINITY ? tm : 0.f)) * ch) : 0.f);
    const double qz = warp_sum_d(mine && !(t.e == 0.0) ? t.e * (double)z : 0.0);
    if (lane == 0) { sh.top_m[warp] = tm; sh.top_s[warp] = ts; sh.qz[warp] = qz; }
  }
  {
    const float wm = warp_max(m);
    s = warp_sum((s + s1) * (m > -INFINITY ? ex2((m - wm) * ch) : 1.f));        // without a maximum 0, or NaN
    if (lane == 0) { sh.warp_m[warp] = wm; sh.warp_s[warp] = s; }
  }
  __syncthreads();
  cluster_started_wait(a.cluster);
  TeacherRow tr;
  if (top_warp) tr = teacher_row(a, sh.teacher);
  if (warp == 0) {
    const float wm = lane < nw ? sh.warp_m[lane] : -INFINITY, ws = lane < nw ? sh.warp_s[lane] : 0.f;
    const float tm = lane < DISTILL_TOP_WARPS ? sh.top_m[lane] : -INFINITY, ts = lane < DISTILL_TOP_WARPS ? sh.top_s[lane] : 0.f;
    const float cm = warp_max(fmaxf(wm, tm));
    const double others = warp_sum_d((double)(ws * (wm > -INFINITY ? ex2((wm - cm) * ch) : 1.f)));
    const double tops = warp_sum_d((double)(ts * (tm > -INFINITY ? ex2((tm - cm) * ch) : 1.f)));
    double qz = 0.0;
#pragma unroll
    for (int w = 0; w < DISTILL_TOP_WARPS; ++w) if (!(sh.qz[w] == 0.0)) qz += sh.qz[w] * tr.f[w];
    if (lane < a.cluster) {
      const uint32_t to = mapa_of(a.cluster, smem_u32(&sh.part[rank]), lane);
      st_cluster_u64(to, (unsigned long long)__float_as_uint(cm));
      st_cluster_u64(to + 8, __double_as_longlong(others));
      st_cluster_u64(to + 16, __double_as_longlong(tops));
      st_cluster_u64(to + 24, __double_as_longlong(qz));
    }
  }
  sync_all_of(a.cluster);
  // the row's sums, by each warp that needs them
  float rm = -INFINITY;
  double others = 0.0, tops = 0.0, qz = 0.0;
  if (warp == 0) {
    for (int c = 0; c < a.cluster; ++c) rm = fmaxf(rm, sh.part[c].m);
    for (int c = 0; c < a.cluster; ++c) {
      const DistillPart &p = sh.part[c];
      const double f = p.m > -INFINITY ? (double)ex2((p.m - rm) * ch) : 1.0;
      others += p.others * f; tops += p.tops * f; qz += p.qz;
    }
    if (!tail) tops = 0.0;                                  // they are among the others
  }
  const double total = others + tops;
  const bool none = total == 0.0;                           // no finite logit
  if (GRAD) {
    if (top_warp && mine) sh.q[tid] = t.e * tr.mine();
    if (tid == 0) {
      const double scale = none || tr.total == 0.0 ? 0.0 : (double)(a.row_scale ? a.row_scale[row] : 1.f) * a.inv_tau;
      sh.scale = scale;
      sh.m = none ? 0.f : rm; sh.d = log2f((float)total);
      sh.coef = scale == 0.0 ? 0.f : (float)(scale * (tr.total - (tr.rest > 0.0 && others > 0.0 ? tr.rest * (total / others) : 0.0)));
    }
    __syncthreads();
    const double scale = sh.scale;
    const float ref = sh.m, d = sh.d, coef = sh.coef;
    T *dst = (T *)a.grad + row * a.grad_ld + base;
    if (scale == 0.0) {                                     // padding: zeros, whatever the logits hold
      for (int i = tid * VEC; i < n; i += nt * VEC) store_vec<T, VEC>(dst, i, n, a.grad_vec, make_uint4(0u, 0u, 0u, 0u));
    } else {
      for (int j = 0; j < steps; ++j) {
        const int i = (j * nt + tid) * VEC;
        if (i >= n) break;
        float l[VEC], g[VEC];
        unpack_vec<T, VEC>(vals[j * nt + tid], l);
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
          const float2 y = fma_pair(add_pair(make_float2(l[e], l[e + 1]), make_float2(-ref, -ref)), make_float2(ch, ch), make_float2(-d, -d));
          const float2 o = mul_pair(make_float2(ex2(y.x), ex2(y.y)), make_float2(coef, coef));
          g[e] = o.x; g[e + 1] = o.y;
        }
        store_vec<T, VEC>(dst, i, n, a.grad_vec, pack_vec<T, VEC>(g));
      }
      __syncthreads();                                      // the listed ids' own gradients replace what was written
      if (first) {
        double qj = sh.q[tid];
        if (sh.repeated) {
          qj = 0.0;
          for (int j = 0; j < a.top; ++j) if (sh.id[j] == t.id) qj += sh.q[j];
        }
        dst[t.id - base] = from_f<T>((float)(scale * (tr.total * (double)ex2(fmaf(z - ref, ch, -d)) - qj)));
      }
    }
  }
  if (rank == 0 && tid == 0) {
    const double lse = (double)rm * a.inv_tau + log(total);
    double loss = -tr.shift - qz * a.inv_tau + (tr.total - tr.rest) * lse;
#pragma unroll
    for (int w = 0; w < DISTILL_TOP_WARPS; ++w) if (!(sh.teacher.log[w] == 0.0)) loss += sh.teacher.log[w] * tr.f[w];
    if (tail) {
      const double log_rest = others > 0.0 ? -log1p(tops / others) : others == 0.0 ? -INFINITY : others;
      if (tr.rest > 0.0) loss += tr.rest * (log(tr.rest) - log_rest);
      a.log_rest[row] = none ? -INFINITY : (float)log_rest;
    }
    a.loss[row] = (float)(tr.total == 0.0 ? 0.0 : none ? (double)INFINITY : loss);
    a.lse[row] = none ? -INFINITY : (float)lse;
  }
}

// The gradient from a saved log-sum-exp (and, with teacher_lse, log_rest).  A CTA walks `cta_elems` logits of a row, the next loads always on
// their way.
#define DISTILL_GRAD_THREADS 256
template <typename T>
__global__ void __launch_bounds__(DISTILL_GRAD_THREADS, 4)
k_distill_grad(const __grid_constant__ DistillArgs a) {
  __shared__ TeacherSums teacher;
  __shared__ double sq[DISTILL_MAX_TOP];
  __shared__ int sid[DISTILL_MAX_TOP];
  constexpr int VEC = 16 / sizeof(T), U = 4, STEP = DISTILL_GRAD_THREADS * VEC;
  kernel_entry(TR_k_distill_grad);
  const int parts = (a.vocab + a.cta_elems - 1) / a.cta_elems, row = blockIdx.x / parts, base = (blockIdx.x - row * parts) * a.cta_elems,
            n = min(a.cta_elems, a.vocab - base), tid = threadIdx.x;
  const T *src = (const T *)a.logits + row * a.ld + base;
  T *dst = (T *)a.grad + row * a.grad_ld + base;
  const float rs = a.row_scale ? a.row_scale[row] : 1.f;
  if (rs == 0.f || a.lse[row] == -INFINITY) {               // a row of padding is not read
    for (int i = tid * VEC; i < n; i += STEP) store_vec<T, VEC>(dst, i, n, a.grad_vec, make_uint4(0u, 0u, 0u, 0u));
    return;
  }
  uint4 q[2][U];
  auto fetch = [&](uint4 (&b)[U], int i0) {
#pragma unroll
    for (int k = 0; k < U; ++k) b[k] = load_vec<T, VEC>(src, i0 + (k * DISTILL_GRAD_THREADS + tid) * VEC, n, a.vec, -INFINITY);
  };
  fetch(q[0], 0);
  const double lse = (double)a.lse[row];
  Entry t = {-1, -INFINITY, 0.0};
  if (tid < DISTILL_MAX_TOP) {
    t = load_entry(a, row);
    teacher_sums(a, row, t, teacher);
  }
  __syncthreads();
  const TeacherRow tr = teacher_row(a, teacher);
  const double scale = tr.total == 0.0 ? 0.0 : (double)rs * a.inv_tau;
  const double tail = tr.rest > 0.0 ? tr.rest * exp(-(double)a.log_rest[row]) : 0.0;
  // logits relative to tau lse, so that the difference that the exponential sees is small where p is not
  const float ch = (float)(a.inv_tau * 1.4426950408889634), ref = (float)(lse / a.inv_tau),
              d = (float)((lse - (double)ref * a.inv_tau) * 1.4426950408889634), coef = (float)(scale * (tr.total - tail));
  const int id = t.id - base;
  const bool mine = t.id >= 0 && id >= 0 && id < n && scale != 0.0;
  float g_top = 0.f;
  if (tid < DISTILL_MAX_TOP) { sq[tid] = t.e * tr.mine(); sid[tid] = t.id; }
  __syncthreads();
  if (mine) {                                               // every entry of an id computes the same value
    double qj = 0.0;
    for (int j = 0; j < a.top; ++j) if (sid[j] == t.id) qj += sq[j];
    g_top = (float)(scale * (tr.total * exp((double)to_f(src[id]) * a.inv_tau - lse) - qj));
  }
  __syncthreads();                                          // before any gradient is written: the two may be one buffer
  auto turn = [&](const uint4 (&b)[U], int i0) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int i = i0 + (k * DISTILL_GRAD_THREADS + tid) * VEC;
      float l[VEC], g[VEC];
      unpack_vec<T, VEC>(b[k], l);
#pragma unroll
      for (int e = 0; e < VEC; e += 2) {
        const float2 y = fma_pair(add_pair(make_float2(l[e], l[e + 1]), make_float2(-ref, -ref)), make_float2(ch, ch), make_float2(-d, -d));
        const float2 o = mul_pair(make_float2(ex2(y.x), ex2(y.y)), make_float2(coef, coef));
        g[e] = o.x; g[e + 1] = o.y;
      }
      if (i < n) store_vec<T, VEC>(dst, i, n, a.grad_vec, pack_vec<T, VEC>(g));
    }
  };
  for (int i0 = 0; i0 < n; i0 += 2 * U * STEP) {
    if (i0 + U * STEP < n) fetch(q[1], i0 + U * STEP);
    turn(q[0], i0);
    if (i0 + 2 * U * STEP < n) fetch(q[0], i0 + 2 * U * STEP);
    if (i0 + U * STEP < n) turn(q[1], i0 + U * STEP);
  }
  __syncthreads();
  if (mine) dst[id] = from_f<T>(g_top);
}
